"""GPU parity of the 4-bit cache and of attention over it against the float64 oracle.

The cache is compared bit for bit with the oracle's codes (where a quotient is not within fp32 rounding of a border), read back with
one rounding.  Attention is tested on keys and values that 4 bits hold exactly: low + step * code with steps that are powers of two.

Tolerances.  u = 2^-24, additions in tensor cores 2 u.  A score is step (sum of q code) + low (sum of q) a group: with |low| + 15 step in the
place of |k| its products' absolute sum bounds it, e = 2 (D + 16) u times that and the scale.  p step is rounded to fp16: 2^-11 relative next
to codes of up to 15, and 2^-25 absolute of a scale that brings the largest step to one or more.  With n keys:
|out - want| <= (2 e + (4 n + 64) u) sum w (|low| + 15 step) + 2^-11 sum w 15 step + 2^-25 n 15 step_max, plus the output's rounding."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")
TYPES = [torch.bfloat16, torch.float16]


def _exact(g, T, n, D, group, t, spread=2):
    """Values that 4 bits hold exactly, each group with its lowest and highest code; sizes by token from 2^-spread to 2^spread."""
    codes = torch.randint(0, 16, (T, n, D // group, group), generator=g)
    ends = torch.rand(T, n, D // group, group, generator=g).argsort(-1)[..., :2]
    codes.scatter_(-1, ends, torch.tensor([0, 15]).expand(*ends.shape))
    step = 2.0 ** torch.randint(-spread - 3, spread - 2, (T, n, D // group, 1), generator=g)
    low = step * torch.randint(-20, 6, step.shape, generator=g)
    return (low + step * codes).view(T, n, D).to(t), (low.abs() + 15 * step).expand_as(codes).reshape(T, n, D).double().numpy(), step.expand_as(codes).reshape(T, n, D).double().numpy()


class Case:
    """Sequences on shuffled pages, n query rows each."""
    many = False

    def __init__(self, seed, lens, n, n_q, n_k, D, group, page, t, spread=2, ragged=False, tree=False, holes=True, values=_exact):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.t, self.D, self.n_q, self.n_k, self.page = lens, t, D, n_q, n_k, page
        self.n = n if isinstance(n, list) else [n] * len(lens)
        width = max(1, max(-(-x // page) for x in lens))
        pages = width * len(lens) + 2
        self.table = torch.randperm(pages, generator=g)[:width * len(lens)].view(len(lens), width).int()
        self.cache = lmhead.Kv4Cache(pages, page, n_k, D, group=group, dtype=t)
        if holes:
            self.cache.pages.fill_(255)                       # what nothing was stored to: steps and lowest values of NaN
        self.k, self.v, self.ksize, self.vsize, self.vstep = [], [], [], [], []
        for s, x in enumerate(lens):
            k, ks, _ = values(g, x, n_k, D, group, t, 1)
            v, vs, st = values(g, x, n_k, D, group, t, spread)
            j = torch.arange(x)
            k, v = ((a, a) if torch.is_tensor(a) else a for a in (k, v))     # what is stored, and what 4 bits make of it
            self.cache.store(k[0].cuda(), v[0].cuda(), (self.table[s].long()[j // page] * page + j % page).cuda())
            for into, what in zip((self.k, self.v, self.ksize, self.vsize, self.vstep), (k[1], v[1], ks, vs, st)):
                into.append(what.double().numpy() if torch.is_tensor(what) else what)
        rows = sum(self.n)
        self.q = torch.randn(rows, n_q, D, generator=g).to(t).cuda()
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(self.n)]), device="cuda") if isinstance(n, list) or ragged else None
        self.masks = None
        if tree:
            self.masks = [[sum(1 << b for b in range(i + 1) if b == i or torch.rand((), generator=g) < 0.5) for i in range(m)] for m in self.n]
            self.mask = torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for w in self.masks for x in w], device="cuda")

    def run(self, scale=None, table=None, lens=None, max_q=None, stream=None, out=None, lse=None):
        out = torch.full_like(self.q, 9.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 9.0, device="cuda") if lse is None else lse
        self.cache.attend(self.q, (self.table if table is None else table).cuda(), torch.tensor(self.lens if lens is None else lens, dtype=torch.int32).cuda(),
                          max_q=max(max(self.n), 1) if max_q is None else max_q, q_offsets=self.offsets, tree_mask=self.mask if self.masks else None, scale=scale,
                          out=out, out_lse=lse, stream=stream)
        return out, lse

    def check(self, got, scale=None, seen=None):
        assert self.cache.status() == 0
        out, lse = (x.double().cpu().numpy() for x in got)
        scale = self.D ** -0.5 if scale is None else scale
        q, a, half = self.q.double().cpu().numpy(), 0, torch.finfo(self.t).eps / 2
        for s, (x, n) in enumerate(zip(self.lens, self.n)):
            sees = (ao.tree(self.masks[s], n, x) if self.masks else ao.causal(n, x)) if seen is None else seen[s]
            w_out, w_lse, _, _, m = ao.attend(q[a:a + n], self.k[s], self.v[s], sees, scale)
            if x:
                ones, of = np.ones((n, 1, 1)), np.repeat(np.arange(self.n_k), self.n_q // self.n_k)
                e = 2 * ((2 if self.many else 1) * self.D + 16) * U * abs(scale) * (np.einsum("ihd,jhd->ihj", np.abs(q[a:a + n]), self.ksize[s][:, of]) * sees[:, None]).max(-1)[..., None]
                weigh = lambda size: ao.attend(q[a:a + n], self.k[s], size, sees, scale)[0]
                tol = (2 * e + (4 * m[:, None, None] + 64) * U) * weigh(self.vsize[s]) + 2.0 ** -11 * 15 * weigh(self.vstep[s])
                tol = tol + 2.0 ** -25 * 15 * m[:, None, None] * self.vstep[s].max() * ones
                if self.many:
                    tol = self.many_tol(e, m, weigh(self.vsize[s]), sees, self.vsize[s][:, of])
                tol = tol + half * (np.abs(w_out) + tol) + (2.0 ** -25 if self.t == torch.float16 else 0)
                off = np.abs(out[a:a + n] - w_out)
                assert np.all(off <= tol), (s, "out", float(np.max(off / tol)))
                none = m == 0
                off = np.abs(lse[a:a + n][~none] - w_lse[~none])
                tol = (e[..., 0] + (2 * m[:, None] + 64) * U)[~none] + 4 * U * np.abs(w_lse[~none])
                assert np.all(off <= tol), (s, "lse", float(np.max(off / tol)))
            none = m == 0
            assert np.all(out[a:a + n][none] == 0) and np.all(np.isneginf(lse[a:a + n][none]))
            a += n


# ---- tokens into the cache and back ---------------------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,n,D,group,page", [(1, 1, 64, 32, 16), (50, 2, 64, 64, 16), (33, 3, 128, 32, 48), (200, 8, 128, 64, 64), (77, 1, 128, 128, 256), (1000, 4, 64, 32, 32)])
def test_store_and_load(T, n, D, group, page, t):
    g = torch.Generator().manual_seed(T + D)
    pages = -(-T // page) + 1
    fused = (torch.randn(T, 3 * n, D, generator=g) * 4 + torch.randn(3 * n, D, generator=g)).to(t).cuda()
    fused[0, 0, :group] = 2.5                                 # a group of one value
    k, v = fused[:, :n], fused[:, 2 * n:]
    cache = lmhead.Kv4Cache(pages, page, n, D, group=group, dtype=t)
    slots = torch.randperm(pages * page, generator=g)[:T].cuda()
    cache.store(k, v, slots)
    got = cache.load(slots)
    for x, y in zip((k, v), got):
        low, step, codes, border = ao.held(x.double().cpu().numpy(), group, lambda s: torch.from_numpy(s).to(t).double().numpy())
        want = ao.stands_for(low, step, codes)
        half = torch.finfo(t).eps / 2
        off = np.abs(y.double().cpu().numpy() - want) > half * np.abs(want) + 2.0 ** -25
        assert not (off & (border.reshape(off.shape) > 2.0 ** -19)).any()
        assert np.all(np.abs(y.double().cpu().numpy() - x.double().cpu().numpy()) <= (np.broadcast_to(step, codes.shape).reshape(off.shape) * 0.54 + half * np.abs(want) + 2.0 ** -25))
    one = torch.full_like(got[0], 3.0)
    cache.load(slots, out_v=one)
    assert torch.equal(one, got[1])


def test_slots_outside_and_neighbours():
    g = torch.Generator().manual_seed(1)
    cache = lmhead.Kv4Cache(3, 32, 2, 64, group=32)
    k, v = (torch.randn(96, 2, 64, generator=g).bfloat16().cuda() for _ in range(2))
    cache.store(k, v, torch.arange(96, device="cuda"))
    before = cache.load(torch.arange(96, device="cuda"))
    other = torch.randn(6, 2, 64, generator=g).bfloat16().cuda()
    cache.store(other, other, torch.tensor([-1, 5, 96, 2 ** 40, 40, -2 ** 62], device="cuda"))
    after = cache.load(torch.arange(96, device="cuda"))
    keep = torch.ones(96, dtype=torch.bool)
    keep[[5, 40]] = False
    for a, b in zip(after, before):
        assert torch.equal(a[keep], b[keep]) and not torch.equal(a[5], b[5]) and not torch.equal(a[40], b[40])
    some = cache.load(torch.tensor([-1, 5, 96, 2 ** 33 + 5], device="cuda"))
    assert torch.equal(some[0][1], after[0][5]) and not some[0][[0, 2, 3]].any() and not some[1][[0, 2, 3]].any()
    cache.store(other[:0], other[:0], torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert cache.load(torch.zeros(0, dtype=torch.int64, device="cuda"))[0].shape == (0, 2, 64)


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_a_group_that_is_not_finite(bad):
    cache = lmhead.Kv4Cache(1, 16, 1, 64, group=32)
    x = torch.randn(3, 1, 64, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    slots = torch.tensor([3, 4, 9], device="cuda")
    cache.store(x, x, slots)
    want = cache.load(slots)
    y = x.clone()
    y[1, 0, 40] = bad
    cache.store(y, x, slots)
    k, v = cache.load(slots)
    assert k[1, 0, 32:].isnan().all() and torch.equal(v, want[1])
    k[1, 0, 32:] = want[0][1, 0, 32:]
    assert torch.equal(k, want[0])


def test_extreme_values():
    """Half a step, the step's rounding at 15 steps (2^-8 of them, or, among fp16's subnormals, 15 * 2^-25) and the result's rounding."""
    for t, top in ((torch.bfloat16, 3e38), (torch.float16, 65000.0)):
        cache = lmhead.Kv4Cache(1, 16, 1, 64, group=64, dtype=t)
        for a, b in ((0.0, top), (-top / 4, top / 4), (0.0, 1e-7), (-top, -top)):
            x = torch.linspace(a, b, 64).to(t).view(1, 1, 64).cuda()
            cache.store(x, x, torch.zeros(1, dtype=torch.int64, device="cuda"))
            k, v = cache.load(torch.zeros(1, dtype=torch.int64, device="cuda"))
            assert torch.equal(k, v) and k.isfinite().all()
            assert ((k.double() - x.double()).abs() <= (b - a) / 15 * 0.6 + 2.0 ** -8 * max(abs(a), abs(b)) + 16 * 2.0 ** -25).all()


# ---- attention ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("n_q,n_k", [(1, 1), (8, 2), (9, 1), (14, 2)])
def test_next_tokens(n_q, n_k, D, group, t):
    c = Case(D + group + n_q, [1, 15, 16, 17, 130, 0, 700], 1, n_q, n_k, D, group, 32, t)
    c.check(c.run())


@pytest.mark.parametrize("page", [16, 48, 64, 256, 1024])
def test_pages(page):
    c = Case(page, [300, 5, 1025], 2, 4, 2, 64, 32, page, torch.bfloat16)
    c.check(c.run())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,n_q,n_k", [(2, 4, 4), (3, 4, 1), (4, 8, 1), (17, 4, 2), (33, 4, 2), (60, 8, 2), (64, 4, 1), (150, 2, 1)])
def test_several_rows(n, n_q, n_k, t):
    c = Case(n, [n + 70, max(1, n // 2), n, 400], n, n_q, n_k, 64, 64, 32, t)       # one shorter than its queries: rows that see none
    c.check(c.run())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,D,group", [(1, 64, 32), (9, 128, 32), (60, 128, 64), (64, 64, 64)])
def test_trees(n, D, group, t):
    c = Case(n + 1, [n + 90, n, n + 1, 3, 333], n, 4, 2, D, group, 16, t, tree=True)
    c.check(c.run())


def test_ragged_rows():
    c = Case(3, [40, 7, 200, 0, 90], [3, 0, 20, 0, 1], 6, 2, 64, 32, 32, torch.bfloat16)
    got = c.run()
    c.check(got)
    c = Case(3, [40, 7, 200], [3, 5, 20], 6, 2, 64, 32, 32, torch.bfloat16)
    want = c.run()
    c.check(want)
    # rows from max_q on are left as they are; those in front of them mean what they meant (the work is cut otherwise: other roundings)
    out, lse = c.run(max_q=4)
    done = torch.tensor([True] * 3 + [True] * 4 + [False] + [True] * 4 + [False] * 16)
    assert (out[~done] == 9).all() and (lse[~done] == 9).all()
    for got, w in ((out, want[0]), (lse, want[1])):
        got[~done] = w[~done]
    c.check((out, lse))


@pytest.mark.parametrize("tree", [False, True])
def test_max_q_above_the_rows(tree):
    """A bound on the rows of a sequence larger than any has: other kernels and blocks without work, the same results up to rounding."""
    c = Case(17, [40, 0, 300, 7], [3, 0, 9, 1], 6, 2, 64, 32, 32, torch.bfloat16, tree=tree)
    for max_q in (9, 12, 64) + (() if tree else (1000, 100000)):
        c.check(c.run(max_q=max_q))


def test_many_sequences():
    g = torch.Generator().manual_seed(18)
    lens = [int(x) for x in torch.randint(0, 40, (3000,), generator=g)]
    c = Case(18, lens, 1, 2, 1, 64, 64, 16, torch.float16)
    c.check(c.run())


def test_long_caches_are_split():
    for lens, n in (([20000, 3], 1), ([9000], 12), ([33000], 1)):
        c = Case(len(lens), lens, n, 8, 2, 64, 64, 64, torch.bfloat16)
        c.check(c.run())


def test_table_wider_than_the_lengths_and_shorter():
    c = Case(4, [300, 40], 1, 4, 2, 64, 32, 16, torch.bfloat16)
    want = c.run()
    wide = torch.full((2, 500), -7, dtype=torch.int32)
    wide[:, :c.table.shape[1]] = c.table
    got = c.run(table=wide)                                    # split otherwise: the same up to rounding
    c.check(got)
    room = torch.full((2, 60), 10 ** 9, dtype=torch.int32)
    room[:, 7:7 + c.table.shape[1]] = c.table
    room = room.cuda()
    out = torch.empty_like(want[0])
    c.cache.attend(c.q, room[:, 7:7 + c.table.shape[1]], torch.tensor(c.lens, dtype=torch.int32).cuda(), out=out)
    assert torch.equal(out, want[0])
    long = c.run(lens=[10 ** 6, 40])                           # clamped to what the table has room for: the rest of the last page counts
    full = c.run(lens=[c.table.shape[1] * 16, 40])
    assert torch.equal(long[0].nan_to_num(), full[0].nan_to_num()) and torch.equal(long[0][1], want[0][1])


def test_pages_outside_hold_no_tokens():
    c = Case(5, [100, 64], 1, 4, 2, 64, 32, 16, torch.bfloat16)
    table, pages = c.table.clone(), c.cache.cfg.n_pages
    table[0, 2], table[0, 5], table[1, 0], table[1, 3] = -1, pages, 2 ** 31 - 1, -2 ** 31
    seen = [np.ones((1, 100), bool), np.ones((1, 64), bool)]
    seen[0][:, 32:48] = seen[0][:, 80:96] = seen[1][:, :16] = seen[1][:, 48:64] = False
    c.check(c.run(table=table), seen=seen)
    got = c.run(table=torch.full_like(table, -1))
    assert not got[0].any() and (got[1] == -INF).all()


@pytest.mark.parametrize("tree", [False, True])
def test_what_a_row_does_not_see_has_no_influence(tree):
    """Tokens that are not finite: seen by the rows from their own on (or those with their bit), unseen by the rest."""
    c = Case(6, [50, 40], 6, 4, 2, 64, 32, 16, torch.bfloat16, tree=tree)
    want = c.run()
    bad = torch.full((1, 2, 64), NAN, dtype=torch.bfloat16, device="cuda")
    good = torch.from_numpy(c.k[0][47:48]).bfloat16().cuda(), torch.from_numpy(c.v[0][47:48]).bfloat16().cuda()
    slot = (c.table[0, 47 // 16].long() * 16 + 47 % 16).view(1).cuda()
    see = (ao.tree(c.masks[0], 6, 50) if tree else ao.causal(6, 50))[:, 47]
    assert see.any() and not see.all()
    for k, v in ((bad, good[1]), (good[0], bad), (bad, bad)):
        c.cache.store(k, v, slot)
        out, lse = c.run()
        rows = np.flatnonzero(~see).tolist() + list(range(6, 12))
        assert torch.equal(out[rows], want[0][rows]) and torch.equal(lse[rows], want[1][rows])
        assert out[np.flatnonzero(see)].isnan().all()


@pytest.mark.parametrize("n,tree", [(1, False), (8, True), (40, True)])
def test_pages_beyond_32_bit_offsets(n, tree):
    """The same tokens on the last pages of a cache of 5 GB: the same bits, and read back from there."""
    c = Case(16, [n + 90, 600], n, 4, 2, 128, 32, 64, torch.bfloat16, tree=tree)
    want, pages = c.run(), 2 ** 18
    big = lmhead.Kv4Cache(pages, 64, 2, 128, group=32, dtype=torch.bfloat16)
    assert big.pages.numel() > 2 ** 32
    c.table += pages - c.cache.cfg.n_pages
    for s, x in enumerate(c.lens):
        j = torch.arange(x)
        slots = (c.table[s].long()[j // 64] * 64 + j % 64).cuda()
        k, v = (torch.from_numpy(a[s]).bfloat16().cuda() for a in (c.k, c.v))
        big.store(k, v, slots)
        assert all(torch.equal(a, b) for a, b in zip(big.load(slots), (k, v)))
    c.cache = big
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_steps_of_very_different_size():
    c = Case(7, [500], 1, 4, 2, 64, 32, 16, torch.bfloat16, spread=40)
    c.check(c.run())
    c = Case(8, [300, 9], 3, 4, 2, 128, 128, 16, torch.float16, spread=6)
    c.check(c.run())


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 2.0 ** 30, 2.0 ** 100])
def test_queries_of_any_size(size):
    c = Case(9, [130, 20], 1, 4, 2, 64, 64, 16, torch.bfloat16)
    c.q = (c.q.float() * size).bfloat16()
    c.check(c.run(scale=0.125 / size), scale=0.125 / size)


def test_scores_that_move_the_maximum_and_scales():
    c = Case(10, [600, 100], 2, 4, 1, 64, 32, 16, torch.bfloat16)
    for scale in (0.0, -0.3, 4.0, 1e-20):
        c.check(c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("t,power", [(torch.bfloat16, 40), (torch.bfloat16, 15), (torch.bfloat16, 52), (torch.float16, 11)])
@pytest.mark.parametrize("n,n_q,n_k", [(1, 4, 2), (5, 8, 2), (20, 8, 2)])
def test_scores_of_any_size(n, n_q, n_k, t, power):
    """Scores so far apart that one key has all the weight, above or below zero: its value, and its score as the log of the sum (products
    in two halves of the key: 4 D + 32 roundings of their absolute sum)."""
    for sign in (1, -1):
        c = Case(power + n, [200, 1000], n, n_q, n_k, 64, 64, 16, t)
        c.q = (sign * 2.0 ** power * c.q.abs().float()).to(t)
        for s in range(2):
            c.k[s] = np.abs(c.k[s])                            # all products of one sign: every score is far from zero
            j = torch.arange(c.lens[s])
            codes = torch.from_numpy(c.k[s])
            c.cache.store(codes.to(t).cuda(), torch.from_numpy(c.v[s]).to(t).cuda(), (c.table[s].long()[j // 16] * 16 + j % 16).cuda())
            slots = (c.table[s].long()[j // 16] * 16 + j % 16).cuda()
            c.k[s] = c.cache.load(slots)[0].double().cpu().numpy()
        out, lse = (x.double().cpu().numpy() for x in c.run(scale=1.0))
        q, of = c.q.double().cpu().numpy(), np.repeat(np.arange(n_k), n_q // n_k)
        for s, x in enumerate(c.lens):
            sc = np.einsum("ihd,jhd->ihj", q[s * n:s * n + n], c.k[s][:, of])
            sc = np.where(ao.causal(n, x)[:, None], sc, -np.inf)
            order = np.sort(sc, -1)
            off = (4 * 64 + 32) * U * np.abs(order[..., -1]) + 2 * np.abs(order[..., -1]) * torch.finfo(t).eps       # read back with one rounding
            clear = order[..., -1] - order[..., -2] > 2 * off + 40
            best = sc.argmax(-1)
            want = c.v[s][best, of[None]]
            got, g_lse = out[s * n:s * n + n], lse[s * n:s * n + n]
            assert np.isfinite(got).all() and np.isfinite(g_lse).all() and (power < 12 or n == 1 or clear.any())
            assert np.abs(got - want)[clear].max(initial=0) <= 2.0 ** -9 * np.abs(want).max()
            assert np.all(np.abs(g_lse - order[..., -1])[clear] <= off[clear] + 1e-6)


def test_a_bad_row_stays_in_its_row():
    c = Case(11, [100, 50], 3, 8, 2, 64, 32, 16, torch.bfloat16)
    want = c.run()
    for bad in (NAN, INF):
        keep = c.q.clone()
        c.q[1, 2, 7] = bad
        out, lse = c.run()
        ok = torch.ones(6, 8, dtype=torch.bool)
        ok[1, 2] = False
        assert torch.equal(out[ok], want[0][ok]) and torch.equal(lse[ok], want[1][ok]) and not (lse[1, 2].isfinite() and out[1, 2].isfinite().all())
        c.q = keep


def test_strides_and_new_outputs():
    c = Case(12, [100, 50], 3, 4, 2, 128, 64, 16, torch.bfloat16)
    want = c.run()
    fused = torch.full((6, 9, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    fused[:, 1:5] = c.q
    c.q = fused[:, 1:5]
    room = torch.full((6, 7, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    got = c.run(out=room[:, 2:6])
    assert torch.equal(got[0], want[0]) and (room[:, :2] == 3).all() and (room[:, 6:] == 3).all()
    table, lens = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda()
    assert torch.equal(c.cache.attend(c.q, table, lens, max_q=3), want[0])
    new = c.cache.attend(c.q, table, lens, max_q=3, q_offsets=torch.tensor([0, 3, 5], device="cuda"))
    assert torch.equal(new[:3], want[0][:3]) and not new[5].any()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert c.cache.attend(c.q[:0], table[:0], none).shape == (0, 4, 128)


def test_repeat_streams_graph_and_two_at_once():
    a, b = Case(13, [3000, 100], 1, 8, 2, 128, 128, 64, torch.bfloat16), Case(14, [90, 400, 30], 20, 4, 2, 64, 32, 16, torch.float16, tree=True)
    want = [x.run() for x in (a, b)]
    for _ in range(10):
        assert torch.equal(a.run()[0], want[0][0]) and torch.equal(b.run()[0], want[1][0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = [(x.q, x.table.cuda(), torch.tensor(x.lens, dtype=torch.int32).cuda()) for x in (a, b)]
    outs = [torch.zeros_like(x.q) for x in (a, b)]
    kw = [dict(max_q=1), dict(max_q=20, tree_mask=b.mask)]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, r, o, k, st in zip((a, b), args, outs, kw, streams):
            x.cache.attend(*r, out=o, stream=st, **k)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0][0]) and torch.equal(outs[1], want[1][0]) and a.cache.status() == 0 == b.cache.status()
    graphs = []
    for x, r, o, k in zip((a, b), args, outs, kw):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.cache.attend(*r, out=o, **k)
        graphs.append(g)
        o.zero_()
    torch.cuda.synchronize()
    for g, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            for _ in range(5):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0][0]) and torch.equal(outs[1], want[1][0])


def test_binding_refuses_wrong_tensors():
    c = Case(15, [40, 20], 2, 4, 2, 64, 32, 16, torch.bfloat16)
    table, lens = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda()
    call = lambda q=c.q, table=table, lens=lens, max_q=2, **kw: c.cache.attend(q, table, lens, max_q=max_q, **kw)
    for kw in (dict(q=c.q.half()), dict(q=c.q[:, :3]), dict(q=c.q[..., :32]), dict(table=table.long()), dict(table=table[:1]), dict(lens=lens.long()), dict(lens=c.lens),
               dict(max_q=0), dict(max_q=3), dict(scale=NAN), dict(q_offsets=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(q=c.q.cpu()),
               dict(q_offsets=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(tree_mask=torch.zeros(3, dtype=torch.int64, device="cuda")),
               dict(tree_mask=torch.zeros(4, dtype=torch.int32, device="cuda")), dict(out=torch.empty(4, 4, 64, device="cuda")),
               dict(out_lse=torch.empty(4, 3, device="cuda"))):
        with pytest.raises((ValueError, AttributeError, lmhead.CoralError)):
            call(**kw)
    x, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for args in ((x.half(), x, slots), (x, x[:2], slots), (x, x[..., :32], slots), (x, x, slots.int()), (x, x, slots[:2]), (x.cpu(), x, slots)):
        with pytest.raises((ValueError, lmhead.CoralError)):
            c.cache.store(*args)
    with pytest.raises(ValueError):
        lmhead.coral_lmhead_kv4_store(c.cache.cfg, c.cache.pages[:-256], x, x, slots)
    with pytest.raises(ValueError):
        lmhead.coral_lmhead_kv4_attention(c.cache.cfg, c.cache.pages, c.q, table, lens, torch.empty_like(c.q), 2, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        lmhead.Kv4Cache(1, 16, 1, 64, dtype=torch.float32)
    with pytest.raises(lmhead.CoralError):
        lmhead.Kv4Cache(1, 20, 1, 64)
