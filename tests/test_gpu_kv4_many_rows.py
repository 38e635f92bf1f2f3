"""GPU parity of attention of many rows (33 and more of a key head) over the 4-bit cache against the float64 oracle.

Values are ordinary ones: what the cache holds of them (low + step code) needs more bits than the type has.  A quotient within fp32's
rounding of a border between two codes is moved away from it, so that the oracle knows the codes.

Tolerances, u = 2^-24.  A key enters as two fp16 numbers, its score as 2 D products: e = 2 (2 D + 16) u times the products' absolute sum.
Weights and values are rounded to fp16, 2^-12 each, a value by at most 2^-13 of its token's largest more where it is far below the step's; and
a weight by at most 2^-22 of the largest:
|out - want| <= (2 e + (4 n + 64) u + 2^-11 + 2^-12) sum w (|low| + 15 step) + 2^-22 sum (|low| + 15 step), plus the output's rounding."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from tests.test_gpu_kv4 import Case, INF, NAN, TYPES, U, _exact

pytestmark = pytest.mark.gpu


def _ordinary(g, T, n, D, group, t, spread):
    x = (torch.randn(T, n, D, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g) * 0.5) + torch.randn(n, D, generator=g)).to(t)
    if T == 0:
        return _exact(g, T, n, D, group, t, spread)
    to = lambda s: torch.from_numpy(s).to(t).double().numpy()
    for _ in range(2):
        low, step, codes, border = ao.held(x.double().numpy(), group, to)
        near = torch.from_numpy(border < 2.0 ** -17).view(T, n, -1, group)
        x = torch.where(near, torch.from_numpy(low).to(t), x.view(T, n, -1, group)).view(T, n, D)
    low, step, codes, border = ao.held(x.double().numpy(), group, to)
    assert border.min() >= 2.0 ** -17
    size = np.broadcast_to(np.abs(low) + 15 * step, codes.shape).reshape(T, n, D)
    return (x, torch.from_numpy(ao.stands_for(low, step, codes))), size, np.broadcast_to(step, codes.shape).reshape(T, n, D)


class Many(Case):
    many = True

    def __init__(self, *args, values=_ordinary, **kw):
        super().__init__(*args, values=values, **kw)
        assert max(self.n) * self.n_q // self.n_k >= 33

    def many_tol(self, e, m, weighed, sees, size):
        return (2 * e + (4 * m[:, None, None] + 64) * U + 2.0 ** -11 + 2.0 ** -12) * weighed + 2.0 ** -22 * np.einsum("ij,jhd->ihd", sees.astype(float), size)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("n,n_q,n_k,tree", [(33, 2, 2, True), (60, 8, 2, True), (64, 6, 1, True), (35, 2, 2, False), (150, 4, 2, False), (9, 12, 3, False)])
def test_rows(n, n_q, n_k, tree, D, group, t):
    c = Many(n + D + group, [n + 1, n, 64, 65, n // 2, 0, n + 300], n, n_q, n_k, D, group, 32, t, tree=tree)
    c.check(c.run())


def test_ragged_rows():
    c = Many(1, [40, 7, 200, 0, 90, 130], [33, 0, 20, 0, 1, 70], 6, 2, 64, 32, 32, torch.bfloat16)
    c.check(c.run())
    c = Many(1, [40, 70, 200], [33, 64, 20], 6, 2, 64, 32, 32, torch.bfloat16, tree=True)
    c.check(c.run())


@pytest.mark.parametrize("page", [16, 48, 256, 1024])
def test_pages(page):
    c = Many(page, [300, 50, 1025], 40, 4, 2, 64, 32, page, torch.bfloat16)
    c.check(c.run())


@pytest.mark.parametrize("lens,n,tree", [([20000, 70], 20, True), ([9000], 64, True), ([5000, 4999, 100], 130, False)])
def test_long_caches_are_split(lens, n, tree):
    c = Many(len(lens), lens, n, 8, 2, 128, 64, 64, torch.bfloat16, tree=tree)
    c.check(c.run())


@pytest.mark.parametrize("tree", [False, True])
def test_what_a_row_does_not_see_has_no_influence(tree):
    c = Many(2, [90, 200], 40, 4, 2, 64, 32, 16, torch.bfloat16, tree=tree)
    bad = torch.full((1, 2, 64), NAN, dtype=torch.bfloat16, device="cuda")
    at = 77
    see = (ao.tree(c.masks[0], 40, 90) if tree else ao.causal(40, 90))[:, at]
    assert see.any() and not see.all()
    slot = (c.table[0, at // 16].long() * 16 + at % 16).view(1).cuda()
    want = c.run()
    rows = torch.from_numpy(np.concatenate([see, np.zeros(40, bool)]))
    one = torch.ones_like(bad)
    for k, v in ((bad, one), (one, bad), (bad, bad)):
        c.cache.store(k, v, slot)
        out, lse = c.run()
        assert out[rows].isnan().all()
        out[rows], lse[rows] = want[0][rows], want[1][rows]
        c.check((out, lse))


@pytest.mark.parametrize("t,far", [(torch.bfloat16, 60), (torch.bfloat16, -60), (torch.bfloat16, 14), (torch.float16, -9), (torch.float16, 8)])
@pytest.mark.parametrize("lens,n", [([100, 300], 40), ([4000], 64)])
def test_tokens_of_very_different_size(lens, n, t, far):
    """Tokens 2^far times the others, in the tree or (values) in front of it too, where every row sees them."""
    for which, where in (("k", [-5, -30]), ("v", [-5, -30]), ("v", [3, 40, -5])):
        def values(g, T, n_k, D, group, t, spread):
            x, size, step = _exact(g, T, n_k, D, group, t, 0)
            if (spread == 1) == (which == "k"):
                by = torch.ones(T, 1, 1)
                by[where] = 2.0 ** far
                x, size, step = (x.float() * by).to(t), size * by.double().numpy(), step * by.double().numpy()
            return x, size, step
        c = Many(far + 100, lens, n, 4, 2, 64, 64, 16, t, tree=True, values=values)
        c.check(c.run())


def test_values_of_zero():
    def values(g, T, n_k, D, group, t, spread):
        x, size, step = _exact(g, T, n_k, D, group, t, 0)
        if spread == 2:
            x[:130], size[:130], step[:130] = 0, 0, 0
        return x, size, step
    for lens in ([300, 100], [40, 130], [2000]):
        c = Many(3, lens, 36, 4, 2, 128, 64, 16, torch.bfloat16, tree=True, values=values)
        c.check(c.run())


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -20, 2.0 ** 30, 2.0 ** 100])
def test_queries_of_any_size(size):
    c = Many(4, [130, 50], 34, 4, 2, 64, 64, 16, torch.bfloat16)
    c.q = (c.q.float() * size).bfloat16()
    c.check(c.run(scale=0.125 / size), scale=0.125 / size)


def test_scores_that_move_the_maximum_and_scales():
    c = Many(5, [600, 100], 36, 4, 1, 64, 32, 16, torch.bfloat16, tree=True)
    for scale in (0.0, -0.3, 4.0, 1e-20):
        c.check(c.run(scale=scale), scale=scale)


def test_a_bad_row_stays_in_its_row():
    c = Many(6, [100, 50], 34, 8, 2, 64, 32, 16, torch.bfloat16)
    want = c.run()
    for bad in (NAN, INF, -INF):
        keep = c.q.clone()
        c.q[1, 2, 7] = bad
        out, lse = c.run()
        ok = torch.ones(68, 8, dtype=torch.bool)
        ok[1, 2] = False
        assert torch.equal(out[ok], want[0][ok]) and torch.equal(lse[ok], want[1][ok]) and not (lse[1, 2].isfinite() and out[1, 2].isfinite().all())
        c.q = keep


def test_pages_outside_hold_no_tokens():
    c = Many(7, [100, 64], 17, 4, 2, 64, 32, 16, torch.bfloat16)
    table, pages = c.table.clone(), c.cache.cfg.n_pages
    table[0, 2], table[0, 5], table[1, 0], table[1, 3] = -1, pages, 2 ** 31 - 1, -2 ** 31
    seen = [ao.causal(17, 100), ao.causal(17, 64)]
    seen[0][:, 32:48] = seen[0][:, 80:96] = seen[1][:, :16] = seen[1][:, 48:64] = False
    c.check(c.run(table=table), seen=seen)
    got = c.run(table=torch.full_like(table, -1))
    assert not got[0].any() and (got[1] == -INF).all()


def test_rows_from_max_q_on_and_strides():
    c = Many(8, [100, 200], [60, 40], 4, 2, 128, 64, 16, torch.bfloat16)
    want = c.run()
    out, lse = c.run(max_q=50)
    done = torch.tensor([True] * 50 + [False] * 10 + [True] * 40)
    assert (out[~done] == 9).all() and (lse[~done] == 9).all()
    out[~done], lse[~done] = want[0][~done], want[1][~done]
    c.check((out, lse))
    fused = torch.full((100, 9, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    fused[:, 1:5] = c.q
    c.q = fused[:, 1:5]
    room = torch.full((100, 7, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    got = c.run(out=room[:, 2:6])
    assert torch.equal(got[0], want[0]) and (room[:, :2] == 3).all() and (room[:, 6:] == 3).all()


def test_repeat_streams_graphs_and_two_at_once():
    a, b = Many(9, [3000, 100], 60, 8, 2, 128, 128, 64, torch.bfloat16, tree=True), Many(10, [90, 400, 80], 70, 4, 2, 64, 32, 16, torch.float16)
    want = [x.run() for x in (a, b)]
    for _ in range(10):
        assert torch.equal(a.run()[0], want[0][0]) and torch.equal(b.run()[0], want[1][0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = [(x.q, x.table.cuda(), torch.tensor(x.lens, dtype=torch.int32).cuda()) for x in (a, b)]
    outs = [torch.zeros_like(x.q) for x in (a, b)]
    kw = [dict(max_q=60, tree_mask=a.mask), dict(max_q=70)]
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
