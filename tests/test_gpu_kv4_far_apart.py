"""GPU parity of attention over the 4-bit cache where values lie very far apart: a token that a row does not see, a token that it sees with next to
no weight, or a group of columns, 2^8 to 2^100 times the rest.  Each row, and each of its groups of columns, is as exact as without them.

Values are ones that 4 bits hold exactly (a power of two times those of test_gpu_kv4).  Tolerances, u = 2^-24, e a score's error as there.
Up to 32 rows of a key head: p step is rounded to fp16, 2^-11 relative next to codes of up to 15, and where it is subnormal 2^-25 absolute of a scale
that brings the row's and group's own largest p step to 2^6 or more: 2^-31 of that one.  With w the weights, n of them:
|out - want| <= (2 e + (4 n + 64) u) sum w (|low| + 15 step) + 2^-11 sum w 15 step + 2^-31 15 n max(w step), plus the output's rounding.
More rows: the tolerances of test_gpu_kv4_many_rows, which go by a column's own values."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from tests.test_gpu_kv4 import Case, TYPES, U, _exact
from tests.test_gpu_kv4_many_rows import Many

pytestmark = pytest.mark.gpu
# The largest power, and how many powers below 2^-3 the ordinary steps are (fp16: steps of 2^-11 and 2^9).
BIG, SMALL = {torch.bfloat16: 100, torch.float16: 20}, {torch.bfloat16: 0, torch.float16: 8}


def _scaled(where, far, keys=False, small=0):
    """_exact times 2^-small, and where(by, f) sets the factor by [T, 1, groups, 1] of some of the values (or keys) to f, 2^far times that."""
    def values(g, T, n, D, group, t, spread):
        x, size, step = _exact(g, T, n, D, group, t, 0)
        by = torch.full((T, 1, D // group, 1), 2.0 ** -small)
        if (spread == 1) == keys and T:
            where(by, 2.0 ** (far - small))
        by = by.expand(T, n, D // group, group).reshape(T, n, D)
        return (x.double() * by).to(t), size * by.double().numpy(), step * by.double().numpy()
    return values


def _weights(q, k, sees, scale):
    of = np.repeat(np.arange(k.shape[1]), q.shape[1] // k.shape[1])
    s = np.einsum("ihd,jhd->ihj", q, k[:, of]) * scale
    s = np.where(sees[:, None], s, -np.inf)
    w = np.exp(s - s.max(-1, keepdims=True))
    return w / w.sum(-1, keepdims=True), s.max(-1) + np.log(w.sum(-1)), of


def _check(c, got, scale=None):
    """Every row that sees something, by what it sees itself."""
    assert c.cache.status() == 0
    out, lse = (x.double().cpu().numpy() for x in got)
    scale = c.D ** -0.5 if scale is None else scale
    q, a, half = c.q.double().cpu().numpy(), 0, torch.finfo(c.t).eps / 2
    for s, (x, n) in enumerate(zip(c.lens, c.n)):
        sees = ao.tree(c.masks[s], n, x) if c.masks else ao.causal(n, x)
        w, w_lse, of = _weights(q[a:a + n], c.k[s], sees, scale)
        e = 2 * (c.D + 16) * U * abs(scale) * (np.einsum("ihd,jhd->ihj", np.abs(q[a:a + n]), c.ksize[s][:, of]) * sees[:, None]).max(-1)[..., None]
        m = sees.sum(1)[:, None, None]
        sum_of = lambda v: np.einsum("ihj,jhd->ihd", w, v[:, of])
        want, step = sum_of(c.v[s]), c.vstep[s][:, of].transpose(1, 0, 2)
        most = np.stack([(w[:, h, :, None] * step[h][None]).max(1) for h in range(len(of))], 1)
        tol = (2 * e + (4 * m + 64) * U) * sum_of(c.vsize[s]) + 2.0 ** -11 * 15 * sum_of(c.vstep[s]) + 2.0 ** -31 * 15 * m * most
        tol = tol + half * (np.abs(want) + tol) + (2.0 ** -25 if c.t == torch.float16 else 0)
        off = np.abs(out[a:a + n] - want)
        assert np.all(off <= tol), (s, "out", float(np.max(off / tol)))
        off = np.abs(lse[a:a + n] - w_lse)
        tol = e[..., 0] + (2 * m[..., 0] + 64) * U + 4 * U * np.abs(w_lse)
        assert np.all(off <= tol), (s, "lse", float(np.max(off / tol)))
        a += n


ROWS = [(2, 4, 4), (2, 4, 1), (5, 2, 2), (8, 8, 2), (16, 2, 1)]      # query tokens, query heads, key heads: 2 to 32 rows of a key head


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,n_q,n_k", ROWS)
@pytest.mark.parametrize("tree", [False, True])
def test_tokens_that_a_row_does_not_see(n, n_q, n_k, tree, t):
    for far in (8, 24, BIG[t]):
        def last(by, f):
            by[-1] = f
            by[-max(1, n // 2)] = f
        c = Case(far, [200, n + 20, 3000], n, n_q, n_k, 64, 32, 16, t, tree=tree, values=_scaled(last, min(far, BIG[t]), small=SMALL[t]))
        _check(c, c.run())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,group", [(64, 64), (128, 32), (128, 64), (128, 128)])
def test_groups_of_columns(D, group, t):
    for n, n_q, n_k in ROWS:
        def first(by, f):
            by[:, :, 0] = f
            by[3::7, :, -1] = f
        c = Case(n + D, [70, 1200], n, n_q, n_k, D, group, 32, t, values=_scaled(first, BIG[t], small=SMALL[t]))
        _check(c, c.run())


@pytest.mark.parametrize("n,n_q,n_k", [(1, 4, 1)] + ROWS)
@pytest.mark.parametrize("lens", [[300, 90], [20000]])
def test_tokens_seen_with_next_to_no_weight(lens, n, n_q, n_k):
    """Values 2^60 times the others, of weights about 2^-55, 2^-100, 2^-200 and none: queries above zero, keys of -2 to -32 there."""
    at, keys = [1, 2, 40, 77], torch.tensor([-2.0, -4.0, -8.0, -32.0])

    def some(by, f):
        by[at] = f
    c = Case(n, lens, n, n_q, n_k, 64, 64, 16, torch.bfloat16, values=_scaled(some, 60))
    c.q = c.q.abs() + 0.25
    for s, x in enumerate(lens):
        c.k[s][at] = keys.view(-1, 1, 1).numpy()                # groups of one value
        c.ksize[s][at] = -keys.view(-1, 1, 1).numpy()
        j = torch.arange(x)
        c.cache.store(torch.from_numpy(c.k[s]).to(c.t).cuda(), torch.from_numpy(c.v[s]).to(c.t).cuda(), (c.table[s].long()[j // 16] * 16 + j % 16).cuda())
    _check(c, c.run(scale=0.25), scale=0.25)


@pytest.mark.parametrize("n,n_q,n_k", [(8, 8, 2), (2, 4, 1)])
def test_rows_are_the_same_bits_whatever_they_do_not_see(n, n_q, n_k):
    """A token that some rows see, at ordinary and at very large values: the others keep their bits."""
    c = Case(3, [230], n, n_q, n_k, 64, 32, 16, torch.bfloat16)
    slot = (c.table[0, 229 // 16].long() * 16 + 229 % 16).view(1).cuda()
    want = c.run()
    for far in (2.0 ** 20, 2.0 ** 90):
        c.cache.store(torch.from_numpy(c.k[0][229:]).to(c.t).cuda(), (torch.from_numpy(c.v[0][229:]) * far).to(c.t).cuda(), slot)
        got = c.run()
        assert torch.equal(got[0][:-1], want[0][:-1]) and torch.equal(got[1][:-1], want[1][:-1])
        assert not torch.equal(got[0][-1], want[0][-1])

@pytest.mark.parametrize("n,n_q,n_k,lens", [(40, 4, 2, [100, 300]), (64, 2, 1, [4000])])
@pytest.mark.parametrize("far", [30, -60, 100])
def test_groups_of_columns_with_many_rows(far, n, n_q, n_k, lens):
    """Values of one group of columns 2^far times those of the next; keys 2^20 apart, with queries that make up for it."""
    def first(by, f):
        by[:, :, 0] = f
    c = Many(far + 200, lens, n, n_q, n_k, 64, 32, 16, torch.bfloat16, tree=True, values=_scaled(first, far))
    c.check(c.run())
    power = 20 if far > 0 else -20
    c = Many(far + 201, lens, n, n_q, n_k, 64, 32, 16, torch.bfloat16, tree=True, values=_scaled(first, power, keys=True))
    c.q[..., :32] = (c.q[..., :32].float() * 2.0 ** -power).to(c.t)
    c.check(c.run())
