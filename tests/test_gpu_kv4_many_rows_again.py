"""Attention of many rows over the 4-bit cache where results are not finite, rightly or not, and where sums pass fp32's range on their way."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from tests.test_gpu_kv4 import _exact
from tests.test_gpu_kv4_many_rows import Many

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _spoil(c, s, j, cols):
    """Token j of sequence s gets NaN in some columns of its values."""
    v = torch.from_numpy(c.v[s][j:j + 1]).to(c.t).cuda()
    v[..., cols] = NAN
    k = torch.from_numpy(c.k[s][j:j + 1]).to(c.t).cuda()
    c.cache.store(k, v, (c.table[s, j // c.page].long() * c.page + j % c.page).view(1).cuda())


@pytest.mark.parametrize("lens,n,tree", [([300, 90], 40, True), ([300, 90], 40, False), ([6000, 900], 64, True)])
@pytest.mark.parametrize("at", [5, 200])
def test_rows_that_see_it_keep_the_rest_of_their_bits(at, lens, n, tree):
    """A value that is not finite in one group of columns, seen by all rows of its sequence: the other groups, and the other sequence, keep
    their bits (nothing is computed again)."""
    c = Many(at, lens, n, 4, 2, 64, 32, 16, torch.bfloat16, tree=tree, values=_exact)
    want, lse = c.run()
    _spoil(c, 0, at, 40)
    out, got_lse = c.run()
    assert torch.equal(got_lse, lse) and torch.equal(out[n:], want[n:])
    assert out[:n, :, 32:].isnan().all() and torch.equal(out[:n, :, :32], want[:n, :, :32])


@pytest.mark.parametrize("tree", [False, True])
def test_unseen_and_seen_at_once(tree):
    """One that all rows see, in one group, and one of the query tokens that some do not, in the other."""
    c = Many(3, [200], 48, 4, 2, 64, 32, 16, torch.bfloat16, tree=tree, values=_exact)
    want, lse = c.run()
    _spoil(c, 0, 7, 3)
    _spoil(c, 0, 180, 40)
    sees = torch.from_numpy((ao.tree(c.masks[0], 48, 200) if tree else ao.causal(48, 200))[:, 180])
    assert sees.any() and not sees.all()
    out, _ = c.run()
    assert out[..., :32].isnan().all() and out[sees][..., 32:].isnan().all() and out[~sees][..., 32:].isfinite().all()
    out[..., :32], out[sees] = want[..., :32], want[sees]
    c.check((out, lse))


def test_sums_beyond_the_range_on_their_way():
    """Values of 2^117: weights of up to 2^7 times them pass 2^128 in a sum of 300, the quotient does not."""
    def values(g, T, n_k, D, group, t, spread):
        x, size, step = _exact(g, T, n_k, D, group, t, 0)
        by = 2.0 ** 116 if spread == 2 else 1.0
        return (x.double() * by).to(t), size * by, step * by
    c = Many(4, [300, 90], 40, 4, 2, 64, 32, 16, torch.bfloat16, tree=True, values=values)
    assert max(np.abs(v).max() for v in c.v) > 2.0 ** 117
    c.check(c.run())
