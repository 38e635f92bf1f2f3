"""Prompt attention where rows are computed again, or must not be: values that are not finite, seen and unseen, sums that pass fp32's range on their
way, and scores beyond 2^22, over several turns of a block and long prompts.  Tolerances and oracle as in test_gpu_prompt_attention."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prompt_attention import INF, NAN, _close, _make, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("D,n_q,n_k", [(64, 2, 1), (128, 4, 4), (72, 7, 1)])
@pytest.mark.parametrize("lens,at", [([300, 40], 5), ([1500, 700, 9], 200), ([3000], 0)])
def test_rows_that_see_it_keep_the_rest_of_their_bits(lens, at, D, n_q, n_k, bad):
    """An early value that is not finite in one column: of the rows that see it the other columns keep their bits (nothing is computed again:
    the result is what that value makes of it), and the rows in front of it stay what they were."""
    d = _make(D + at, lens, lens, n_q, n_k, D, torch.bfloat16)
    want, want_lse = _run(d)
    clean = d["v"].clone()
    d["v"][at, :, 3] = bad
    out, lse = _run(d)
    assert torch.equal(lse, want_lse) and torch.equal(out[lens[0]:], want[lens[0]:])
    seen, rest = out[at:lens[0]], [c for c in range(D) if c != 3]
    assert not seen[..., 3].isfinite().any() and torch.equal(seen[..., rest], want[at:lens[0]][..., rest])
    out[at:lens[0], :, 3] = want[at:lens[0], :, 3]
    _close(dict(d, v=clean), (out, lse), rows={0: list(range(0, at, 7))})


def test_unseen_and_seen_at_once():
    """Values that are not finite early on (seen) and in the last steps of some rows (unseen): each row by what it sees."""
    lens, D = [400], 64
    d = _make(2, lens, lens, 4, 1, D, torch.bfloat16)
    want, lse = _run(d)
    clean = d["v"].clone()
    d["v"][10, :, 3], d["v"][200, :, 7], d["v"][399, :, 9] = NAN, INF, NAN
    out, got_lse = _run(d)
    assert torch.equal(got_lse, lse)
    for col, at in ((3, 10), (7, 200), (9, 399)):
        assert not out[at:, :, col].isfinite().any() and out[:at, :, col].isfinite().all()
        out[at:, :, col] = want[at:, :, col]
    _close(dict(d, v=clean), (out, lse))


def test_sums_beyond_the_range_on_their_way():
    """Values of 2^120 and scores that rise by 2^7 in weight from the first steps to the last: the weighted sum passes 2^128, its quotient does not."""
    lens, D = [150], 64
    d = _make(4, lens, lens, 1, 1, D, torch.bfloat16)
    d["q"], d["k"] = torch.ones_like(d["q"]), torch.zeros_like(d["k"])
    d["k"][70:, :, 0] = 7.0                                     # behind the reference that the first step sets, by less than what moves it
    d["v"] = (torch.rand(d["v"].shape, generator=torch.Generator().manual_seed(1)) + 0.5).bfloat16().cuda() * 2.0 ** 120
    _close(d, _run(d, 0.6931471805599453), 0.6931471805599453)


@pytest.mark.parametrize("t,power", [(torch.bfloat16, 30), (torch.float16, 11)])
@pytest.mark.parametrize("lens,n", [([1200, 700, 65], 16), ([9 + i % 17 for i in range(200)], 8)])
def test_far_scores_over_several_turns(lens, n, t, power):
    """More tiles than SMs, up to 128 sequences and more: rows of scores beyond 2^22 come out as those of their sequence alone."""
    d = _make(power, lens, lens, n, n, 64, t)
    d["q"] = (d["q"].float() * 2.0 ** power).to(t)
    d["k"] = (d["k"].float() * 2.0 ** (power if t == torch.float16 else 0)).to(t)
    out, lse = _run(d, 1.0)
    assert out.isfinite().all() and lse.isfinite().all() and (lse.abs() > 2.0 ** 22).any()
    for s in range(0, len(lens), max(1, len(lens) // 12)):
        a = sum(lens[:s])
        at = slice(a, a + lens[s])
        alone = _run(dict(q=d["q"][at], k=d["k"][at], v=d["v"][at], lens=[lens[s]], k_lens=[lens[s]]), 1.0)
        assert torch.equal(alone[0], out[at]) and torch.equal(alone[1], lse[at])


def test_an_infinity_early_in_a_long_prompt():
    """All rows of a long fp16 prompt see an infinity: they are computed again while nothing waits, so the status stays 0 (asserted by every run)."""
    lens, D = [12000], 64
    d = _make(6, lens, lens, 4, 1, D, torch.float16)
    clean = d["v"].clone()
    want = _run(d)
    d["v"][3, :, 5] = INF
    out, lse = _run(d)
    assert torch.equal(lse, want[1]) and (out[3:, :, 5] == INF).all()
    out[:, :, 5] = want[0][:, :, 5]
    _close(dict(d, v=clean), (out, lse), rows={0: [0, 2, 3, 4, 127, 128, 6000, 11999]})
