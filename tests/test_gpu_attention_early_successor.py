"""The drafter's attention behind a kernel that lets its successor start early and writes (or reads) its data only then: a call waits for
whatever runs before it on its stream, however that was launched."""
import pytest
import torch

from paper_2502_16880_b200 import lmhead
from tests.test_gpu_early_successor import _follows, late_copy  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _rnd(*s, t=torch.bfloat16, seed=0):
    return torch.randn(*s, generator=torch.Generator().manual_seed(seed)).to(t).cuda()


@pytest.mark.parametrize("T", [1, 900])
def test_qk_rotate_and_its_gradient(late_copy, T):  # noqa: F811
    q, k, dq, dk = _rnd(T, 8, 64), _rnd(T, 2, 64, seed=1), _rnd(T, 8, 64, seed=2), _rnd(T, 2, 64, seed=3)
    pos, f, w = torch.arange(T, device="cuda").int(), torch.rand(32, device="cuda"), torch.rand(64, device="cuda").bfloat16()
    a, b, c, d = (torch.empty_like(x) for x in (q, k, dq, dk))
    w1, w2 = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    ws = torch.empty(lmhead.coral_lmhead_qk_rotate_backward_bytes(T, 8, 2, 64), dtype=torch.uint8, device="cuda")
    _follows(late_copy, lambda: lmhead.coral_lmhead_qk_rotate(q, k, pos, f, a, b, w_q=w, w_k=w), q, [a, b])
    _follows(late_copy, lambda: lmhead.coral_lmhead_qk_rotate_backward(q, k, pos, f, dq, dk, c, d, w_q=w, w_k=w, dw_q=w1, dw_k=w2, workspace=ws), dq, [c, d, w1, w2])
    if T > 1:
        _follows(late_copy, lambda: lmhead.coral_lmhead_qk_rotate(q, k, pos, f, a, b), pos, [a, b])


@pytest.mark.parametrize("lens", [[3], [500, 20, 700]])
def test_prompt_attention(late_copy, lens):  # noqa: F811
    T = sum(lens)
    q, k, v = _rnd(T, 4, 128), _rnd(T, 2, 128, seed=1), _rnd(T, 2, 128, seed=2)
    off = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device="cuda")
    out, lse = torch.empty_like(q), torch.empty(T, 4, device="cuda")
    for x in (v, q):
        _follows(late_copy, lambda: lmhead.coral_lmhead_prompt_attention(q, k, v, off, out, out_lse=lse), x, [out, lse])


@pytest.mark.parametrize("length,n_seq", [(40, 2), (5000, 1)])
def test_cache(late_copy, length, n_seq):  # noqa: F811
    width = -(-length // 16)
    cache = lmhead.Kv4Cache(width * n_seq, 16, 2, 64, group=32)
    T = width * 16 * n_seq
    k, v, q = _rnd(T, 2, 64), _rnd(T, 2, 64, seed=1), _rnd(n_seq, 4, 64, seed=2)
    slots, got = torch.arange(T, device="cuda"), [torch.empty(T, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table, lens = torch.arange(width * n_seq, device="cuda").int().view(n_seq, width), torch.full((n_seq,), length, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n_seq, 4, device="cuda")
    _follows(late_copy, lambda: (cache.store(k, v, slots), cache.load(slots, *got)), k, got)
    _follows(late_copy, lambda: cache.attend(q, table, lens, out=out, out_lse=lse), cache.pages, [out, lse])

    def step():
        cache.store(k, v, slots)
        cache.attend(q, table, lens, out=out, out_lse=lse)
    _follows(late_copy, step, v, [out, lse])
