"""Attention of several rows over the 4-bit cache (warp and tensor-core kernel, whole and split caches) behind a kernel that lets its successor start
early and writes one of its arguments only then: every one of them is waited for, the small ones too."""
import pytest
import torch

from paper_2502_16880_b200 import lmhead
from tests.test_gpu_early_successor import _follows, late_copy  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("max_q", [5, 15, 20, 60])
@pytest.mark.parametrize("lens", [[100, 75, 130], [5000, 4100, 2600]])
def test_rows(late_copy, lens, max_q, tree):  # noqa: F811
    n_seq, g = len(lens), torch.Generator().manual_seed(max_q)
    width = -(-max(lens) // 16)
    T, rows = width * 16 * n_seq, max_q * n_seq
    rnd = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()
    cache = lmhead.Kv4Cache(width * n_seq, 16, 2, 64, group=32)
    cache.store(rnd(T, 2, 64), rnd(T, 2, 64), torch.arange(T, device="cuda"))
    q, table = rnd(rows, 4, 64), torch.randperm(width * n_seq, generator=g).int().view(n_seq, width).cuda()
    lens, offsets = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.arange(n_seq + 1, device="cuda") * max_q
    mask = torch.randint(0, 2 ** 62, (rows,), generator=g).cuda()
    out, lse = torch.empty_like(q), torch.empty(rows, 4, device="cuda")

    def call():
        cache.attend(q, table, lens, max_q=max_q, q_offsets=offsets, tree_mask=mask if tree else None, out=out, out_lse=lse)
    for late in (cache.pages, q, table, lens, offsets) + ((mask,) if tree else ()):
        _follows(late_copy, call, late, [out, lse])
    assert cache.status() == 0
