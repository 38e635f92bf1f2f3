"""The operators behind a kernel that lets its successor start early and writes (or reads) its data only then: a call must wait for
whatever runs before it on its stream, however that was launched.  The kernel in front is compiled here."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2502_16880_b200 import build, lmhead

pytestmark = pytest.mark.gpu

SOURCE = """
#include <cuda_runtime.h>
// Starts its successor, waits (bounded: about 100 us, 4096 turns at most), then copies.
__global__ void late_copy(unsigned char* to, const unsigned char* from, size_t bytes) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long begin = clock64();
    for (int i = 0; i < 4096 && clock64() - begin < 200000; ++i) __nanosleep(200);
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < bytes; i += (size_t)gridDim.x * blockDim.x) to[i] = from[i];
}
extern "C" int late_copy_launch(void* to, const void* from, size_t bytes, void* stream) {
    late_copy<<<32, 256, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<unsigned char*>(to), static_cast<const unsigned char*>(from), bytes);
    return cudaGetLastError() != cudaSuccess;
}
"""


@pytest.fixture(scope="module")
def late_copy(tmp_path_factory):
    folder = tmp_path_factory.mktemp("late_copy")
    src, lib = folder / "late_copy.cu", folder / "late_copy.so"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("NVCC", "nvcc"), *build.NVCC_FLAGS, "-o", str(lib), str(src)], check=True)
    launch = ctypes.CDLL(str(lib)).late_copy_launch
    launch.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]

    def copy(to, source):
        assert to.dtype == source.dtype and to.shape == source.shape and to.is_contiguous() and source.is_contiguous()
        n = to.numel() * to.element_size()
        assert launch(to.data_ptr(), source.data_ptr(), n, torch.cuda.current_stream().cuda_stream) == 0
    return copy


def _follows(late_copy, call, x, outs):
    """call() reads x and writes outs: the same whether x is there long before or written just in front of it, and what is in outs
    can still be read just in front of it."""
    new, old = x.clone(), x.flip(0).roll(1, -1).contiguous()
    call()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for _ in range(3):
        x.copy_(old)
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        late_copy(x, new)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    keep = torch.empty_like(outs[0])
    outs[0].zero_()
    torch.cuda.synchronize()
    late_copy(keep, outs[0])
    call()
    torch.cuda.synchronize()
    assert not keep.any() and all(torch.equal(o, w) for o, w in zip(outs, want))


def _weights(N, K, group, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8).cuda(),
            (0.01 + 0.01 * torch.rand(N, K // group, generator=g)).bfloat16().cuda())


@pytest.mark.parametrize("M,N,K", [(1, 4001, 4096), (1, 300, 8192), (2, 4001, 4096), (3, 500, 256), (3, 500, 4096), (8, 2000, 1024),
                                   (16, 300, 2048), (24, 5000, 512), (65, 3001, 4096)])
def test_product(late_copy, M, N, K):
    head = lmhead.Q4Linear(*_weights(N, K, 64))
    x = torch.randn(M, K, generator=torch.Generator().manual_seed(M)).bfloat16().cuda()
    out = torch.empty(M, N, device="cuda")
    _follows(late_copy, lambda: head.forward(x, out=out), x, [out])


def test_product_of_weights_just_written(late_copy):
    """Bytes written, packed and multiplied one behind the other."""
    Wq, scales = _weights(700, 1024, 32)
    head = lmhead.Q4Linear(Wq, scales)
    for M in (1, 8, 24):
        x, out = torch.randn(M, 1024, device="cuda").bfloat16(), torch.empty(M, 700, device="cuda")

        def call():
            lmhead.coral_lmhead_q4_pack(head.cfg, Wq, scales, None, head.packed)
            head.forward(x, out=out)
        _follows(late_copy, call, Wq, [out])


@pytest.mark.parametrize("M", [8, 16, 24, 60, 65])
def test_one_row_of_a_product_into_the_next(M):
    first, second = lmhead.Q4Linear(*_weights(2048, 512, 64)), lmhead.Q4Linear(*_weights(900, 2048, 128, 1))
    x = torch.randn(M, 512, generator=torch.Generator().manual_seed(M)).bfloat16().cuda()
    mid, out = torch.empty(M, 2048, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 900, device="cuda")
    first.forward(x, out=mid)
    torch.cuda.synchronize()
    second.forward(mid[M - 1:], out=out)
    torch.cuda.synchronize()
    want = out.clone()
    for _ in range(20):
        mid.zero_()
        first.forward(x, out=mid)
        second.forward(mid[M - 1:], out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("M", [1, 700])
def test_block_norm_and_its_gradient(late_copy, M):
    H = 1024
    x, r, dy, dh = (torch.randn(M, H, device="cuda").bfloat16() for _ in range(4))
    w = torch.rand(H, device="cuda").bfloat16()
    y, h, dx, dr = (torch.empty_like(x) for _ in range(4))
    d_post, d_pre = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    ws = torch.empty(lmhead.coral_lmhead_block_norm_backward_bytes(M, H), dtype=torch.uint8, device="cuda")
    _follows(late_copy, lambda: lmhead.coral_lmhead_block_norm(x, r, w, 1e-5, y, h, w_post=w), x, [y, h])
    _follows(late_copy, lambda: lmhead.coral_lmhead_block_norm_backward(x, r, w, 1e-5, dy, dh, ws, dx, dr, d_pre, w_post=w,
                                                                        out_dw_post=d_post), x, [dx, dr, d_pre, d_post])


@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("t", [torch.float32, torch.float16])
@pytest.mark.parametrize("M", [2, 300])
def test_logits(late_copy, M, t, lists):
    V, k = 20000, 10
    x = torch.randn(M, V, generator=torch.Generator().manual_seed(M)).to(t).cuda()
    out, ids = torch.empty_like(x), torch.empty(M, k, dtype=torch.int32, device="cuda")
    lps, lse = torch.empty(M, k, device="cuda"), torch.empty(M, device="cuda")
    kw = dict(row_seq=torch.zeros(M, dtype=torch.int32, device="cuda"), output_tokens=torch.arange(0, V, 7, dtype=torch.int32, device="cuda"),
              output_offsets=torch.tensor([0, (V + 6) // 7], device="cuda"), presence=torch.ones(1, device="cuda")) if lists else {}
    _follows(late_copy, lambda: lmhead.coral_lmhead_logits_process(x, out_logits=out, out_ids=ids, out_logprobs=lps, out_lse=lse, **kw),
             x, [out, ids, lps, lse])


def test_logits_with_a_list_just_written(late_copy):
    M, V = 2, 5000
    x = torch.randn(M, V, device="cuda")
    tokens = torch.randperm(V, generator=torch.Generator().manual_seed(1))[:600].int().cuda()
    out = torch.empty_like(x)
    kw = dict(output_tokens=tokens, output_offsets=torch.tensor([0, 250, 600], device="cuda"), presence=torch.ones(2, device="cuda"))
    _follows(late_copy, lambda: lmhead.coral_lmhead_logits_process(x, out_logits=out, **kw), tokens, [out])
