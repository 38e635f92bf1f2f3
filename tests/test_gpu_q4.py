"""GPU parity of the product with 4-bit weights against the float64 oracle.

Tolerance.  u = 2^-24.  Integers and activations are exact operands; one MMA step adds 16 products and the running sum, each
kept to at least 24 bits below the largest of them, so a step is off by at most 17 u of the sizes it adds and a group of g
columns by 17 g / 16 u.  The sums run over q x and z x apart, whose sizes together are at most (15 + z) / max(|q - z|) times the
size of (q - z) x a column; a whole group's sizes are added up here as they are ("parts" below).  The activations' own sum adds
g / 8 + 8 roundings, the groups add K / g, the split of the columns at most 16 more, the zero point and the scale 2.
Then one rounding to the output type.
"""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oor
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _make(seed, M, N, K, group, zeros, xt, st):
    g = torch.Generator().manual_seed(seed)
    Wq = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand(N, K // group, generator=g)) * 0.01).to(st)
    z = torch.randint(0, 16, (N, K // group), generator=g, dtype=torch.uint8) if zeros else None
    return Wq, scales, z, torch.randn(M, K, generator=g).to(xt)


def _linear(Wq, scales, z):
    return lmhead.Q4Linear(Wq.cuda(), scales.cuda(), None if z is None else z.cuda())


def _check(got, Wq, scales, z, x, group):
    want, size = oor.q4_linear(Wq.numpy(), scales.double().numpy(), None if z is None else z.numpy(), x.double().numpy())
    K = x.shape[1]
    q = oor.q4_unpack(Wq.numpy()).astype(np.float64) + (8.0 if z is None else np.repeat(z.numpy().astype(np.float64), group, axis=1))
    parts = np.abs(x.double().numpy()) @ (q * np.repeat(np.abs(scales.double().numpy()), group, axis=1)).T
    tol = (17 * group / 16 + group / 8 + K / group + 26) * U * parts
    tol = tol + torch.finfo(got.dtype).eps / 2 * (np.abs(want) + tol) + (2.0 ** -25 if got.dtype == torch.float16 else 0)
    off = np.abs(got.double().cpu().numpy() - want)
    assert np.all(off <= tol), float(np.max(off / tol))


@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_types_groups_and_row_counts(xt, group, zeros):
    for i, (M, N, K) in enumerate([(1, 1, group), (2, 17, 3 * group), (8, 500, 1024), (9, 129, 5 * 128), (16, 4001, 256), (61, 48, 384),
                                   (150, 33, 7 * group)]):
        st = [torch.bfloat16, torch.float16][i % 2]
        Wq, s, z, x = _make(i * 7 + group, M, N, K, group, zeros, xt, st)
        lin = _linear(Wq, s, z)
        for ot in (torch.float32, xt) if i else (torch.float32, torch.bfloat16, torch.float16):
            _check(lin.forward(x.cuda(), out_dtype=ot), Wq, s, z, x, group)


@pytest.mark.parametrize("M", [1, 2, 7, 8, 13, 16, 17, 31, 33, 60, 64, 65])
def test_wide_products(M):
    """Column splits over many warps, several passes over the rows, more tiles than the device holds at once."""
    for N, K, group in [(3000, 4096, 128), (40000, 512, 64), (100, 8192, 32)]:
        Wq, s, z, x = _make(M, M, N, K, group, M % 2 == 0, torch.bfloat16, torch.bfloat16)
        _check(_linear(Wq, s, z).forward(x.cuda()), Wq, s, z, x, group)


def test_longest_columns():
    for M, K in [(1, 65536), (3, 28672), (10, 14336)]:
        Wq, s, z, x = _make(K, M, 40, K, 128, True, torch.float16, torch.float16)
        _check(_linear(Wq, s, z).forward(x.cuda()), Wq, s, z, x, 128)


@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [1, 8, 16, 24, 60])
def test_whole_numbers_are_exact(M, xt):
    """Small integers and scales that are powers of two: every sum is exact, so a wrong or missing term shows."""
    g = torch.Generator().manual_seed(M)
    N, K, group = 300, 1152, 32
    Wq = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    s = (2.0 ** torch.randint(-2, 3, (N, K // group), generator=g).float()).to(xt)
    z = torch.randint(0, 128, (N, K // group), generator=g, dtype=torch.uint8)
    x = torch.randint(-4, 5, (M, K), generator=g).to(xt)
    got = _linear(Wq, s, z).forward(x.cuda())
    want, _ = oor.q4_linear(Wq.numpy(), s.double().numpy(), z.numpy(), x.double().numpy())
    assert np.array_equal(got.double().cpu().numpy(), want)
    # one column at a time lands where it belongs
    for col in (0, 1, 5, 37, K - 1):
        e = torch.zeros(M, K, dtype=xt)
        e[M - 1, col] = 1
        got = _linear(Wq, s, z).forward(e.cuda()).double().cpu().numpy()
        want, _ = oor.q4_linear(Wq.numpy(), s.double().numpy(), z.numpy(), e.double().numpy())
        assert np.array_equal(got, want), col


def test_a_bad_row_stays_in_its_row():
    Wq, s, z, x = _make(3, 20, 200, 256, 64, True, torch.bfloat16, torch.bfloat16)
    clean = _linear(Wq, s, z).forward(x.cuda())
    x[11, 7] = float("nan")
    x[2, 9] = float("inf")
    got = _linear(Wq, s, z).forward(x.cuda())
    assert torch.all(torch.isnan(got[11])) and not torch.any(torch.isfinite(got[2]))
    keep = [m for m in range(20) if m not in (2, 11)]
    assert torch.equal(got[keep], clean[keep])


def test_repeat_streams_graph_and_neighbours():
    Wq, s, z, x = _make(4, 24, 1003, 512, 128, False, torch.bfloat16, torch.float16)
    lin, x = _linear(Wq, s, z), x.cuda()
    first = lin.forward(x)
    assert torch.equal(first, lin.forward(x))
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty_like(first) for _ in streams]
    torch.cuda.synchronize()
    for st, o in zip(streams, outs):                        # the same packed copy on several streams at once
        lin.forward(x, out=o, stream=st)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)
    big = torch.full((26, 1003), 5.0, device="cuda")
    lin.forward(x, out=big[1:25])                            # rows before and behind stay as they were
    assert torch.equal(big[1:25], first) and torch.all(big[0] == 5) and torch.all(big[25] == 5)
    out = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lin.forward(x, out=out)
    x.mul_(-2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first * -2)                      # a power of two scales every sum exactly


def test_binding_refuses_wrong_tensors():
    Wq, s, z, x = _make(5, 4, 64, 256, 64, True, torch.bfloat16, torch.bfloat16)
    lin = _linear(Wq, s, z)
    x = x.cuda()
    for bad in [x.float(), x[:, :128].contiguous(), x.cpu(), x.t()]:
        with pytest.raises((ValueError, lmhead.CoralError)):
            lin.forward(bad, out=torch.empty(4, 64, device="cuda"))
    for out in [torch.empty(4, 63, device="cuda"), torch.empty(3, 64, device="cuda"), torch.empty(4, 64, device="cuda", dtype=torch.int32)]:
        with pytest.raises((ValueError, lmhead.CoralError)):
            lin.forward(x, out=out)
    with pytest.raises((ValueError, lmhead.CoralError)):     # a group of 16 columns
        lmhead.Q4Linear(Wq.cuda(), torch.ones(64, 16, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        lmhead.Q4Linear(Wq.cuda(), s.float().cuda())
    with pytest.raises(ValueError):
        lmhead.Q4Linear(Wq.cuda(), s.cuda(), z[:, :2].contiguous().cuda())


def test_status_of_a_workspace():
    """Calls of many rows leave their status in the workspace, the others have none."""
    Wq, s, z, x = _make(6, 33, 300, 512, 64, False, torch.bfloat16, torch.bfloat16)
    lin, x = _linear(Wq, s, z), x.cuda()
    n = lmhead.coral_lmhead_q4_workspace_bytes(lin.cfg, 33)
    assert n > 0 and lmhead.coral_lmhead_q4_workspace_bytes(lin.cfg, 1) == 0
    out = torch.empty(33, 300, device="cuda")
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    lmhead.coral_lmhead_q4_linear(lin.cfg, lin.packed, x, out, ws)
    assert lmhead.coral_lmhead_q4_status(ws) == 0
    _check(out, Wq, s, z, x.cpu(), 64)
    for bad in (None, torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8)):
        with pytest.raises((ValueError, lmhead.CoralError)):
            lmhead.coral_lmhead_q4_linear(lin.cfg, lin.packed, x, out, bad)


@pytest.mark.parametrize("M,N,K,group", [(33, 4001, 37 * 64, 64), (60, 38001, 2048, 128), (18, 70000, 1056, 32), (130, 257, 4096, 128),
                                         (64, 16 * 148 * 16, 256, 64)])
def test_left_over_passes_split_by_columns(M, N, K, group):
    """Whole passes, left-over ones in parts of unequal size, a last part that ends inside a block of columns, no left-over pass."""
    Wq, s, z, x = _make(M + N, M, N, K, group, True, torch.bfloat16, torch.float16)
    lin, xc = _linear(Wq, s, z), x.cuda()
    got = lin.forward(xc)
    _check(got, Wq, s, z, x, group)
    for _ in range(3):
        assert torch.equal(lin.forward(xc), got)
    _check(lin.forward(xc, out_dtype=torch.bfloat16), Wq, s, z, x, group)


@pytest.mark.parametrize("M", [1, 3, 8, 16, 24, 60])
def test_rows_of_any_size(M):
    """A row is scaled by a power of two before it becomes fp16, so rows times a power of two give outputs times that power, bit for
    bit, from the smallest bf16 numbers to the largest.  (Weight scales near 2^-10 keep the largest outputs finite; those below
    2^-126 are rounded at 2^-150.)"""
    N, K, group = 75, 1024, 64
    Wq, s, z, x = _make(50 + M, M, N, K, group, M % 2 == 0, torch.bfloat16, torch.bfloat16)
    s, x = (s / 8).bfloat16(), ((x * 16).round() / 16).bfloat16()             # (few bits, so that they stay exact below 2^-126 too)
    lin = _linear(Wq, s, z)
    base = lin.forward(x.cuda()).double().cpu()
    for k in (-118, -100, -87, -60, 60, 86, 100, 116, 120, 124):
        scaled = (x.double() * 2.0 ** k).bfloat16()
        assert torch.equal(scaled.double(), x.double() * 2.0 ** k)
        got = lin.forward(scaled.cuda()).double().cpu()
        assert torch.all((got - base * 2.0 ** k).abs() <= (2.0 ** -150 if k < -100 else 0)), k
    # the very smallest, and the largest beside ordinary ones, row by row
    tiny = (torch.randint(-127, 128, (M, K), generator=torch.Generator().manual_seed(M)).double() * 2.0 ** -133).bfloat16()
    ones = (tiny.double() * 2.0 ** 133).bfloat16()
    got, want = lin.forward(tiny.cuda()).double().cpu(), lin.forward(ones.cuda()).double().cpu() * 2.0 ** -133
    assert torch.all((got - want).abs() <= 2.0 ** -150)
    big = torch.full((K,), torch.finfo(torch.bfloat16).max).bfloat16() * torch.where(torch.arange(K) % 3 == 0, 1.0, -0.5).bfloat16()
    mixed = x.clone()
    mixed[M - 1] = big
    got = lin.forward(mixed.cuda())
    assert torch.all(torch.isfinite(got)) and torch.equal(got[:M - 1].double().cpu(), base[:M - 1])
    _check(got[M - 1:], Wq, s, z, big[None], group)
    mixed[M - 1] = 0
    assert not lin.forward(mixed.cuda())[M - 1].any()


@pytest.mark.parametrize("xt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M", [1, 8, 24])
def test_small_activations_beside_a_large_one(M, xt):
    """Activations become fp16 numbers (every second column's divided by 16) under a power of two that brings the row's largest to
    2^14..2^15.  A value of 2^-24 of the largest is then at least 2^-10, an exact operand of 11 bits; a smaller one is off by half a
    subnormal step, 2^-25, times 16: 2^-35 of the largest.  The large value stands at a weight of zero, the small ones in columns
    of one parity at a time or alone; scales are powers of two, so an output of one column is exact but for the operand."""
    N, K, group = 48, 128, 32
    g = torch.Generator().manual_seed(M)
    q = torch.randint(1, 16, (N, K), generator=g)
    q[:, 40] = 0
    Wq = (q[:, 0::2] | q[:, 1::2] << 4).to(torch.uint8)
    s, z = torch.full((N, K // group), 0.25).to(xt), torch.zeros(N, K // group, dtype=torch.uint8)
    lin = _linear(Wq, s, z)
    weight = q.double() * 0.25
    for top in (2.0 ** 14, 2.0 ** 15 - 16, 2.0 ** 14 * 1.5):
        top = torch.tensor(top).to(xt)
        largest = float(top)
        for power in (-9, -10, -11, -12, -14, -16, -20, -24):                  # of the small values; fp16 holds no smaller ones
            v = ((1 + torch.rand(M, K, generator=g)) * 2.0 ** power * torch.where(torch.rand(M, K, generator=g) < 0.5, -1, 1)).to(xt)
            for cols in [list(range(p, K, 2)) for p in (0, 1)] + [[c] for c in range(8)]:
                x = torch.zeros(M, K, dtype=xt)
                x[:, cols] = v[:, cols]
                x[:, 40] = top
                got = lin.forward(x.cuda()).double().cpu()
                small = x.double()
                small[:, 40] = 0
                want, size = small @ weight.T, small.abs() @ weight.T
                exact = small.abs().amax() == 0 or float(small[small != 0].abs().min()) >= 2.0 ** -24 * largest
                off = 0 if exact else 2.0 ** -35 * largest * weight[:, cols].sum(1)
                rounding = 0 if len(cols) == 1 else (17 * group / 16 + group / 8 + K / group + 26) * U * size
                assert torch.all((got - want).abs() <= off + rounding), (power, cols[:2])


def test_status_of_the_last_product():
    Wq, s, z, x = _make(7, 130, 900, 1024, 64, True, torch.bfloat16, torch.bfloat16)
    lin, x, st = _linear(Wq, s, z), x.cuda(), torch.cuda.Stream()
    lin.forward(x)
    assert lin.status() == 0
    for M in (1, 8, 17, 64, 130):
        out = torch.empty(M, 900, device="cuda")
        torch.cuda.synchronize()
        lin.forward(x[:M], out=out, stream=st)
        assert lin.status(st) == 0                           # (the stream has been waited for)
        _check(out, Wq, s, z, x[:M].cpu(), 64)


@pytest.mark.parametrize("M", [1, 40])
def test_a_new_output_belongs_to_the_stream_that_writes_it(M):
    """Memory that the current stream still has work on must not become the output of a call on another stream, and that output's
    memory must not be written there while the current stream still reads it."""
    Wq, s, z, x = _make(8, M, 3000, 256, 64, False, torch.bfloat16, torch.bfloat16)
    lin, x = _linear(Wq, s, z), x.cuda()
    want = lin.forward(x)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for dtype in (torch.float32, torch.bfloat16):
        old = [torch.empty_like(want, dtype=dtype) for _ in range(4)]
        torch.cuda._sleep(20_000_000)                        # ~10 ms before the current stream writes to it
        for o in old:
            o.fill_(9)
        del old, o
        out = lin.forward(x, out_dtype=dtype, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(out, want.to(dtype))
        torch.cuda._sleep(20_000_000)
        copy = out.clone()                                   # read late, freed before
        del out
        with torch.cuda.stream(st):
            new = [torch.full_like(want, 7, dtype=dtype) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(copy, want.to(dtype))
        del new


def test_status_waits_for_a_call_on_another_stream():
    Wq, s, z, x = _make(9, 40, 300, 512, 64, False, torch.bfloat16, torch.bfloat16)
    lin, x, st = _linear(Wq, s, z), x.cuda(), torch.cuda.Stream()
    out = torch.empty(40, 300, device="cuda")
    n = lmhead.coral_lmhead_q4_workspace_bytes(lin.cfg, 40)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(st):
            junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]    # what the scratch holds at first
            del junk
            torch.cuda._sleep(20_000_000)
        lin.forward(x, out=out, stream=st)
        assert lin.status() == 0
    _check(out, Wq, s, z, x.cpu(), 64)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lin.forward(x, out=out)
    g.replay()
    assert lin.status() == 0
