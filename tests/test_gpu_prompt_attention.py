"""GPU parity of prompt attention against the float64 oracle.

Tolerances.  u = 2^-24; tensor cores add with truncation, 2 u an addition.  A score of D products is off by e = 2 (D + 8) u times the sum of their
absolute values (times the scale); that shifts its weight, and the sum of all weights, by e relative.  A weight is rounded to the
type, eps / 2 relative (fp16 also 2^-25 absolute next to a largest weight of at least one); n of them and their products are added
up in fp32, 4 n u.  So an output is within (eps / 2 + 2 e + (4 n + 64) u) sum w |v| of the oracle's, plus its own rounding, and the
log-sum-exp within e + (2 n + 64) u + 4 u |lse|."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


def _offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64), device="cuda")


def _make(seed, lens, k_lens, n_q, n_k, D, t, q_scale=1.0, extra_rows=0):
    g = torch.Generator().manual_seed(seed)
    T, Tk = sum(lens) + extra_rows, sum(k_lens) + extra_rows
    return dict(q=(torch.randn(T, n_q, D, generator=g) * q_scale).to(t).cuda(), k=(torch.randn(Tk, n_k, D, generator=g) + torch.randn(n_k, D, generator=g)).to(t).cuda(),
                v=torch.randn(Tk, n_k, D, generator=g).to(t).cuda(), lens=lens, k_lens=k_lens)


def _run(d, scale=None, **kw):
    out = torch.full(d["q"].shape, 9.0, dtype=d["q"].dtype, device="cuda")
    lse = torch.full(d["q"].shape[:2], 9.0, device="cuda")
    ws = lmhead.coral_lmhead_prompt_attention(d["q"], d["k"], d["v"], _offsets(d["lens"]), out, k_offsets=_offsets(d["k_lens"]), scale=scale, out_lse=lse, **kw)
    if ws is not None:
        assert lmhead.coral_lmhead_attention_status(ws) == 0
    return out, lse


def _close(d, got, scale=None, rows=None):
    """rows: {sequence: rows of it}; all if None."""
    out, lse = (x.double().cpu().numpy() for x in got)
    t = d["q"].dtype
    half, D = torch.finfo(t).eps / 2, d["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    q, k, v = (d[n].double().cpu().numpy() for n in "qkv")
    a = b = 0
    for s, (nq, nk) in enumerate(zip(d["lens"], d["k_lens"])):
        at = np.arange(nq) if rows is None else np.asarray(rows.get(s, []), int)
        with np.errstate(invalid="ignore"):
            w_out, w_lse, vsize, ssize, n = ao.attend(q[a:a + nq][at], k[b:b + nk], v[b:b + nk], ao.causal(nq, nk)[at], scale)
        e = 2 * (D + 8) * U * ssize[..., None]
        tiny = 2.0 ** -25 * n[:, None, None] * (np.abs(v[b:b + nk]).max() if nk else 0) if t == torch.float16 else 0
        tol = (half + 2 * e + (4 * n[:, None, None] + 64) * U) * vsize + tiny
        tol = tol + half * (np.abs(w_out) + tol) + (2.0 ** -25 if t == torch.float16 else 0)
        off = np.abs(out[a:a + nq][at] - w_out)
        assert np.all(off <= tol), (s, "out", float(np.max(off / np.maximum(tol, 1e-300))))
        none = n == 0
        assert np.all(np.isneginf(lse[a:a + nq][at][none]))
        off = np.abs(lse[a:a + nq][at][~none] - w_lse[~none])
        tol = (e[..., 0] + (2 * n[:, None] + 64) * U)[~none] + 4 * U * np.abs(w_lse[~none])
        assert np.all(off <= tol), (s, "lse", float(np.max(off / tol)))
        a, b = a + nq, b + nk


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n_q,n_k,D", [(4, 2, 128), (3, 1, 64), (2, 2, 72), (7, 1, 16), (8, 1, 8), (12, 4, 120), (32, 1, 64)])
def test_heads_and_columns(n_q, n_k, D, t):
    d = _make(D + n_q, [37, 1, 150], [37, 1, 150], n_q, n_k, D, t)
    _close(d, _run(d))


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
def test_lengths_about_the_tiles(n, G, t):
    d = _make(n, [n], [n], G, 1, 64, t)
    _close(d, _run(d))


@pytest.mark.parametrize("nq,nk", [(1, 700), (5, 133), (40, 128), (64, 385), (130, 131), (3, 2), (20, 1), (5, 0), (200, 70), (300, 150)])
def test_keys_from_before_and_rows_that_see_none(nq, nk):
    d = _make(nq + nk, [nq, 3], [nk, 9], 4, 2, 128, torch.bfloat16)
    got = _run(d)
    _close(d, got)
    if nk < nq:
        assert not got[0][:nq - nk].any() and (got[1][:nq - nk] == -INF).all()


def test_long_rows():
    d = _make(3, [2900], [5000], 2, 1, 128, torch.bfloat16)
    _close(d, _run(d), rows={0: [0, 1, 127, 128, 1500, 2771, 2898, 2899]})


def test_many_and_empty_sequences():
    lens = [(7 * i) % 5 for i in range(700)]                 # more sequences than a block has threads, a fifth of them empty
    k_lens = [n + (i % 3) for i, n in enumerate(lens)]
    d = _make(4, lens, k_lens, 2, 1, 64, torch.float16)
    _close(d, _run(d))


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_scores_that_move_the_maximum(t):
    """Keys that grow along the sequence, by more than 2^8 in weight from tile to tile, and some that fall."""
    d = _make(5, [700], [700], 2, 1, 64, t)
    d["k"] = (d["k"].float() * torch.linspace(0.1, 12, 700, device="cuda")[:, None, None]).to(t)
    _close(d, _run(d, 0.5), 0.5)
    d["k"] = d["k"].flip(0).contiguous()
    _close(d, _run(d, 0.5), 0.5)
    d["q"] = (d["q"].float() * 30).to(t)                      # weights of one key only
    _close(d, _run(d, 0.5), 0.5)


@pytest.mark.parametrize("t,power", [(torch.bfloat16, 20), (torch.bfloat16, 11), (torch.bfloat16, 50), (torch.float16, 9)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(sign, t, power):
    """Scores so far apart that one key has all the weight, all of them far above or below zero: its value, and its score as the log of the
    sum (D products and the scale, each with two roundings of the absolute sum)."""
    lens, n_q, n_k, D = [70, 200], 4, 2, 64
    d = _make(power, lens, [130, 200], n_q, n_k, D, t)
    d["q"], d["k"] = (sign * d["q"].abs().float() * 2.0 ** power).to(t), (d["k"].abs().float() * 2.0 ** (power if power < 50 else 4)).to(t)
    out, lse = _run(d, 1.0)
    q, k, v, out, lse = (x.double().cpu().numpy() for x in (d["q"], d["k"], d["v"], out, lse))
    of, a, b, some = np.repeat(np.arange(n_k), n_q // n_k), 0, 0, False
    for nq, nk in zip(lens, d["k_lens"]):
        sc = np.einsum("ihd,jhd->ihj", q[a:a + nq], k[b:b + nk][:, of])
        sc = np.where(ao.causal(nq, nk)[:, None], sc, -np.inf)
        order = np.sort(sc, -1)
        off = (2 * D + 16) * U * np.abs(order[..., -1])
        clear = order[..., -1] - order[..., -2] > 2 * off + 40
        some |= clear.any()
        want = v[b:b + nk][sc.argmax(-1), of[None]]
        assert np.isfinite(out[a:a + nq]).all() and np.isfinite(lse[a:a + nq]).all()
        assert np.abs(out[a:a + nq] - want)[clear].max(initial=0) <= torch.finfo(t).eps * np.abs(want).max()
        assert np.all(np.abs(lse[a:a + nq] - order[..., -1])[clear] <= off[clear] + 1e-6)
        a, b = a + nq, b + nk
    assert some


def test_no_keys_at_all():
    d = _make(1, [3, 5], [0, 0], 4, 2, 64, torch.bfloat16)
    out, lse = _run(d)
    assert not out.any() and (lse == -INF).all()


def test_rows_beyond_32_bit_offsets():
    """Tokens 2^20 elements apart, the last of them 2^31 elements from the first: the same bits as side by side."""
    d = _make(2, [1100, 1000], [1100, 1000], 4, 2, 64, torch.bfloat16)
    want = _run(d)
    room = torch.empty(2100, 2 ** 20, dtype=torch.bfloat16, device="cuda")
    at = 0
    for n in "qkv":
        x = room[:, at:at + d[n].shape[1] * 64].view(2100, -1, 64)
        x.copy_(d[n])
        d[n], at = x, at + 512
    out = room[:, at:at + 256].view(2100, 4, 64)
    lmhead.coral_lmhead_prompt_attention(d["q"], d["k"], d["v"], _offsets(d["lens"]), out)
    assert torch.equal(out, want[0])


@pytest.mark.parametrize("D", [64, 72, 128])
def test_what_stands_behind_a_sequence_does_not_matter(D):
    """The same bits whatever the rows behind the last sequence, and the next sequence's, hold."""
    d = _make(3, [300, 77, 130], [310, 77, 200], 4, 2, D, torch.bfloat16, extra_rows=40)
    want = _run(d)
    for bad in (NAN, INF):
        d["k"][587:], d["v"][587:] = bad, bad
        got = _run(d)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    d["v"][310 + 77:587] = NAN                                 # the third sequence's: the others stay
    got = _run(d)
    assert torch.equal(got[0][:377], want[0][:377]) and torch.equal(got[1], want[1]) and got[0][377:507].isnan().all()


def test_scales():
    d = _make(6, [90], [90], 2, 1, 64, torch.bfloat16)
    for scale in (1e-30, 0.01, 3.0):
        _close(d, _run(d, scale), scale)


def _rows_of(lens, s, rows):
    at = sum(lens[:s])
    return [at + r for r in rows]


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("n_q,n_k,D", [(2, 1, 64), (4, 4, 128)])
def test_what_a_row_does_not_see_has_no_influence(bad, n_q, n_k, D):
    lens = [200, 70, 33]
    d = _make(7, lens, lens, n_q, n_k, D, torch.bfloat16)
    want, want_lse = _run(d)
    d["v"][150, :, 3] = bad                                   # a value and, of another sequence, a key
    d["k"][200 + 40, :, 5] = bad
    out, lse = _run(d)
    before = list(range(150)) + _rows_of(lens, 1, range(40)) + _rows_of(lens, 2, range(33))
    # rows that were computed again differ from those that were not by what the weights' rounding moves
    near = lambda a, b: ((a - b).abs() <= 2 ** -6 * b.abs() + 0.02).all()
    assert near(out[before].float(), want[before].float()) and torch.equal(lse[:200], want_lse[:200]) and torch.equal(lse[before], want_lse[before])
    assert not out[150:200, :, 3].isfinite().any()            # those who see the value have it in its column, and only there
    rest = [c for c in range(D) if c != 3]
    assert near(out[150:200][..., rest].float(), want[150:200][..., rest].float())
    if bad != -INF:                                           # a score of NaN or of both infinities' signs reaches the whole row
        seen = out[240:270]
        assert not (seen.isfinite() & lse[240:270].isnan().unsqueeze(-1)).any() and lse[240:270].isfinite().float().mean() < 1
    d["v"][150, :, 3], d["k"][240, :, 5] = 0.5, 0.5
    _close(d, _run(d))


def test_keys_and_values_behind_a_sequence_and_rows_outside():
    lens, k_lens = [100, 20], [130, 20]
    d = _make(8, lens, k_lens, 4, 2, 64, torch.bfloat16, extra_rows=37)
    d["k"][150:], d["v"][150:], d["q"][120:] = NAN, INF, NAN
    out, lse = _run(d)
    _close(d, (out, lse))
    assert (out[120:] == 9).all() and (lse[120:] == 9).all()


def test_offsets_that_do_not_fit_are_clamped():
    d = _make(9, [64], [64], 2, 1, 64, torch.bfloat16)
    out = torch.full_like(d["q"], 9.0)
    off = torch.tensor([-5, 20, 10, 900], device="cuda")       # rows 0..20, none, 10..64
    lmhead.coral_lmhead_prompt_attention(d["q"], d["k"], d["v"], off, out)
    part = dict(d, q=d["q"][10:], k=d["k"][10:], v=d["v"][10:], lens=[54], k_lens=[54])
    assert torch.equal(out[20:], _run(part)[0][10:])
    lmhead.coral_lmhead_prompt_attention(d["q"], d["k"], d["v"], torch.tensor([70, 80], device="cuda"), out.fill_(9.0))
    assert (out == 9).all()


def test_strides_and_no_lse():
    g = torch.Generator().manual_seed(10)
    fused = torch.randn(77, 4 + 2 + 2, 128, generator=g).to(torch.bfloat16).cuda()
    d = dict(q=fused[:, :4], k=fused[:, 4:6], v=fused[:, 6:], lens=[50, 27], k_lens=[50, 27])
    want = _run(dict(d, q=d["q"].contiguous(), k=d["k"].contiguous(), v=d["v"].contiguous()))
    got = _run(d)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    _close(d, got)
    room = torch.full((77, 9, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lmhead.coral_lmhead_prompt_attention(d["q"], d["k"], d["v"], _offsets([50, 27]), room[:, 2:6])
    assert torch.equal(room[:, 2:6], want[0]) and (room[:, :2] == 3).all() and (room[:, 6:] == 3).all()


def test_nothing_to_do():
    for T, lens in ((0, []), (0, [0, 0]), (5, [])):
        q = torch.ones(T, 2, 64, dtype=torch.bfloat16, device="cuda")
        out = torch.full_like(q, 9.0)
        lmhead.coral_lmhead_prompt_attention(q, q[:, :1], q[:, :1], _offsets(lens), out)
        assert (out == 9).all()


def test_repeat_streams_graph_and_two_at_once():
    d, other = _make(11, [300, 500, 64], [300, 500, 64], 8, 2, 128, torch.bfloat16), _make(12, [900], [900], 4, 4, 64, torch.float16)
    want, want_other = _run(d), _run(other)
    for _ in range(20):
        assert torch.equal(_run(d)[0], want[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, offs = [torch.empty_like(x["q"]) for x in (d, other)], [_offsets(x["lens"]) for x in (d, other)]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, f, st in zip((d, other), outs, offs, streams):
            lmhead.coral_lmhead_prompt_attention(x["q"], x["k"], x["v"], f, o, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want_other[0])
    graphs = []
    for x, o, f in zip((d, other), outs, offs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lmhead.coral_lmhead_prompt_attention(x["q"], x["k"], x["v"], f, o)
            lmhead.coral_lmhead_prompt_attention(x["q"], x["k"], x["v"], f, o)
        graphs.append(g)
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for g, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            for _ in range(5):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want_other[0])


def test_binding_refuses_wrong_tensors():
    d = _make(13, [20], [20], 4, 2, 64, torch.bfloat16)
    off, out = _offsets([20]), torch.empty_like(d["q"])
    call = lambda q=d["q"], k=d["k"], v=d["v"], off=off, out=out, **kw: lmhead.coral_lmhead_prompt_attention(q, k, v, off, out, **kw)
    for kw in (dict(q=d["q"].float()), dict(k=d["k"].half()), dict(v=d["v"][:19]), dict(out=out[:19]), dict(off=off.int()), dict(q=d["q"].cpu()),
               dict(k_offsets=_offsets([10, 10])), dict(out_lse=torch.empty(20, 3, device="cuda")), dict(scale=-1.0), dict(k=d["k"][:10], v=d["v"][:10]),
               dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), dict(q=d["q"][:, :3]), dict(q=d["q"].transpose(0, 1)),
               dict(q=d["q"][..., :12], k=d["k"][..., :12], v=d["v"][..., :12], out=out[..., :12])):
        with pytest.raises((ValueError, lmhead.CoralError)):
            call(**kw)
    call()
