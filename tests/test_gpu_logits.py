"""GPU parity of the logits step.  Processed logits and candidate ids are the oracle's float32 steps bit for bit.

Tolerance of the log-sum-exp.  u = 2^-24.  A thread adds the exponentials of a span of 4096 tokens in a tree (4 additions at most)
and up to 8 spans one after the other, each rescaled once; a warp's 32 sums take 5 additions, a row's parts (64 tokens of a span
each at least) 1 a thread and a rescaling for every 256 of them, then 5 and 8: fewer than 16 (V // 65536 + 1) + 37 + 6.  An
exponential is off by 2 ulp and its argument, at most 40 where it still counts, by one rounding: the sum is off by at most
(16 (V // 65536 + 1) + 43 + 40) u relative, which is what the logarithm is off by absolutely; adding the maximum and subtracting
from a logit round once each.
"""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as oor
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _csr(lists, dtype=torch.int32):
    off = torch.tensor(np.concatenate([[0], np.cumsum([len(x) for x in lists])]), dtype=torch.int64)
    flat = torch.tensor([t for x in lists for t in x], dtype=dtype)
    return flat, off


def _cuda(t):
    return None if t is None else t.cuda()


def _run(logits, k, write=True, n_seq=0, row_seq=None, prompt=None, output=None, path=None, rep=None, freq=None, pres=None, bias=None,
         mask=None, mask_rows=None, logits_dev=None, out=None, stream=None):
    """logits: CPU tensor; lists: python lists per sequence; bias: lists of (token, value).  Returns numpy results."""
    M, V = logits.shape
    kw = {}
    if prompt is not None:
        kw["prompt_tokens"], kw["prompt_offsets"] = map(_cuda, _csr(prompt))
    if output is not None:
        kw["output_tokens"], kw["output_offsets"] = map(_cuda, _csr(output))
    if bias is not None:
        kw["bias_tokens"], kw["bias_offsets"] = map(_cuda, _csr([[t for t, _ in b] for b in bias]))
        kw["bias_values"] = torch.tensor([v for b in bias for _, v in b], dtype=torch.float32).cuda()
    f = lambda v: None if v is None else torch.tensor(v, dtype=torch.float32).cuda()
    x = logits.cuda() if logits_dev is None else logits_dev
    out = torch.empty(M, V, dtype=logits.dtype, device="cuda") if write and out is None else out
    ids = torch.empty(M, k, dtype=torch.int32, device="cuda") if k else None
    lps = torch.empty(M, k, dtype=torch.float32, device="cuda") if k else None
    lse = torch.empty(M, dtype=torch.float32, device="cuda")
    kw.update(row_seq=_cuda(row_seq), path_tokens=_cuda(path), repetition=f(rep), frequency=f(freq), presence=f(pres),
              mask_words=_cuda(mask), mask_rows=_cuda(mask_rows), out_logits=out, out_ids=ids, out_logprobs=lps, out_lse=lse)
    lmhead.coral_lmhead_logits_process(x, stream=stream, **kw)
    torch.cuda.synchronize()
    return dict(out=out, ids=None if ids is None else ids.cpu().numpy(), lps=None if lps is None else lps.cpu().numpy(), lse=lse.cpu().numpy())


def _check(got, logits, k, rows=None, n_seq=0, row_seq=None, prompt=None, output=None, path=None, rep=None, freq=None, pres=None,
           bias=None, mask=None, mask_rows=None):
    M, V = logits.shape
    for m in range(M) if rows is None else rows:
        s = m if row_seq is None else int(row_seq[m])
        known = 0 <= s < n_seq
        of = lambda a, d: a[s] if a is not None and known else d
        mr = (m if mask_rows is None else int(mask_rows[m])) if mask is not None else -1
        nothing = mask is not None and mr >= mask.shape[0]
        v, ids, lps, lse = oor.logits_row(
            logits[m].float().numpy(), V, k, of(prompt, ()), of(output, ()), path[m].tolist() if path is not None and known else (),
            of(rep, None), of(freq, None), of(pres, None), of(bias, ()), mask[mr].numpy() if mr >= 0 and not nothing else None, nothing)
        if got["out"] is not None:
            want = torch.from_numpy(v).to(logits.dtype)
            assert torch.equal(torch.nan_to_num(got["out"][m].cpu(), nan=123.0), torch.nan_to_num(want, nan=123.0)), m
        tol = (16 * (V // 8192 // 8 + 1) + 83) * U
        if np.isfinite(lse):
            assert abs(got["lse"][m] - lse) <= tol + U * abs(lse), (m, got["lse"][m], lse)
        else:
            assert np.array_equal(got["lse"][m], np.float32(lse), equal_nan=True), m
        if k:
            assert np.array_equal(got["ids"][m], ids), (m, got["ids"][m], ids)
            a, b = got["lps"][m], lps
            fin = np.isfinite(b)
            assert np.array_equal(np.isnan(a), np.isnan(b)) and np.all(a[np.isneginf(b)] == -np.inf)
            assert np.all(np.abs(a[fin] - b[fin]) <= tol + U * (abs(lse) + np.abs(b[fin])))


def _random(seed, M, V, t, n_seq, plen, olen, path_len, n_bias, std=2.5):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(M, V, generator=g) * std).to(t)
    tok = lambda n: (rng.random(n) ** 3 * V).astype(int).tolist()
    d = dict(n_seq=n_seq, row_seq=torch.tensor(rng.integers(0, n_seq, M), dtype=torch.int32),
             prompt=[tok(max(0, plen - 5 * s)) for s in range(n_seq)], output=[tok(max(0, olen - 3 * s)) for s in range(n_seq)],
             rep=(1 + rng.random(n_seq)).astype(np.float32).tolist(), freq=rng.random(n_seq).astype(np.float32).tolist(),
             pres=rng.random(n_seq).astype(np.float32).tolist())
    if path_len:
        d["path"] = torch.tensor(rng.integers(-V, V, (M, path_len)), dtype=torch.int32)
    if n_bias:
        d["bias"] = [[(t, float(np.float32(b))) for t, b in zip(tok(n_bias), rng.normal(size=n_bias) * 3)] for _ in range(n_seq)]
    W = (V + 31) // 32
    d["mask"] = torch.tensor(rng.integers(-2 ** 31, 2 ** 31, (M, W)), dtype=torch.int32)
    d["mask_rows"] = torch.tensor(rng.integers(-1, M, M), dtype=torch.int32)
    return logits, d


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,V,k", [(1, 1, 1), (3, 31, 5), (2, 1000, 10), (5, 4001, 32), (9, 8192, 10), (4, 8193, 7), (10, 32000, 10),
                                   (3, 70001, 32), (2, 152064, 10), (12, 140003, 1)])
def test_random_rows(M, V, k, t):
    logits, d = _random(M * 1000 + V, M, V, t, 3, 300, 200, 4, 40)
    _check(_run(logits, k, **d), logits, k, **d)
    plain = {}
    _check(_run(logits, k, **plain), logits, k, **plain)                     # nothing to apply: log-softmax and candidates


@pytest.mark.parametrize("t", TYPES)
def test_parts_alone(t):
    logits, d = _random(5, 6, 9001, t, 2, 100, 50, 3, 20)
    seqs = dict(n_seq=2, row_seq=d["row_seq"])
    for names in (["prompt", "rep"], ["output", "freq"], ["output", "pres"], ["path", "freq", "pres"], ["path", "rep"], ["bias"]):
        kw = dict(seqs, **{n: d[n] for n in names})
        _check(_run(logits, 10, **kw), logits, 10, **kw)
    kw = dict(mask=d["mask"], mask_rows=d["mask_rows"])
    _check(_run(logits, 10, **kw), logits, 10, **kw)
    kw = dict(mask=d["mask"])
    _check(_run(logits, 10, **kw), logits, 10, **kw)
    _check(_run(logits, 0, **kw), logits, 0, **kw)                           # no candidates wanted
    got = _run(logits, 10, write=False, **kw)                                # ... or no logits
    _check(got, logits, 10, **kw)


def test_rows_without_sequence_or_mask():
    logits, d = _random(6, 8, 500, torch.float32, 3, 50, 50, 2, 10)
    d["row_seq"] = torch.tensor([0, -1, 1, 3, 2, 1000, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)
    d["mask_rows"] = torch.tensor([0, -1, 8, 7, 100, -5, 3, 2 ** 31 - 1], dtype=torch.int32)
    _check(_run(logits, 5, **d), logits, 5, **d)


@pytest.mark.parametrize("V", [40, 5000, 20000, 100000])
def test_ties_and_piles(V):
    """Equal logits (the lower id wins), values that pile up just under the best ones, sorted rows, few distinct values."""
    rows = [torch.zeros(V), torch.arange(V).float(), -torch.arange(V).float(), (torch.arange(V) % 7).float(),
            torch.full((V,), -3.0e38), torch.where(torch.arange(V) % 5 == 0, 1.0, 0.999), torch.full((V,), -float("inf"))]
    rows[6][V // 2] = -7.5
    blocky = torch.zeros(V)
    blocky[:min(V, 2048)] = 5 + torch.rand(min(V, 2048), generator=torch.Generator().manual_seed(0))
    one_lane = torch.full((V,), -9.0)                                        # the best values all lie with few threads
    one_lane[::2048] = torch.arange(len(one_lane[::2048])).float()
    logits = torch.stack(rows + [blocky, one_lane, torch.full((V,), float("-0.0"))])
    logits[-1, 1::2] = 0.0                                                    # -0 and +0 are equal
    for t in TYPES:
        x = logits.to(t)
        for k in (1, 10, 32):
            _check(_run(x, k), x, k)


def test_empty_rows_and_non_finite_values():
    V, W = 9000, (9000 + 31) // 32
    g = torch.Generator().manual_seed(1)
    logits = torch.randn(8, V, generator=g)
    mask = torch.zeros(8, W, dtype=torch.int32)
    mask[1, 280] = 1 << 5                                                     # one token
    mask[2, 0] = 0b1011
    mask[3:] = -1
    mask[5, 3] = 0
    logits[0, 5] = float("nan")                                               # masked: no influence
    logits[1, :] = float("inf")
    logits[1, 280 * 32 + 5] = 1.25
    logits[3, 77] = float("nan")                                              # allowed
    logits[4, 99] = float("inf")
    logits[5, 96:128] = torch.tensor([float("inf"), float("nan")] * 16)       # masked
    logits[6, :] = -float("inf")
    logits[7, :] = torch.finfo(torch.float32).min
    got = _run(logits, 10, mask=mask)
    _check(got, logits, 10, mask=mask)
    assert np.all(got["ids"][0] == oor.NO_TOKEN) and got["lse"][0] == -np.inf and np.all(got["lps"][0] == -np.inf)
    assert got["ids"][1][0] == 280 * 32 + 5 and got["lps"][1][0] == 0.0 and got["ids"][1][1] == oor.NO_TOKEN
    for t in (torch.bfloat16, torch.float16):
        x = torch.nan_to_num(logits, nan=0.0, posinf=float("inf"), neginf=-float("inf")).to(t)
        _check(_run(x, 10, mask=mask), x, 10, mask=mask)


def test_long_lists_repeats_and_bad_entries():
    """Histories far longer than a block, one token thousands of times, padding and tokens past the vocabulary, two biases for
    one token, offsets that leave the list."""
    V, rng = 30011, np.random.default_rng(3)
    logits = torch.randn(4, V, generator=torch.Generator().manual_seed(2))
    out = [[7] * 5000 + rng.integers(0, V, 30000).tolist(), [], [-1, V, V + 1, 2 ** 31 - 1, -2 ** 31, 3, 3], [V - 1, 0]]
    prompt = [[], rng.integers(0, V, 40000).tolist(), [5, -1], [0]]
    bias = [[(7, 1.0), (7, 2.0), (8, -1.0), (7, 3.5)], [], [(-1, 9.0), (V, 9.0), (3, 0.5)], [(0, float("inf"))]]
    d = dict(n_seq=4, prompt=prompt, output=out, bias=bias, rep=[1.3, 2.0, 0.5, 1.0], freq=[0.01, 0.5, -0.25, 0.1], pres=[0.5, 0.1, 0.2, 0.3])
    _check(_run(logits, 10, **d), logits, 10, **d)
    flat, off = _csr(out)
    bad = off.clone()
    bad[0], bad[4] = -50, 10 ** 15                                            # clamped to the list
    ids = [torch.empty(4, 10, dtype=torch.int32, device="cuda") for _ in range(2)]
    lps = torch.empty(4, 10, device="cuda")
    for o, i in zip((off, bad), ids):
        lmhead.coral_lmhead_logits_process(logits.cuda(), output_tokens=flat.cuda(), output_offsets=o.cuda(),
                                           frequency=torch.tensor(d["freq"]).cuda(), out_ids=i, out_logprobs=lps)
    assert torch.equal(*ids)


@pytest.mark.parametrize("V,wide", [(400003, False), (200010, True)])
def test_vocabularies_longer_than_the_table(V, wide):
    """The token table then covers a row in several passes, built anew for each row."""
    logits, d = _random(21, 10, V, torch.float32, 3, 400, 300, 4, 30)
    if wide:
        d["output"][0] = d["output"][0] + [11] * 33000                      # counts past 15 bits
    _check(_run(logits, 10, **d), logits, 10, rows=[0, 3, 9], **d)


@pytest.mark.parametrize("V", [33333, 32002, 32000])
def test_tree_nodes_of_a_few_sequences(V):
    """Rows of one sequence follow one another and differ in their path only; rows without a sequence stand between them."""
    M = 310
    logits, d = _random(22, M, V, torch.bfloat16, 5, 300, 200, 6, 25)
    d["row_seq"] = torch.arange(M, dtype=torch.int32) // 62
    d["row_seq"][40::41] = -1
    d["path"][:, 2] = d["path"][:, 1]                                        # a token twice on one path
    d["path"][1::2, 0] = torch.tensor([d["output"][int(s)][0] if s >= 0 else 0 for s in d["row_seq"][1::2]], dtype=torch.int32)
    _check(_run(logits, 10, **d), logits, 10, rows=list(range(0, M, 17)) + [40, 41, 42, 61, 62, 63], **d)
    d["row_seq"] = torch.arange(M, dtype=torch.int32) % 5                    # the sequences in turn
    _check(_run(logits, 10, **d), logits, 10, rows=range(0, M, 31), **d)


@pytest.mark.parametrize("t", TYPES)
def test_row_distance_alignment_in_place(t):
    """Rows that lie apart and start on any address, outputs aligned otherwise, the columns behind a row left as they were."""
    V, M = 12345, 5
    logits, d = _random(9, M, V, t, 2, 60, 60, 2, 9)
    for off, ld, ooff, old in [(1, V + 3, 0, V), (3, V + 8, 3, V + 8), (0, V + 1, 5, V + 2), (7, 16384, 2, 12352)]:
        buf = torch.full((off + ld * M + 8,), 3.0, dtype=t, device="cuda")
        obuf = torch.full((ooff + old * M + 8,), 4.0, dtype=t, device="cuda")
        x = buf[off:off + ld * M].view(M, ld)[:, :V]
        o = obuf[ooff:ooff + old * M].view(M, old)[:, :V]
        x.copy_(logits)
        _check(_run(logits, 10, logits_dev=x, out=o, **d), logits, 10, **d)
        touched = torch.zeros_like(obuf, dtype=torch.bool)
        touched[ooff:ooff + old * M].view(M, old)[:, :V] = True
        assert torch.all(obuf[~touched] == 4.0)
        _check(_run(logits, 10, logits_dev=x, out=x, **d), logits, 10, **d)   # in place
        inside = torch.zeros_like(buf, dtype=torch.bool)
        inside[off:off + ld * M].view(M, ld)[:, :V] = True
        assert torch.all(buf[~inside] == 3.0)


def test_many_rows_repeat_stream_and_graph():
    M, V = 700, 20000
    logits, d = _random(10, M, V, torch.bfloat16, 16, 400, 300, 6, 10)
    a = _run(logits, 10, **d)
    _check(a, logits, 10, rows=range(0, M, 53), **d)
    st = torch.cuda.Stream()
    b = _run(logits, 10, stream=st, **d)
    for n in ("ids", "lps", "lse"):
        assert np.array_equal(a[n], b[n]), n
    assert torch.equal(a["out"], b["out"])
    x = logits.cuda()
    ids, lps, lse = torch.empty(M, 10, dtype=torch.int32, device="cuda"), torch.empty(M, 10, device="cuda"), torch.empty(M, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lmhead.coral_lmhead_logits_process(x, out_ids=ids, out_logprobs=lps, out_lse=lse)
    x.copy_(logits.flip(0))
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    want = _run(logits.flip(0), 10)
    assert np.array_equal(ids.cpu().numpy(), want["ids"]) and np.array_equal(lps.cpu().numpy(), want["lps"])


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(4, 64, device="cuda")
    ids, lps = torch.empty(4, 5, dtype=torch.int32, device="cuda"), torch.empty(4, 5, device="cuda")
    call = lmhead.coral_lmhead_logits_process
    one = torch.ones(4, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    i64 = lambda *s: torch.zeros(*s, dtype=torch.int64, device="cuda")
    for bad in [dict(out_logprobs=None), dict(out_logprobs=lps[:, :4].contiguous()), dict(repetition=torch.ones(3, device="cuda")),
                dict(repetition=one, frequency=torch.ones(5, device="cuda")), dict(prompt_tokens=i32(7)), dict(prompt_offsets=i64(5)),
                dict(prompt_tokens=i32(7), prompt_offsets=i32(5)), dict(mask_words=i32(4, 1)), dict(mask_words=i32(3, 2)),
                dict(bias_tokens=i32(3), bias_offsets=i64(5)), dict(bias_tokens=i32(3), bias_offsets=i64(5), bias_values=torch.ones(2, device="cuda")),
                dict(path_tokens=i32(3, 2), repetition=one), dict(row_seq=i64(4)), dict(mask_rows=i32(4)), dict(out_lse=torch.empty(3, device="cuda")),
                dict(out_logits=torch.empty(4, 64, device="cuda").half()), dict(out_logits=torch.empty(64, 4, device="cuda").t())]:
        kw = dict(out_ids=ids, out_logprobs=lps)
        kw.update(bad)
        with pytest.raises((ValueError, lmhead.CoralError)):
            call(x, **kw)
    with pytest.raises(ValueError):
        call(torch.zeros(64, 4, device="cuda").t(), out_ids=ids, out_logprobs=lps)
    with pytest.raises(lmhead.CoralError):
        call(x, out_ids=torch.empty(4, 33, dtype=torch.int32, device="cuda"), out_logprobs=torch.empty(4, 33, device="cuda"))


def test_scratch_belongs_to_the_stream_that_runs_the_call():
    """Memory that another stream still has work on must not become the scratch of a call."""
    M, V = 64, 5000
    logits, d = _random(12, M, V, torch.float32, 4, 200, 100, 3, 5)
    want = _run(logits, 10, **d)
    st = torch.cuda.Stream()
    kw = dict(out_ids=torch.empty(M, 10, dtype=torch.int32, device="cuda"), out_logprobs=torch.empty(M, 10, device="cuda"),
              out_lse=torch.empty(M, device="cuda"))
    x = logits.cuda()
    plain = _run(logits, 10, write=False)
    torch.cuda.synchronize()
    for kb in (8, 16, 64, 256, 1024):                        # whatever size the scratch has
        old = [torch.empty(kb << 10, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda._sleep(20_000_000)                        # ~10 ms before the current stream writes to it
        for o in old:
            o.fill_(255)
        del old, o
        lmhead.coral_lmhead_logits_process(x, stream=st, **kw)
        torch.cuda.synchronize()
        assert np.array_equal(kw["out_ids"].cpu().numpy(), plain["ids"]) and np.array_equal(kw["out_lse"].cpu().numpy(), plain["lse"])
    assert not np.array_equal(want["ids"], plain["ids"])


def test_decreasing_offsets_stay_in_bounds():
    """Offsets that go back (a caller's mistake): the sequences whose lists do not overlap are right, nothing else is touched."""
    M, V = 200, 9000
    rng = np.random.default_rng(13)
    logits = torch.from_numpy(rng.normal(size=(M, V)).astype(np.float32))
    tok = torch.from_numpy(rng.integers(0, V, 600).astype(np.int32)).cuda()
    off = torch.tensor([0, 400, 100, 380, 390], device="cuda")                    # [0, 400), none, [100, 380), [380, 390)
    seq = torch.tensor([m % 5 - 1 for m in range(M)], dtype=torch.int32)
    out = torch.full((M + 2, V), 7.0, device="cuda")
    for rows in (M, 3):                                                           # both kernels: many rows and few
        lmhead.coral_lmhead_logits_process(logits[:rows].cuda(), row_seq=seq[:rows].cuda(), output_tokens=tok, output_offsets=off,
                                           presence=torch.ones(4, device="cuda"), out_logits=out[1:rows + 1])
        torch.cuda.synchronize()
        assert torch.all(out[0] == 7) and torch.all(out[M + 1] == 7)
        for m in range(rows):
            if seq[m] in (-1, 1):
                assert torch.equal(out[m + 1].cpu(), logits[m]), m


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,V,plen", [(300, 9001, 3000), (400, 60001, 6000), (200, 32768, 10)])
def test_many_rows_alignment_in_place_and_special_values(M, V, plen, t):
    """The pipelined kernel: one span a block and several, dense lists (more than a block's threads in a span), rows that start on
    any address, in place, rows that allow nothing, infinities and NaN in masked and in allowed places."""
    logits, d = _random(M + V, M, V, t, 7, plen, plen // 2, 5, 30)
    bad = [float("inf"), float("-inf"), float("nan")]
    for i in range(0, M, 5):
        logits[i, (i * 37) % V] = bad[i % 3]
    d["mask"][3] = 0
    d["mask_rows"][9:12] = torch.tensor([3, M, 2 ** 31 - 1], dtype=torch.int32)       # nothing, and no such mask
    d["rep"][2], d["rep"][4] = 1.0, 0.7
    rows = sorted({0, 1, 4, 5, 9, 10, 11, M // 2, M - 2, M - 1, *range(0, M, max(5, M // 40 * 5))})[:40]
    for off, ld, ooff, old in [(0, V, 0, V), (3, V + 5, 1, V + 2)]:
        buf = torch.full((off + ld * M + 8,), 3.0, dtype=t, device="cuda")
        obuf = torch.full((ooff + old * M + 8,), 4.0, dtype=t, device="cuda")
        x = buf[off:off + ld * M].view(M, ld)[:, :V]
        o = obuf[ooff:ooff + old * M].view(M, old)[:, :V]
        x.copy_(logits)
        _check(_run(logits, 10, logits_dev=x, out=o, **d), logits, 10, rows=rows, **d)
        touched = torch.zeros_like(obuf, dtype=torch.bool)
        touched[ooff:ooff + old * M].view(M, old)[:, :V] = True
        assert torch.all(obuf[~touched] == 4.0)
        apart = o.clone()
        _check(_run(logits, 10, logits_dev=x, out=x, **d), logits, 10, rows=rows[:6], **d)
        assert torch.equal(torch.nan_to_num(x, nan=9.0), torch.nan_to_num(apart, nan=9.0))
        assert torch.all(buf[off:off + ld * M].view(M, ld)[:, V:] == 3.0)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V,k", [(40, 32), (1500, 32), (20000, 1), (9000, 32)])
def test_ends_of_very_many_rows(V, k, t):
    """More rows than the wide blocks of the last kernel that fit at once: ties, few pieces, rows with less than k candidates, in place."""
    M = 640
    logits, d = _random(V + k, M, V, t, 5, 200, 150, 3, 8)
    logits[::3] = torch.round(logits[::3])                  # ties
    logits[1::4, 7:] = float("-inf")
    want = _run(logits, k, **d)
    rows = list(range(0, M, 29))
    _check(want, logits, k, rows=rows, **d)
    x = logits.cuda()
    got = _run(logits, k, logits_dev=x, out=x, **d)
    for n in ("ids", "lps", "lse"):
        assert np.array_equal(got[n], want[n], equal_nan=n != "ids"), n
    assert torch.equal(torch.nan_to_num(got["out"], nan=9.0), torch.nan_to_num(want["out"], nan=9.0))


@pytest.mark.parametrize("V", [40, 5000, 100000])
def test_piles_in_very_many_rows(V):
    """Equal values, sorted rows and values that pile up, each row 130 times over: every copy gives the first one's answer."""
    n = torch.arange(V)
    rows = torch.stack([torch.zeros(V), n.float(), -n.float(), (n % 7).float(), torch.where(n % 5 == 0, 1.0, 0.999)])
    for t in TYPES:
        x = rows.to(t).repeat(130, 1)
        for k in (1, 10, 32):
            got = _run(x, k, write=False)
            _check(got, x, k, rows=range(5))
            for name in ("ids", "lps", "lse"):
                a = got[name].reshape(130, 5, -1)
                assert np.array_equal(a, np.broadcast_to(a[:1], a.shape), equal_nan=name != "ids"), (name, k)     # 99999 is +inf in fp16


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("path_len", [6, 31, 33, 48, 64])
def test_tokens_again_and_again_on_long_paths(path_len, t):
    """A path's token is penalised once, with the count of its repeats, wherever on the path they stand (also 32 and more apart,
    next to one another, listed or not, everywhere), for few and many rows, written apart and in place."""
    for M, V in ((3, 9001), (300, 9001), (120, 32768)):
        logits, d = _random(path_len + M, M, V, t, 4, 80, 60, path_len, 9)
        p, half = d["path"], path_len // 2
        p[:, path_len - half:] = p[:, :half]                                 # the second half repeats the first
        p[1::4, :] = p[1::4, :1].abs().clamp(max=V - 1)                      # one token all along
        p[2::4, ::3] = torch.tensor([d["output"][int(s)][0] for s in d["row_seq"][2::4]], dtype=torch.int32)[:, None]      # a listed one
        p[3::4, 1::2] = p[3::4, ::2][:, :path_len // 2]                      # pairs
        got = _run(logits, 10, **d)
        _check(got, logits, 10, rows=range(0, M, max(1, M // 60)), **d)
        for _ in range(3):
            x = logits.cuda()
            again = _run(logits, 10, logits_dev=x, out=x, **d)
            assert torch.equal(torch.nan_to_num(again["out"].float(), nan=1.0), torch.nan_to_num(got["out"].float(), nan=1.0))
            assert np.array_equal(again["ids"], got["ids"]) and np.array_equal(again["lps"], got["lps"]) and np.array_equal(again["lse"], got["lse"])
