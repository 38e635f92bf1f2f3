"""What the operators around the grouped LM-head draft step are measured on: the block norm that makes the hidden rows
(forward and backward), the product with 4-bit weights (the dense head and the drafter's projections), and the
penalties, biases and grammar masks on dense logits with the candidates that feed the tree.

`run` computes a case in elementary torch operations where `own` is false, and by the library's calls where it is true.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GATES = {"none": 0, "channel": 1, "row": 2, "full": 3}         # CORAL_GATE_*
NO_TOKEN = 0x7FFFFFFF          # id of a candidate that does not exist (fewer active tokens than candidates)
EPS = 1e-5


def listed():
    return [
        # one row against the dense 4-bit Llama3-8B-shaped head: the logits that verify a draft, batch of one
        dict(name="q4_head_llama3_m1", op="q4", M=1, N=128256, K=4096, group=128, zeros=False, x="bf16", out="f32"),
        # the tree of one sequence (60 nodes) against the dense 4-bit Qwen2.5-7B-shaped head
        dict(name="q4_head_qwen_m60", op="q4", M=60, N=152064, K=3584, group=64, zeros=True, x="bf16", out="bf16"),
        # eight sequences against the Llama2-7B-shaped head, fp16 activations and scales with zero points
        dict(name="q4_head_llama2_m8", op="q4", M=8, N=32000, K=4096, group=128, zeros=True, x="f16", out="f32"),
        # a small projection with an odd number of rows and outputs: the smallest call, where latency counts
        dict(name="q4_small_m3", op="q4", M=3, N=4001, K=256, group=32, zeros=True, x="f16", out="f16"),
        # sampling the next token of one sequence: long prompt, some output, a few biased tokens
        dict(name="logits_next_token", op="logits", M=1, V=128256, n_seq=1, type="f32", prompt=1500, output=200, path=0,
             bias=50, mask="none", k=10, write=False),
        # the 60 tree nodes of one sequence under a grammar, candidates only (they go to the tree expansion)
        dict(name="logits_tree_grammar", op="logits", M=60, V=152064, n_seq=1, type="bf16", prompt=700, output=300, path=6,
             bias=0, mask="rows", k=10, write=False),
        # 16 sequences x 60 nodes, processed logits wanted for sampling as well
        dict(name="logits_16x60", op="logits", M=960, V=128256, n_seq=16, type="f32", prompt=2000, output=1000, path=6,
             bias=20, mask="seqs", k=10, write=True),
        # a small odd vocabulary in fp16, most candidates, one row whose mask leaves nothing
        dict(name="logits_small_odd", op="logits", M=5, V=4001, n_seq=5, type="f16", prompt=60, output=33, path=0,
             bias=7, mask="empty", k=32, write=True),
        # one token of one sequence: the norm that feeds the draft step
        dict(name="norm_one_token", op="norm", M=1, H=4096, type="bf16", post=False, gate="none", alpha=1.0),
        # prefill of 16384 tokens with a norm behind the block and a gate per channel
        dict(name="norm_prefill", op="norm", M=16384, H=4096, type="bf16", post=True, gate="channel", alpha=0.7),
        # training batches: the backward pass, 4 sequences of 2048 tokens, and an odd one with a gate per row
        dict(name="norm_backward_8k", op="norm_backward", M=8192, H=4096, type="bf16", post=True, gate="channel", alpha=0.7),
        dict(name="norm_backward_odd", op="norm_backward", M=777, H=3584, type="f16", post=False, gate="row", alpha=1.0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["q4", "logits", "norm", "norm_backward"])
    if op == "q4":
        group = rng.choice([32, 64, 128])
        K = group * _log(rng, 256 // group, 8192 // group)
        M = _log(rng, 1, 60)
        N = _log(rng, 200, min(152064, 152064 * 3584 // K))
        return dict(op=op, M=M, N=N, K=K, group=group, zeros=rng.random() < 0.5, x=rng.choice(["bf16", "f16"]),
                    out=rng.choice(["f32", "f32", "bf16", "f16"]))
    if op == "logits":
        V = _log(rng, 1000, 152064)
        n_seq = _log(rng, 1, 16)
        M = n_seq * _log(rng, 1, min(60, max(1, 960 * 128256 // (V * n_seq))))
        return dict(op=op, M=M, V=V, n_seq=n_seq, type=rng.choice(["f32", "bf16", "f16"]), prompt=rng.choice([0, _log(rng, 1, 8192)]),
                    output=rng.choice([0, _log(rng, 1, 4096)]), path=rng.choice([0, 6]), bias=rng.choice([0, _log(rng, 1, 300)]),
                    mask=rng.choice(["none", "rows", "seqs", "empty"]), k=rng.choice([0, 1, 10, 32]), write=True)
    H = 8 * _log(rng, 32, 1024)
    M = _log(rng, 1, min(16384, 16384 * 4096 // H)) if op == "norm" else _log(rng, 1, min(8192, 8192 * 4096 // H))
    kind = rng.choice(["bf16", "f16", "f32"])
    return dict(op=op, M=M if kind != "f32" else (M + 1) // 2, H=H, type=kind, post=rng.random() < 0.5,
                gate=rng.choice(["none", "channel", "row", "full"]), alpha=rng.choice([1.0, 0.7]))


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _tokens(g, n, V):
    """Token ids as text has them: a few frequent ones, many rare ones."""
    return (torch.rand(n, generator=g, device="cuda").double().pow(4) * V).long().clamp_(max=V - 1).int()


def _lists(g, n_seq, length, V):
    """Ragged lists of about `length` tokens each (0 for the second sequence), flat, with their offsets."""
    lens = [max(0, length - 3 * s) if s != 1 else 0 for s in range(n_seq)]
    offsets = torch.tensor([sum(lens[:s]) for s in range(n_seq + 1)], dtype=torch.int64, device="cuda")
    return _tokens(g, sum(lens), V), offsets


def _prepare_q4(case, g):
    N, K, M, group = case["N"], case["K"], case["M"], case["group"]
    x = TYPES[case["x"]]
    s = dict(case)
    s["Wq"] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s["scales"] = (0.004 * (0.5 + torch.rand(N, K // group, generator=g, device="cuda"))).to(x)
    s["zp"] = torch.randint(5, 12, (N, K // group), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    s["hidden"] = _normal(g, (M, K), 1.0, x)
    s["y"] = torch.empty(M, N, dtype=TYPES[case["out"]], device="cuda")
    if own:
        from paper_2502_16880_b200 import lmhead
        s["head"] = lmhead.Q4Linear(s["Wq"], s["scales"], s["zp"])
    return s


def _prepare_logits(case, g):
    M, V, n_seq, k = case["M"], case["V"], case["n_seq"], case["k"]
    s = dict(case)
    s["logits"] = _normal(g, (M, V), 2.5, TYPES[case["type"]])
    s["row_seq"] = torch.arange(M, device="cuda", dtype=torch.int32) // (M // n_seq)
    s["prompt_tokens"], s["prompt_offsets"] = _lists(g, n_seq, case["prompt"], V) if case["prompt"] else (None, None)
    s["output_tokens"], s["output_offsets"] = _lists(g, n_seq, case["output"], V) if case["output"] else (None, None)
    s["path_tokens"] = _tokens(g, M * case["path"], V).view(M, case["path"]) if case["path"] else None
    if case["path"]:                                             # nodes of different depth: the rest of a row is -1
        depth = torch.randint(0, case["path"] + 1, (M, 1), generator=g, device="cuda")
        s["path_tokens"] = torch.where(torch.arange(case["path"], device="cuda") < depth, s["path_tokens"], -1).int().contiguous()
    s["repetition"] = 1.0 + 0.3 * torch.rand(n_seq, generator=g, device="cuda")
    s["frequency"] = 0.5 * torch.rand(n_seq, generator=g, device="cuda")
    s["presence"] = 0.5 * torch.rand(n_seq, generator=g, device="cuda")
    s["bias_tokens"] = s["bias_values"] = s["bias_offsets"] = None
    if case["bias"]:                                             # distinct tokens in each sequence's list
        first = torch.randint(0, V, (n_seq, 1), generator=g, device="cuda")
        at = first + torch.arange(case["bias"], device="cuda") * max(1, V // case["bias"] - 1)
        s["bias_tokens"] = (at % V).int().reshape(-1)
        s["bias_values"] = _normal(g, (n_seq * case["bias"],), 3.0, torch.float32)
        s["bias_offsets"] = torch.arange(n_seq + 1, device="cuda", dtype=torch.int64) * case["bias"]
    s["mask_words"] = s["mask_rows"] = None
    if case["mask"] != "none":                                   # grammar states: few tokens allowed, or many
        n = n_seq if case["mask"] == "seqs" else M
        W = (V + 31) // 32
        words = torch.randint(-2 ** 31, 2 ** 31, (n, W), generator=g, device="cuda")
        words &= torch.where(torch.rand(n, W, generator=g, device="cuda") < 0.6, -1, 0)
        if case["mask"] == "empty":
            words[n // 2] = 0                                    # a state that allows nothing
        s["mask_words"] = words.int()
        s["mask_rows"] = s["row_seq"].clone() if case["mask"] == "seqs" else torch.arange(M, device="cuda", dtype=torch.int32)
        if case["mask"] == "rows":
            s["mask_rows"][::7] = -1                             # some rows are outside the grammar
    s["out_logits"] = torch.empty_like(s["logits"]) if case["write"] else None
    s["ids"] = torch.empty(M, k, dtype=torch.int32, device="cuda")
    s["logprobs"] = torch.empty(M, k, dtype=torch.float32, device="cuda")
    s["lse"] = torch.empty(M, dtype=torch.float32, device="cuda")
    return s


def _prepare_norm(case, g):
    M, H, t = case["M"], case["H"], TYPES[case["type"]]
    s = dict(case)
    s["block"] = _normal(g, (M, H), 1.3, t)
    s["resid"] = _normal(g, (M, H), 2.0, t)
    s["w_pre"] = (1.0 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(t)
    s["w_post"] = (1.0 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(t) if case["post"] else None
    shape = {"none": None, "channel": (H,), "row": (M,), "full": (M, H)}[case["gate"]]
    s["g"] = None if shape is None else (0.5 + 0.3 * torch.randn(shape, generator=g, device="cuda")).to(t)
    if case["op"] == "norm":
        s["stream"], s["hidden"] = torch.empty_like(s["block"]), torch.empty_like(s["block"])
        return s
    s["d_hidden"] = _normal(g, (M, H), 1.0, t)
    s["d_stream"] = _normal(g, (M, H), 0.5, t)
    s["d_block"], s["d_resid"] = torch.empty_like(s["block"]), torch.empty_like(s["block"])
    s["d_w_pre"] = torch.empty(H, dtype=torch.float32, device="cuda")
    s["d_w_post"] = torch.empty(H, dtype=torch.float32, device="cuda") if case["post"] else None
    s["d_g"] = None if shape is None else torch.empty(shape, dtype=t if case["gate"] == "full" else torch.float32, device="cuda")
    if own:
        from paper_2502_16880_b200 import lmhead
        n = lmhead.coral_lmhead_block_norm_backward_bytes(M, H)
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"q4": _prepare_q4, "logits": _prepare_logits, "norm": _prepare_norm, "norm_backward": _prepare_norm}[case["op"]](case, g)


# ---- the plain forms ---------------------------------------------------------------------------------------
def _plain_q4(s):
    q = torch.stack((s["Wq"] & 15, s["Wq"] >> 4), dim=-1).view(s["N"], -1, s["group"]).float()
    z = 8.0 if s["zp"] is None else s["zp"].float().unsqueeze(-1)
    W = ((q - z) * s["scales"].float().unsqueeze(-1)).view(s["N"], s["K"])
    return (s["hidden"].float() @ W.t()).to(TYPES[s["out"]])


def _rows_of(offsets, total):
    lens = offsets[1:] - offsets[:-1]
    return torch.repeat_interleave(torch.arange(lens.numel(), device="cuda"), lens, output_size=total)


def _plain_logits(s):
    M, V, n_seq, k = s["M"], s["V"], s["n_seq"], s["k"]
    l = s["logits"].float()
    seq = s["row_seq"].long()
    seen = torch.zeros(n_seq, V, dtype=torch.bool, device="cuda")
    count = torch.zeros(n_seq, V, dtype=torch.float32, device="cuda")
    if s["prompt_tokens"] is not None:
        seen[_rows_of(s["prompt_offsets"], s["prompt_tokens"].numel()), s["prompt_tokens"].long()] = True
    if s["output_tokens"] is not None:
        rows = _rows_of(s["output_offsets"], s["output_tokens"].numel())
        count.index_put_((rows, s["output_tokens"].long()), torch.ones((), device="cuda"), accumulate=True)
    count, seen = count[seq], seen[seq]
    if s["path_tokens"] is not None:
        p = s["path_tokens"].long()
        count.scatter_add_(1, p.clamp(min=0), (p >= 0).float())
    seen = seen | (count > 0)
    rep = s["repetition"][seq].unsqueeze(1)
    l = torch.where(seen, torch.where(l > 0, l / rep, l * rep), l)
    l = l - s["frequency"][seq].unsqueeze(1) * count
    l = l - s["presence"][seq].unsqueeze(1) * (count > 0).float()
    if s["bias_tokens"] is not None:
        bias = torch.zeros(n_seq, V, device="cuda")
        bias[_rows_of(s["bias_offsets"], s["bias_tokens"].numel()), s["bias_tokens"].long()] = s["bias_values"]
        l = l + bias[seq]
    if s["mask_words"] is not None:
        bits = ((s["mask_words"].unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).bool().view(-1, s["mask_words"].shape[1] * 32)[:, :V]
        r = s["mask_rows"].long()
        l = torch.where(bits[r.clamp(min=0)] | (r < 0).unsqueeze(1), l, -math.inf)
    m = l.amax(1)
    base = torch.where(m == -math.inf, 0.0, m)
    lse = base + (l - base.unsqueeze(1)).exp().sum(1).log()
    # descending value, equal values by the lower id: one 64-bit key a token
    b = (l + 0.0).view(torch.int32)
    key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long() * 2 ** 32 + (2 ** 32 - 1 - torch.arange(V, device="cuda"))
    ids = 2 ** 32 - 1 - (key.topk(k, dim=1).values & (2 ** 32 - 1)) if k else torch.zeros(M, 0, dtype=torch.int64, device="cuda")
    top = l.gather(1, ids)
    ids = torch.where(top == -math.inf, NO_TOKEN, ids).int()
    logprobs = torch.where(top == -math.inf, -math.inf, top - lse.unsqueeze(1))
    out = dict(ids=ids, logprobs=logprobs, lse=lse)
    if s["write"]:
        out["logits"] = l.to(s["logits"].dtype)
    return out


def _gate_of(s):
    if s["g"] is None:
        return 1.0
    return s["g"].float().unsqueeze(1) if s["gate"] == "row" else s["g"].float()


def _plain_norm(s):
    x, r = s["block"].float(), s["resid"].float()
    if s["w_post"] is not None:
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * s["w_post"].float()
    y = s["alpha"] * r + _gate_of(s) * x
    h = y * torch.rsqrt(y.square().mean(1, keepdim=True) + EPS) * s["w_pre"].float()
    t = s["block"].dtype
    return dict(stream=y.to(t), hidden=h.to(t))


def _plain_norm_backward(s):
    x, r, dh, dy = s["block"].float(), s["resid"].float(), s["d_hidden"].float(), s["d_stream"].float()
    t, gate, post = s["block"].dtype, _gate_of(s), s["w_post"] is not None
    rx = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    b = x * rx * s["w_post"].float() if post else x
    y = s["alpha"] * r + gate * b
    ry = torch.rsqrt(y.square().mean(1, keepdim=True) + EPS)
    yhat = y * ry
    dyhat = dh * s["w_pre"].float()
    dY = dy + ry * (dyhat - yhat * (dyhat * yhat).mean(1, keepdim=True))
    db = gate * dY
    out = dict(d_resid=(s["alpha"] * dY).to(t), d_w_pre=(dh * yhat).sum(0))
    if post:
        xhat = x * rx
        dxhat = db * s["w_post"].float()
        out["d_block"] = (rx * (dxhat - xhat * (dxhat * xhat).mean(1, keepdim=True))).to(t)
        out["d_w_post"] = (db * xhat).sum(0)
    else:
        out["d_block"] = db.to(t)
    if s["gate"] == "channel":
        out["d_gate"] = (dY * b).sum(0)
    elif s["gate"] == "row":
        out["d_gate"] = (dY * b).sum(1)
    elif s["gate"] == "full":
        out["d_gate"] = (dY * b).to(t)
    return out


# ---- the library's calls -----------------------------------------------------------------------------------
def _own_q4(s):
    return s["head"].forward(s["hidden"], out=s["y"])


def _own_logits(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_logits_process(
        s["logits"], row_seq=s["row_seq"], prompt_tokens=s["prompt_tokens"], prompt_offsets=s["prompt_offsets"],
        output_tokens=s["output_tokens"], output_offsets=s["output_offsets"], path_tokens=s["path_tokens"],
        repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias_tokens=s["bias_tokens"],
        bias_values=s["bias_values"], bias_offsets=s["bias_offsets"], mask_words=s["mask_words"], mask_rows=s["mask_rows"],
        out_logits=s["out_logits"], out_ids=s["ids"] if s["k"] else None, out_logprobs=s["logprobs"] if s["k"] else None,
        out_lse=s["lse"])
    out = dict(ids=s["ids"], logprobs=s["logprobs"], lse=s["lse"])
    if s["write"]:
        out["logits"] = s["out_logits"]
    return out


def _own_norm(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_block_norm(s["block"], s["resid"], s["w_pre"], EPS, s["stream"], s["hidden"], w_post=s["w_post"],
                                   gate=s["g"], gate_mode=GATES[s["gate"]], alpha=s["alpha"])
    return dict(stream=s["stream"], hidden=s["hidden"])


def _own_norm_backward(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_block_norm_backward(
        s["block"], s["resid"], s["w_pre"], EPS, s["d_stream"], s["d_hidden"], s["workspace"], s["d_block"], s["d_resid"],
        s["d_w_pre"], w_post=s["w_post"], gate=s["g"], gate_mode=GATES[s["gate"]], alpha=s["alpha"],
        out_dw_post=s["d_w_post"], out_dgate=s["d_g"])
    out = dict(d_resid=s["d_resid"], d_w_pre=s["d_w_pre"], d_block=s["d_block"])
    if s["post"]:
        out["d_w_post"] = s["d_w_post"]
    if s["gate"] != "none":
        out["d_gate"] = s["d_g"]
    return out


def run(state):
    op = state["op"]
    if own:
        return {"q4": _own_q4, "logits": _own_logits, "norm": _own_norm, "norm_backward": _own_norm_backward}[op](state)
    return {"q4": _plain_q4, "logits": _plain_logits, "norm": _plain_norm, "norm_backward": _plain_norm_backward}[op](state)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if case["op"] == "q4":
        M, N, K = case["M"], case["N"], case["K"]
        groups = K // case["group"]
        nbytes = N * K / 2 + N * groups * (2.5 if case["zeros"] else 2) + M * K * size[case["x"]] + M * N * size[case["out"]]
        return {"bytes": nbytes, "flops": 2.0 * M * N * K}
    if case["op"] == "logits":
        M, V, n_seq = case["M"], case["V"], case["n_seq"]
        rows = {"none": 0, "seqs": n_seq}.get(case["mask"], M)
        lists = n_seq * (case["prompt"] + case["output"] + 2 * case["bias"]) + M * case["path"]
        nbytes = M * V * size[case["type"]] * (2 if case["write"] else 1) + rows * V / 8 + 4 * lists + M * (8 * case["k"] + 4)
        return {"bytes": nbytes, "flops": 8.0 * M * V}
    M, H, e = case["M"], case["H"], size[case["type"]]
    back = case["op"] == "norm_backward"
    full = case["gate"] == "full"
    n = (6 if back else 4) + ((2 if back else 1) if full else 0)
    small = H * e * (1 + case["post"]) + (M if case["gate"] == "row" else H) * e + (H * 4 * (1 + case["post"]) + H * 4 if back else 0)
    return {"bytes": n * M * H * e + small, "flops": (35.0 if back else 12.0) * M * H}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------
def _exact_q4(s):
    x = s["hidden"].double()
    parts, K, step = [], s["K"], 8192
    col_group = torch.arange(K, device="cuda") // s["group"]
    for n0 in range(0, s["N"], step):
        byte = s["Wq"][n0:n0 + step].to(torch.int64)
        W = torch.empty(byte.shape[0], K, dtype=torch.float64, device="cuda")
        W[:, 0::2] = (byte % 16).double()
        W[:, 1::2] = (byte // 16).double()
        W -= s["zp"][n0:n0 + step].double()[:, col_group] if s["zp"] is not None else 8
        W *= s["scales"][n0:n0 + step].double()[:, col_group]
        parts.append(torch.einsum("mk,nk->mn", x, W))
    return torch.cat(parts, 1)


def _exact_logits(s):
    M, V, k = s["M"], s["V"], s["k"]
    ids, lps, lses, rows_out = [], [], [], []
    one = lambda name, m: s[name][s["row_seq"][m]].double()

    def part(name, q):
        if s[name + "_tokens"] is None:
            return None, None
        a, b = s[name + "_offsets"][q].item(), s[name + "_offsets"][q + 1].item()
        return s[name + "_tokens"][a:b].long(), slice(a, b)

    for m in range(M):
        q = s["row_seq"][m].item()
        z = s["logits"][m].double()
        out, _ = part("output", q)
        n = torch.zeros(V, dtype=torch.int64, device="cuda") if out is None else torch.bincount(out, minlength=V)
        if s["path_tokens"] is not None:
            p = s["path_tokens"][m]
            n = n + torch.bincount(p[p >= 0].long(), minlength=V)
        prompt, _ = part("prompt", q)
        known = n if prompt is None else n + torch.bincount(prompt, minlength=V)
        z = torch.where(known > 0, torch.where(z > 0, z / one("repetition", m), z * one("repetition", m)), z)
        z = z - one("frequency", m) * n.double() - one("presence", m) * (n > 0).double()
        at, where = part("bias", q)
        if at is not None:
            z[at] += s["bias_values"][where].double()
        if s["mask_words"] is not None and s["mask_rows"][m].item() >= 0:
            word = s["mask_words"][s["mask_rows"][m].item()].long()
            j = torch.arange(V, device="cuda")
            z = z.masked_fill((word[j // 32] >> (j % 32)) & 1 == 0, -math.inf)
        lse = torch.logsumexp(z, 0)
        v, i = torch.sort(z, descending=True, stable=True)
        v, i = v[:k], i[:k]
        ids.append(torch.where(v == -math.inf, NO_TOKEN, i).int())
        lps.append(torch.where(v == -math.inf, v, v - lse))
        lses.append(lse)
        if s["write"]:
            rows_out.append(z)
    out = dict(ids=torch.stack(ids), logprobs=torch.stack(lps), lse=torch.stack(lses))
    if s["write"]:
        out["logits"] = torch.stack(rows_out)
    return out


def _exact_norm(s, back):
    """The formula in 64 bits; the gradients are autograd's."""
    leaf = {n: s[n].double().requires_grad_(back) for n in ("block", "resid", "w_pre", "w_post", "g") if s[n] is not None}

    def rms(v, w):
        return w * v / (v.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS).sqrt()

    b = rms(leaf["block"], leaf["w_post"]) if "w_post" in leaf else leaf["block"]
    if "g" in leaf:
        b = b * (leaf["g"][:, None] if s["gate"] == "row" else leaf["g"])
    y = leaf["resid"] * s["alpha"] + b
    h = rms(y, leaf["w_pre"])
    if not back:
        return dict(stream=y, hidden=h)
    names = [n for n in ("block", "resid", "w_pre", "w_post", "g") if n in leaf]
    grads = torch.autograd.grad([y, h], [leaf[n] for n in names], [s["d_stream"].double(), s["d_hidden"].double()])
    return {"d_gate" if n == "g" else "d_" + n: v for n, v in zip(names, grads)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "q4":
        return _exact_q4(s)
    if case["op"] == "logits":
        return _exact_logits(s)
    return _exact_norm(s, case["op"] == "norm_backward")
