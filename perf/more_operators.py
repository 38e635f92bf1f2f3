"""What the operators of the drafter's attention are measured on: norms of queries and keys for each head with the position
rotation (forward and backward), attention over whole prompts (causal, grouped heads, packed sequences, keys cached before), and
the cache held in 4 bits: storing tokens and reading them back, and attention of few queries (the next token of each
sequence, or the nodes of a draft tree) over its pages.

`run` computes a case in elementary torch operations where `own` is false, and by the library's calls where it is true.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
STYLES = {"halves": 0, "pairs": 1}                               # CORAL_ROPE_*
EPS = 1e-6


def listed():
    return [
        # a prompt of 16384 tokens, 32 query and 8 key heads of 128, rotated whole: what stands in front of prompt attention
        dict(name="qk_prompt_16k", op="qk", T=16384, n_q=32, n_k=8, D=128, rot=128, style="halves", type="bf16", norm=True, base=500000.0, far=0),
        # the next token of one sequence far out in a long context, out of a fused projection: latency
        dict(name="qk_one_token", op="qk", T=1, n_q=28, n_k=4, D=128, rot=128, style="halves", type="bf16", norm=True, base=1000000.0, far=130000),
        # training: four sequences of 2048 tokens
        dict(name="qk_backward_8k", op="qk_backward", T=8192, n_q=32, n_k=8, D=128, rot=128, style="halves", type="bf16", norm=True, base=500000.0, far=0),
        # training, an odd number of tokens, half of a small head rotated in pairs, fp16
        dict(name="qk_backward_odd", op="qk_backward", T=777, n_q=12, n_k=12, D=64, rot=32, style="pairs", type="f16", norm=True, base=10000.0, far=0),
        # one long prompt
        dict(name="prompt_8k", op="prompt", lens="8192", prefix=0, n_q=32, n_k=8, D=128, type="bf16"),
        # nine prompts of one batch, packed, with seven query heads to a key head
        dict(name="prompt_packed", op="prompt", lens="2048 1531 1024 777 512 300 129 64 1", prefix=0, n_q=28, n_k=4, D=128, type="bf16"),
        # short questions behind a part that is cached already, small heads with a key head each, fp16
        dict(name="prompt_short", op="prompt", lens="33 17 130 5", prefix=700, n_q=12, n_k=12, D=64, type="f16"),
        # a prompt's keys and values into the cache, and back for the next part of the prompt
        dict(name="kv4_store_16k", op="kv4_store", T=16384, n_k=8, D=128, group=128, page=64, type="bf16"),
        # one token of each of 64 sequences
        dict(name="kv4_store_64", op="kv4_store", T=64, n_k=4, D=128, group=64, page=16, type="bf16"),
        # the next token of one sequence with a long context: the cache is read once, split over the GPU
        dict(name="kv4_long_context", op="kv4", n_seq=1, longest=131072, nodes=1, tree=False, n_q=32, n_k=8, D=128, group=128, page=64, type="bf16"),
        # the next token of 64 sequences of different lengths
        dict(name="kv4_batch_64", op="kv4", n_seq=64, longest=4096, nodes=1, tree=False, n_q=28, n_k=4, D=128, group=64, page=16, type="bf16"),
        # the 60 nodes of the draft trees of 8 sequences
        dict(name="kv4_trees", op="kv4", n_seq=8, longest=3001, nodes=60, tree=True, n_q=32, n_k=8, D=128, group=32, page=32, type="f16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["qk", "qk_backward", "prompt", "prompt", "kv4_store", "kv4", "kv4"])
    kind = rng.choice(["bf16", "f16"])
    if op in ("qk", "qk_backward"):
        kind = rng.choice(["bf16", "f16", "f32"])
        D = 8 * rng.randint(4, 32)
        n_k = rng.choice([1, 2, 3, 4, 8])
        n_q = n_k * rng.choice([1, 3, 4, 7])
        most = (16384 if op == "qk" else 8192) * 40 * 128 // (D * (n_q + n_k) * (2 if kind == "f32" else 1))
        return dict(op=op, T=_log(rng, 1, min(20000, most)), n_q=n_q, n_k=n_k, D=D, rot=rng.choice([D, 8 * rng.randint(1, D // 8)]),
                    style=rng.choice(["halves", "pairs"]), type=kind, norm=rng.random() < 0.7, base=rng.choice([10000.0, 500000.0]),
                    far=rng.choice([0, _log(rng, 1, 1000000)]))
    n_k, G = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 3, 4, 7, 8])
    if op == "prompt":
        D = rng.choice([64, 128, 128, 8 * rng.randint(2, 16)])
        n_seq = _log(rng, 1, 12)
        longest = _log(rng, 1, min(6000, int(math.sqrt(2 ** 30 / (n_seq * n_k * G)))))
        lens = [longest] + [_log(rng, 1, longest) for _ in range(n_seq - 1)]
        return dict(op=op, lens=" ".join(map(str, lens)), prefix=rng.choice([0, 0, _log(rng, 1, 2000)]), n_q=n_k * G, n_k=n_k, D=D, type=kind)
    D = rng.choice([64, 128])
    group = rng.choice([g for g in (32, 64, 128) if g <= D])
    page = rng.choice([16, 32, 48, 64, 256])
    if op == "kv4_store":
        return dict(op=op, T=_log(rng, 1, 16384 * 8 // max(8, n_k)), n_k=n_k, D=D, group=group, page=page, type=kind)
    n_seq = _log(rng, 1, 64)
    nodes, tree = rng.choice([(1, False), (1, False), (rng.randint(2, 16), False), (rng.randint(2, 64), True)])
    longest = nodes + _log(rng, 1, max(1, min(65536, 64 * 4096 * 4 // (n_seq * n_k * (1 if nodes == 1 else 2)))))
    return dict(op=op, n_seq=n_seq, longest=longest, nodes=nodes, tree=tree, n_q=n_k * G, n_k=n_k, D=D, group=group, page=page, type=kind)


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _keys(g, T, n_k, D, dtype):
    """Keys as a model has them: some channels lie off zero for every token."""
    return (torch.randn(T, n_k, D, generator=g, device="cuda") + 2.0 * torch.randn(n_k, D, generator=g, device="cuda")).to(dtype)


# ---- what a program has in hand ------------------------------------------------------------------------------
def _prepare_qk(case, g):
    T, n_q, n_k, D, t = case["T"], case["n_q"], case["n_k"], case["D"], TYPES[case["type"]]
    s = dict(case)
    fused = _normal(g, (T, n_q + 2 * n_k, D), 1.5, t)            # a fused projection: queries, keys, values
    s["q"], s["k"] = fused[:, :n_q], fused[:, n_q:n_q + n_k]
    s["positions"] = (torch.arange(T, device="cuda") + case["far"]).int()
    s["freqs"] = (case["base"] ** -(torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])).float()
    s["w_q"], s["w_k"] = ((1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(t) if case["norm"] else None for _ in range(2))
    new = lambda h: torch.empty(T, h, D, dtype=t, device="cuda")
    if case["op"] == "qk":
        s["out_q"], s["out_k"] = new(n_q), new(n_k)
        return s
    s["d_out_q"], s["d_out_k"] = _normal(g, (T, n_q, D), 1.0, t), _normal(g, (T, n_k, D), 1.0, t)
    s["dq"], s["dk"] = new(n_q), new(n_k)
    s["dw_q"], s["dw_k"] = (torch.empty(D, device="cuda") if case["norm"] else None for _ in range(2))
    if own:
        from paper_2502_16880_b200 import lmhead
        s["workspace"] = torch.empty(lmhead.coral_lmhead_qk_rotate_backward_bytes(T, n_q, n_k, D), dtype=torch.uint8, device="cuda")
    return s


def _prepare_prompt(case, g):
    n_q, n_k, D, t = case["n_q"], case["n_k"], case["D"], TYPES[case["type"]]
    lens = [int(n) for n in case["lens"].split()]
    s = dict(case)
    s["n_seq"], s["most"], T = len(lens), max(lens), sum(lens)
    s["q_offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device="cuda")
    s["k_offsets"] = s["q_offsets"] + case["prefix"] * torch.arange(len(lens) + 1, device="cuda")
    Tk = T + case["prefix"] * len(lens)
    s["q"] = _normal(g, (T, n_q, D), 1.0, t)
    s["k"], s["v"] = _keys(g, Tk, n_k, D, t), _normal(g, (Tk, n_k, D), 1.0, t)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(T, n_q, device="cuda")
    return s


def _lens_of(case):
    """Lengths of the sequences: the first is the longest, the others fall to about half of it."""
    return [max(case["nodes"], case["longest"] - i * (case["longest"] // (2 * case["n_seq"]))) for i in range(case["n_seq"])]


def _prepare_kv4(case, g):
    n_k, D, P, t = case["n_k"], case["D"], case["page"], TYPES[case["type"]]
    s = dict(case)
    if case["op"] == "kv4_store":
        pages = -(-case["T"] // P) + 3
        s["slots"] = torch.randperm(pages, generator=g, device="cuda").repeat_interleave(P)[:case["T"]] * P + torch.arange(case["T"], device="cuda") % P
        s["k"], s["v"] = _keys(g, case["T"], n_k, D, t), _normal(g, (case["T"], n_k, D), 1.0, t)
        s["got_k"], s["got_v"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    else:
        lens = _lens_of(case)
        width = -(-case["longest"] // P)
        pages = case["n_seq"] * width
        s["table"] = torch.randperm(pages, generator=g, device="cuda").int().view(case["n_seq"], width)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        k, v = _keys(g, pages * P, n_k, D, t), _normal(g, (pages * P, n_k, D), 1.0, t)
        s["q"] = _normal(g, (case["n_seq"] * case["nodes"], case["n_q"], D), 1.0, t)
        s["mask"] = None
        if case["tree"]:                                         # a node sees itself and its ancestors
            parent = (torch.rand(case["n_seq"], case["nodes"], generator=g, device="cuda") * torch.arange(case["nodes"], device="cuda")).long().tolist()
            words = [[0] * case["nodes"] for _ in range(case["n_seq"])]
            for w, p in zip(words, parent):
                for i in range(case["nodes"]):
                    w[i] = 1 << i | (w[p[i]] if i else 0)
            s["mask"] = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in w] for w in words], device="cuda").view(-1)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    if own:
        from paper_2502_16880_b200 import lmhead
        s["cache"] = lmhead.Kv4Cache(pages, P, n_k, D, group=case["group"], dtype=t, device="cuda")
        if case["op"] == "kv4":
            s["cache"].store(k, v, torch.arange(pages * P, device="cuda"))
    elif case["op"] == "kv4":
        s["codes"] = tuple(_quantise(x, case["group"]) for x in (k, v))
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"qk": _prepare_qk, "qk_backward": _prepare_qk, "prompt": _prepare_prompt, "kv4_store": _prepare_kv4, "kv4": _prepare_kv4}[case["op"]](case, g)


# ---- the plain forms ---------------------------------------------------------------------------------------
def _angles(s):
    a = s["positions"].double().unsqueeze(1) * s["freqs"].double()
    return a.cos().float().unsqueeze(1), a.sin().float().unsqueeze(1)


def _split(x, s):
    """The two members of each rotated pair, and the columns that are not rotated."""
    r = s["rot"]
    if s["style"] == "halves":
        return x[..., :r // 2], x[..., r // 2:r], x[..., r:]
    return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]


def _join(a, b, rest, s):
    return torch.cat((torch.cat((a, b), -1) if s["style"] == "halves" else torch.stack((a, b), -1).flatten(-2), rest), -1)


def _plain_qk(s):
    cos, sin = _angles(s)

    def one(x, w):
        t, x = x.dtype, x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        a, b, rest = _split(x, s)
        return _join(a * cos - b * sin, b * cos + a * sin, rest, s).to(t)
    return dict(q=one(s["q"], s["w_q"]), k=one(s["k"], s["w_k"]))


def _plain_qk_backward(s):
    cos, sin = _angles(s)

    def one(x, w, d):
        t, x = x.dtype, x.float()
        a, b, rest = _split(d.float(), s)
        d = _join(a * cos + b * sin, b * cos - a * sin, rest, s)
        if w is None:
            return d.to(t), None
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n = x * r
        dn = d * w.float()
        return (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(t), (d * n).sum((0, 1))
    (dq, dw_q), (dk, dw_k) = one(s["q"], s["w_q"], s["d_out_q"]), one(s["k"], s["w_k"], s["d_out_k"])
    return dict(dq=dq, dk=dk, dw_q=dw_q, dw_k=dw_k) if s["norm"] else dict(dq=dq, dk=dk)


def _attend(q, k, v, seen):
    """q [B, Lq, n_q, D], k, v [B, Lk, n_k, D], seen [B, Lq, Lk]: outputs and log-sum-exp, rows that see nothing 0 and -inf."""
    B, Lq, n_q, D = q.shape
    n_k = k.shape[2]
    z = torch.matmul(q.view(B, Lq, n_k, n_q // n_k, D).permute(0, 2, 3, 1, 4), k.permute(0, 2, 3, 1).unsqueeze(2))
    z.mul_(D ** -0.5).masked_fill_(~seen[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.permute(0, 2, 1, 3).unsqueeze(2)) / torch.where(total == 0, 1.0, total)
    lse = (total.log() + m).squeeze(-1)
    return out.permute(0, 3, 1, 2, 4).reshape(B, Lq, n_q, D), lse.permute(0, 3, 1, 2).reshape(B, Lq, n_q)


def _plain_prompt(s):
    most_k = s["most"] + s["prefix"]
    nq, nk = (o[1:] - o[:-1] for o in (s["q_offsets"], s["k_offsets"]))
    i, j = torch.arange(s["most"], device="cuda"), torch.arange(most_k, device="cuda")
    at_q = (s["q_offsets"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    at_k = (s["k_offsets"][:-1, None] + j).clamp(max=s["k"].shape[0] - 1)
    seen = j <= i[:, None] + (nk - nq)[:, None, None]
    out, lse = _attend(s["q"].float()[at_q], s["k"].float()[at_k], s["v"].float()[at_k], seen)
    real = i < nq[:, None]
    return dict(out=out[real].to(s["q"].dtype), lse=lse[real])


def _quantise(x, group):
    """Codes 0..15 of each group of columns, two to a byte, and the group's step and lowest value in the type of x."""
    T, h, D = x.shape
    g = x.float().view(T, h, D // group, group)
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    step = ((high - low) / 15).to(x.dtype)
    code = torch.where(step > 0, torch.round((g - low) / step.float()).clamp(0, 15), 0.0).to(torch.uint8).view(T, h, D)
    return code[..., 0::2] | code[..., 1::2] << 4, step.squeeze(-1), low.squeeze(-1).to(x.dtype)


def _values(packed, step, low):
    code = torch.stack((packed & 15, packed >> 4), -1).float()
    return (code.view(*step.shape, -1) * step.float().unsqueeze(-1) + low.float().unsqueeze(-1)).view(*packed.shape[:-1], -1)


def _plain_kv4_store(s):
    return dict(k=_values(*_quantise(s["k"], s["group"])).to(s["k"].dtype), v=_values(*_quantise(s["v"], s["group"])).to(s["v"].dtype))


def _plain_kv4(s):
    P, nodes, B = s["page"], s["nodes"], s["n_seq"]
    j = torch.arange(s["longest"], device="cuda")
    slot = s["table"].long()[:, j // P] * P + j % P
    k, v = (_values(*(part[slot] for part in c)) for c in s["codes"])
    at = j - (s["lens"].long()[:, None, None] - nodes)           # 0 ...: the position among the new tokens
    i = torch.arange(nodes, device="cuda")[:, None]
    if s["mask"] is None:
        seen = at <= i
    else:
        bit = (s["mask"].view(B, nodes, 1) >> at.clamp(0, 63)) & 1
        seen = (at < 0) | ((bit == 1) & (at < nodes))
    seen = seen & (j < s["lens"][:, None, None])
    out, lse = _attend(s["q"].float().view(B, nodes, s["n_q"], s["D"]), k, v, seen.expand(B, nodes, -1))
    return dict(out=out.reshape(s["q"].shape).to(s["q"].dtype), lse=lse.reshape(s["lse"].shape))


# ---- the library's calls -----------------------------------------------------------------------------------
def _own_qk(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_qk_rotate(s["q"], s["k"], s["positions"], s["freqs"], s["out_q"], s["out_k"], w_q=s["w_q"], w_k=s["w_k"],
                                  eps=EPS, style=STYLES[s["style"]])
    return dict(q=s["out_q"], k=s["out_k"])


def _own_qk_backward(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_qk_rotate_backward(
        s["q"], s["k"], s["positions"], s["freqs"], s["d_out_q"], s["d_out_k"], s["dq"], s["dk"], w_q=s["w_q"], w_k=s["w_k"], eps=EPS,
        style=STYLES[s["style"]], dw_q=s["dw_q"], dw_k=s["dw_k"], workspace=s["workspace"])
    return dict(dq=s["dq"], dk=s["dk"], dw_q=s["dw_q"], dw_k=s["dw_k"]) if s["norm"] else dict(dq=s["dq"], dk=s["dk"])


def _own_prompt(s):
    from paper_2502_16880_b200 import lmhead
    lmhead.coral_lmhead_prompt_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["out"], k_offsets=s["k_offsets"] if s["prefix"] else None,
                                         out_lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _own_kv4_store(s):
    s["cache"].store(s["k"], s["v"], s["slots"])
    s["cache"].load(s["slots"], out_k=s["got_k"], out_v=s["got_v"])
    return dict(k=s["got_k"], v=s["got_v"])


def _own_kv4(s):
    s["cache"].attend(s["q"], s["table"], s["lens"], max_q=s["nodes"], tree_mask=s["mask"], out=s["out"], out_lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def run(state):
    op = state["op"]
    if own:
        return {"qk": _own_qk, "qk_backward": _own_qk_backward, "prompt": _own_prompt, "kv4_store": _own_kv4_store, "kv4": _own_kv4}[op](state)
    return {"qk": _plain_qk, "qk_backward": _plain_qk_backward, "prompt": _plain_prompt, "kv4_store": _plain_kv4_store, "kv4": _plain_kv4}[op](state)


def work(case):
    D, e, op = case["D"], SIZE[case["type"]], case["op"]
    if op in ("qk", "qk_backward"):
        n = case["T"] * (case["n_q"] + case["n_k"]) * D
        back = op == "qk_backward"
        return {"bytes": n * e * (3 if back and case["norm"] else 2) + 4 * case["T"] + 2 * case["rot"] + (2 * D * (e + 4 * back) if case["norm"] else 0),
                "flops": (14.0 if back else 8.0) * n}
    if op == "prompt":
        lens = [int(x) for x in case["lens"].split()]
        pairs = sum(n * case["prefix"] + n * (n + 1) / 2 for n in lens)
        T, Tk = sum(lens), sum(lens) + case["prefix"] * len(lens)
        return {"bytes": (2 * T * case["n_q"] + 2 * Tk * case["n_k"]) * D * e + 4 * T * case["n_q"], "flops": 4.0 * D * case["n_q"] * pairs}
    token = 2 * case["n_k"] * (D // 2 + 2 * e * (D // case["group"]))      # bytes of a token's keys and values in the cache
    if op == "kv4_store":
        return {"bytes": case["T"] * (4 * case["n_k"] * D * e + 2 * token + 8), "flops": 12.0 * case["T"] * case["n_k"] * D}
    lens = _lens_of(case)
    T = case["n_seq"] * case["nodes"]
    pairs = sum(case["nodes"] * n - (0 if case["tree"] else case["nodes"] * (case["nodes"] - 1) / 2) for n in lens)
    return {"bytes": sum(lens) * token + T * case["n_q"] * (2 * D * e + 4), "flops": 4.0 * D * case["n_q"] * pairs}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------
def _turned(x, s):
    """The rotation as a product with a complex number of size one."""
    r = s["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), s["freqs"].double()))[:, None]
    if s["style"] == "halves":
        z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
        return torch.cat((z.real, z.imag, x[..., r:]), -1)
    z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2)) * turn
    return torch.cat((torch.view_as_real(z).reshape(*x.shape[:-1], r), x[..., r:]), -1)


def _exact_qk(s, back):
    """The formula in 64 bits; the gradients are autograd's."""
    found = {}
    for n in ("q", "k"):
        x = s[n].double().requires_grad_(back)
        leaves = [x]
        y = x
        if s["norm"]:
            leaves.append(s["w_" + n].double().requires_grad_(back))
            y = leaves[1] * x / (x.pow(2).sum(-1, keepdim=True) / s["D"] + EPS).sqrt()
        y = _turned(y, s)
        if not back:
            found[n] = y
            continue
        for name, grad in zip(("d" + n, "dw_" + n), torch.autograd.grad(y, leaves, s["d_out_" + n].double())):
            found[name] = grad
    return found


def _one_head(q, k, v, seen):
    z = (q @ k.t()) / math.sqrt(q.shape[1])
    z = z.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, 1)
    return torch.nan_to_num(torch.softmax(z, 1)) @ v, lse


def _exact_prompt(s):
    outs, lses = [], []
    a, b = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    for n in range(s["n_seq"]):
        nq, nk = a[n + 1] - a[n], b[n + 1] - b[n]
        seen = torch.ones(nq, nk, dtype=torch.bool, device="cuda").tril(nk - nq)
        heads = [_one_head(s["q"][a[n]:a[n + 1], h].double(), s["k"][b[n]:b[n + 1], h * s["n_k"] // s["n_q"]].double(),
                           s["v"][b[n]:b[n + 1], h * s["n_k"] // s["n_q"]].double(), seen) for h in range(s["n_q"])]
        outs.append(torch.stack([o for o, _ in heads], 1))
        lses.append(torch.stack([x for _, x in heads], 1))
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def _held(x, group, dtype):
    """What 4 bits hold of x: the group's lowest value plus a whole number of steps."""
    g = x.double().unflatten(-1, (-1, group))
    low = g.min(-1, keepdim=True).values
    step = ((g.max(-1, keepdim=True).values - low) / 15).to(dtype).double()
    n = torch.nan_to_num(((g - low) / step).round(), nan=0.0).clamp(0, 15)
    return (low + n * step).flatten(-2)


def _exact_kv4(s, case, seed):
    if s["op"] == "kv4_store":
        return {n: _held(s[n], s["group"], s[n].dtype) for n in ("k", "v")}
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    torch.randperm(s["table"].numel(), generator=g, device="cuda")           # as prepare() draws: the table, then the tokens
    T, t = s["table"].numel() * s["page"], TYPES[s["type"]]
    raw = _keys(g, T, s["n_k"], s["D"], t), _normal(g, (T, s["n_k"], s["D"]), 1.0, t)
    rows, lses = [], []
    for b, n in enumerate(s["lens"].tolist()):
        pages = s["table"][b].tolist()
        at = torch.cat([torch.arange(p * s["page"], (p + 1) * s["page"], device="cuda") for p in pages])[:n]
        k, v = (_held(x[at], s["group"], t) for x in raw)
        seen = torch.ones(s["nodes"], n, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen = seen.tril(n - s["nodes"])
        else:
            words = s["mask"].view(-1, s["nodes"])[b].tolist()
            seen[:, n - s["nodes"]:] = torch.tensor([[bool(w >> i & 1) for i in range(s["nodes"])] for w in words], device="cuda")
        q = s["q"].view(-1, s["nodes"], s["n_q"], s["D"])[b].double()
        heads = [_one_head(q[:, h], k[:, h * s["n_k"] // s["n_q"]], v[:, h * s["n_k"] // s["n_q"]], seen) for h in range(s["n_q"])]
        rows.append(torch.stack([o for o, _ in heads], 1))
        lses.append(torch.stack([x for _, x in heads], 1))
    return dict(out=torch.cat(rows), lse=torch.cat(lses))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("qk", "qk_backward"):
        return _exact_qk(s, case["op"] == "qk_backward")
    return _exact_prompt(s) if case["op"] == "prompt" else _exact_kv4(s, case, seed)
