"""The drafter's attention as a program runs it: a block norm makes the rows, a projection (plain matmul) the queries, keys and values;
these are normed and rotated, the prompt attends to itself and goes into the 4-bit cache; then draft steps append tokens and
attend to the pages, the last one with the nodes of a tree, and the prompt's next part attends to what the cache gives back.  Each step
is checked against its oracle on the very input that the step before gave it, with the tolerances of its own tests; the whole run
eagerly, on streams of its own and as replayed graphs."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2502_16880_b200 import lmhead
from tests import test_gpu_kv4 as kv4
from tests import test_gpu_prompt_attention as prompt
from tests import test_gpu_qk_rotate as qk

pytestmark = pytest.mark.gpu
N_Q, N_K, D, GROUP, PAGE, H = 8, 2, 64, 32, 16, 256
LENS, NODES = [70, 33, 5], 6
ALL = N_Q + 2 * N_K


class Layer:
    def __init__(self, seed, t):
        g = torch.Generator().manual_seed(seed)
        self.t, n = t, len(LENS)
        rnd = lambda *s: torch.randn(*s, generator=g).to(t).cuda()
        self.w_qkv, self.w_pre = (rnd(H, ALL * D) * 0.1).to(t), (1 + 0.1 * rnd(H)).to(t)
        self.w_q, self.w_k = ((1 + 0.2 * rnd(D)).to(t) for _ in range(2))
        self.freqs = qk._freqs(D).cuda()
        self.off = prompt._offsets(LENS)
        self.x, self.x_next = rnd(sum(LENS), H), rnd(n * NODES, H)
        at = [np.arange(x) for x in LENS]
        width = -(-(max(LENS) + NODES) // PAGE)
        self.table = torch.randperm(n * width + 1, generator=g)[:n * width].view(n, width).int()
        slot = lambda s, j: self.table[s].long()[torch.from_numpy(j) // PAGE] * PAGE + torch.from_numpy(j) % PAGE
        self.pos = torch.from_numpy(np.concatenate(at)).int().cuda()
        self.slots = torch.cat([slot(s, j) for s, j in enumerate(at)]).cuda()
        new = [x + np.arange(NODES) for x in LENS]
        self.pos_next = torch.from_numpy(np.concatenate(new)).int().cuda()
        self.slots_next = torch.cat([slot(s, j) for s, j in enumerate(new)]).cuda()
        self.lens = torch.tensor([x + NODES for x in LENS], dtype=torch.int32).cuda()
        self.masks = [[sum(1 << b for b in range(i + 1) if b == i or b % 2 == i % 2) for i in range(NODES)] for _ in LENS]
        self.mask = torch.tensor([w for m in self.masks for w in m]).cuda()
        self.cache = lmhead.Kv4Cache(n * width + 1, PAGE, N_K, D, group=GROUP, dtype=t)
        self.cache.pages.fill_(255)
        e = lambda T, h: torch.empty(T, h, D, dtype=t, device="cuda")
        self.h, self.h_next = torch.empty_like(self.x), torch.empty_like(self.x_next)
        self.q, self.k, self.out, self.q_next, self.k_next, self.out_next = (e(T, h) for T in (sum(LENS), n * NODES) for h in (N_Q, N_K, N_Q))
        self.lse, self.lse_next = (torch.empty(T, N_Q, device="cuda") for T in (sum(LENS), n * NODES))
        self.fused, self.fused_next = (torch.empty(T, ALL * D, dtype=t, device="cuda") for T in (sum(LENS), n * NODES))
        self.table = self.table.cuda()

    def run(self, stream=None):
        with torch.cuda.stream(torch.cuda.current_stream() if stream is None else stream):
            for x, h, fused, q, k, pos, slots in ((self.x, self.h, self.fused, self.q, self.k, self.pos, self.slots),
                                                  (self.x_next, self.h_next, self.fused_next, self.q_next, self.k_next, self.pos_next, self.slots_next)):
                lmhead.coral_lmhead_block_norm(x, None, self.w_pre, 1e-5, None, h)
                torch.matmul(h, self.w_qkv, out=fused)
                rows = fused.view(-1, ALL, D)
                lmhead.coral_lmhead_qk_rotate(rows[:, :N_Q], rows[:, N_Q:N_Q + N_K], pos, self.freqs, q, k, w_q=self.w_q, w_k=self.w_k, eps=qk.EPS)
                self.cache.store(k, rows[:, N_Q + N_K:], slots)
                if x is self.x:
                    lmhead.coral_lmhead_prompt_attention(q, k, rows[:, N_Q + N_K:], self.off, self.out, out_lse=self.lse)
                else:
                    self.cache.attend(q, self.table, self.lens, max_q=NODES, tree_mask=self.mask, out=self.out_next, out_lse=self.lse_next)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.h, self.q, self.k, self.out, self.lse, self.q_next, self.k_next, self.out_next, self.lse_next)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_steps_match_the_oracles(t):
    L = Layer(1, t)
    L.run()
    L.results()
    f = qk._np(L.freqs)
    for fused, q, k, pos in ((L.fused, L.q, L.k, L.pos), (L.fused_next, L.q_next, L.k_next, L.pos_next)):
        rows = qk._np(fused.view(-1, ALL, D))
        qk._close(q, *ao.qk(rows[:, :N_Q], qk._np(L.w_q), pos.cpu().numpy(), f, False, qk.EPS), 32, "q")
        qk._close(k, *ao.qk(rows[:, N_Q:N_Q + N_K], qk._np(L.w_k), pos.cpu().numpy(), f, False, qk.EPS), 32, "k")
    v, v_next = (x.view(-1, ALL, D)[:, N_Q + N_K:] for x in (L.fused, L.fused_next))
    prompt._close(dict(q=L.q, k=L.k, v=v, lens=LENS, k_lens=LENS), (L.out, L.lse))
    # what the cache stands for, from the tokens that went in
    c = kv4.Case.__new__(kv4.Case)
    c.t, c.D, c.n_q, c.n_k, c.q, c.masks, c.cache = t, D, N_Q, N_K, L.q_next, L.masks, L.cache
    c.lens, c.n = [x + NODES for x in LENS], [NODES] * len(LENS)
    c.k, c.v, c.ksize, c.vsize, c.vstep, a = [], [], [], [], [], 0
    for s, n in enumerate(LENS):
        for old, new, value, size, steps in ((L.k, L.k_next, c.k, c.ksize, []), (v, v_next, c.v, c.vsize, c.vstep)):
            x = torch.cat((old[a:a + n], new[s * NODES:(s + 1) * NODES])).double().cpu().numpy()
            low, step, codes, border = ao.held(x, GROUP, lambda y: torch.from_numpy(y).to(t).double().numpy())
            # no quotient that fp32 could round to another code (one in the very middle is exact in fp32 too, and goes to the even code)
            assert ((border > 2.0 ** -19) | (border == 0)).all()
            value.append(ao.stands_for(low, step, codes))
            size.append(np.broadcast_to(np.abs(low) + 15 * step, codes.shape).reshape(x.shape))
            steps.append(np.broadcast_to(step, codes.shape).reshape(x.shape))
        a += n
    c.check((L.out_next, L.lse_next))


def test_the_next_part_of_a_prompt_over_what_the_cache_gives_back():
    """The prompt's last rows over keys loaded from the cache: what attention over the cache itself gives, up to what each rounds."""
    L = Layer(2, torch.bfloat16)
    L.run()
    a = 0
    for s, n in enumerate(LENS):
        m = min(n, NODES)
        k, v = L.cache.load(L.slots[a:a + n])
        out = torch.empty(m, N_Q, D, dtype=L.t, device="cuda")
        lmhead.coral_lmhead_prompt_attention(L.q[a + n - m:a + n], k, v, prompt._offsets([m]), out, k_offsets=prompt._offsets([n]))
        got = L.cache.attend(L.q[a + n - m:a + n], L.table[s:s + 1], torch.tensor([n], dtype=torch.int32, device="cuda"), max_q=m)
        # keys rounded to 2^-8 of themselves move a score by 2^-8 sum |q k| / 8, values and weights as much relative
        size = torch.einsum("ihd,jhd->ihj", L.q[a + n - m:a + n].abs().float(), k.abs().float().repeat_interleave(N_Q // N_K, 1)).amax(-1, keepdim=True) / 8
        tol = (2 * 2.0 ** -8 * size + 4 * 2.0 ** -8) * v.abs().float().amax(0).repeat_interleave(N_Q // N_K, 0)
        assert ((out.float() - got.float()).abs() <= tol).all()
        a += n


def test_stream_graph_and_two_at_once():
    L, other = Layer(3, torch.bfloat16), Layer(4, torch.float16)
    L.run()
    other.run()
    want = [x.results() for x in (L, other)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for x in (L, other):
        for t in (x.h, x.q, x.k, x.out, x.q_next, x.out_next, x.cache.pages):
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        L.run(streams[0])
        other.run(streams[1])
    assert all(torch.equal(a, b) for x, w in zip((L, other), want) for a, b in zip(x.results(), w))
    graphs = []
    for x in (L, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
        for t in (x.h, x.q, x.k, x.out, x.q_next, x.out_next, x.cache.pages):
            t.zero_()
    torch.cuda.synchronize()
    for g, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            for _ in range(3):
                g.replay()
    assert all(torch.equal(a, b) for x, w in zip((L, other), want) for a, b in zip(x.results(), w))
