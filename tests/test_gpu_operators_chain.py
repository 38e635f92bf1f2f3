"""Block norm, 4-bit head, logits step and tree expansion one after the other, as a draft step over a dense 4-bit head runs them:
the hidden rows of a level's nodes become the next level's parents.  Each step is checked against its oracle on the very input
that the step before gave it, with the tolerances of its own tests, and the whole run eagerly, on a stream of its own and as a replayed graph."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as nor
from oracle import tree_oracle as tor
from paper_2502_16880_b200 import lmhead
from tests import test_gpu_block_norm as norm
from tests import test_gpu_logits as step
from tests import test_gpu_q4 as q4

pytestmark = pytest.mark.gpu
N_SEQ, NODES, K = 3, 5, 10
M, H, V, GROUP = N_SEQ * NODES, 512, 2003, 64


class Level:
    def __init__(self, seed, t):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.x, self.r = (torch.randn(M, H, generator=g).to(t).cuda() for _ in range(2))
        self.w_pre, self.w_post = ((1 + 0.1 * torch.randn(H, generator=g)).to(t).cuda() for _ in range(2))
        self.Wq = torch.from_numpy(rng.integers(0, 256, (V, H // 2)).astype(np.uint8))
        self.scales = (torch.rand(V, H // GROUP, generator=g) * 0.02 + 0.01).to(t)
        self.head = lmhead.Q4Linear(self.Wq.cuda(), self.scales.cuda())
        self.prompt = torch.from_numpy(rng.integers(0, V, 90).astype(np.int32)).cuda()
        self.off = torch.tensor([0, 50, 50, 90], device="cuda")
        self.path = torch.from_numpy(rng.integers(-1, V, (M, 4)).astype(np.int32)).cuda()
        self.seq = torch.arange(N_SEQ, dtype=torch.int32, device="cuda").repeat_interleave(NODES)
        self.rep, self.freq, self.pres = (torch.tensor(v, device="cuda") for v in ([1.3, 1.0, 2.0], [0.5, 0.0, 0.25], [0.0, 1.0, 0.5]))
        self.mask = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (N_SEQ, (V + 31) // 32)).astype(np.int32)).cuda()
        e = lambda *s, d=torch.float32: torch.empty(*s, dtype=d, device="cuda")
        self.y, self.h, self.logits = e(M, H, d=t), e(M, H, d=t), e(M, V)
        self.ids, self.lps, self.lse, self.out = e(M, K, d=torch.int32), e(M, K), e(M), e(M, V)
        self.parents = torch.from_numpy(-rng.random((N_SEQ, NODES)).astype(np.float32)).cuda()
        self.parent, self.token, self.score = e(N_SEQ, K, d=torch.int32), e(N_SEQ, K, d=torch.int32), e(N_SEQ, K)

    def run(self, stream=None):
        lmhead.coral_lmhead_block_norm(self.x, self.r, self.w_pre, 1e-5, self.y, self.h, w_post=self.w_post, alpha=0.5, stream=stream)
        self.head.forward(self.h, out=self.logits, stream=stream)
        lmhead.coral_lmhead_logits_process(
            self.logits, row_seq=self.seq, prompt_tokens=self.prompt, prompt_offsets=self.off, path_tokens=self.path,
            repetition=self.rep, frequency=self.freq, presence=self.pres, mask_words=self.mask, mask_rows=self.seq,
            out_logits=self.out, out_ids=self.ids, out_logprobs=self.lps, out_lse=self.lse, stream=stream)
        lmhead.coral_tree_expand(self.parents, self.ids.view(N_SEQ, NODES, K), self.lps.view(N_SEQ, NODES, K), K, self.parent,
                                 self.token, self.score, stream)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.y, self.h, self.logits, self.out, self.ids, self.lps, self.parent, self.token, self.score)]


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_level_matches_the_oracles(t):
    lv = Level(1, t)
    lv.run()
    y, h, logits, out, ids, lps, parent, token, score = lv.results()
    d = lambda v: v.double().cpu().numpy()
    wy, wh, sy, sh = nor.forward(d(lv.x), d(lv.r), d(lv.w_pre), 1e-5, d(lv.w_post), None, 0.5)
    norm._close(y, wy, sy, 64, "y")
    norm._close(h, wh, sh, 64, "h")
    q4._check(logits, lv.Wq, lv.scales, None, h.cpu(), GROUP)
    lists = lambda flat: [flat[a:b].tolist() for a, b in zip(lv.off.tolist(), lv.off.tolist()[1:])]
    got = dict(out=out, ids=ids.cpu().numpy(), lps=lps.cpu().numpy(), lse=lv.lse.cpu().numpy())
    step._check(got, logits.cpu(), K, n_seq=N_SEQ, row_seq=lv.seq.cpu(), prompt=lists(lv.prompt.cpu()), path=lv.path.cpu(), rep=lv.rep.tolist(),
                freq=lv.freq.tolist(), pres=lv.pres.tolist(), mask=lv.mask.cpu(), mask_rows=lv.seq.cpu())
    want = tor.expand(lv.parents.cpu().numpy(), got["ids"].reshape(N_SEQ, NODES, K), got["lps"].reshape(N_SEQ, NODES, K), K)
    for g, w in zip((parent, token, score), want):
        assert np.array_equal(g.cpu().numpy(), w)


def test_stream_graph_and_two_at_once():
    lv, other = Level(2, torch.bfloat16), Level(3, torch.bfloat16)
    lv.run()
    other.run()
    first, second = lv.results(), other.results()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for v in (lv, other):
        for t in (v.y, v.h, v.logits, v.out, v.lps, v.score):
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(5):                                       # two levels at a time, their launches in between one another
        lv.run(streams[0])
        other.run(streams[1])
    for v, want in ((lv, first), (other, second)):
        assert all(torch.equal(a, b) for a, b in zip(v.results(), want))
    graphs = []
    for v in (lv, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            v.run()
        graphs.append(g)
    x = lv.x.clone()
    lv.x.copy_(other.x)
    torch.cuda.synchronize()
    lv.run()
    third = lv.results()
    for t in (lv.y, lv.out, lv.score):
        t.zero_()
    torch.cuda.synchronize()
    for g, st in zip(graphs, streams):                       # two captured graphs at once, one with other rows than at its capture
        with torch.cuda.stream(st):
            for _ in range(3):
                g.replay()
    assert all(torch.equal(a, b) for a, b in zip(lv.results(), third))
    assert all(torch.equal(a, b) for a, b in zip(other.results(), second))
    lv.x.copy_(x)
    graphs[0].replay()
    assert all(torch.equal(a, b) for a, b in zip(lv.results(), first))
