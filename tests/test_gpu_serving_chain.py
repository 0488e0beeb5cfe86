"""The serving operators together, as a serving loop uses them: prompts behind a shared prefix, then tokens drawn one by
one, eagerly and as a captured step, against one 64-bit implementation of the whole."""
import math
import threading

import numpy as np
import pytest
import torch

from gpu_common import log
from serving_common import DT, Case
from test_gpu_serving import check_attention, half
from test_gpu_serving_sample import draw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V, H, G, D, PAGE = 1009, 8, 2, 64, 16
PREFIX, PROMPTS, STEPS = 77, [1, 20, 5, 40], 9
SETTINGS = ([1.0, 0.7, 0.0, 1.2], [0, 50, 0, 0], [0.95, 1.0, 1.0, 0.8], [0.0, 0.0, 0.0, 0.02])


class Loop:
    """One attention layer whose queries, keys and values are looked up per token, and a float32 head."""

    def __init__(self, dtype, heads_first):
        from paper_2609_17184_amd import serving
        g = torch.Generator().manual_seed(31)
        self.dtype = DT[dtype]
        self.tq = torch.randn((V, H, D), generator=g).to(self.dtype)
        self.tk, self.tv = (torch.randn((V, G, D), generator=g).to(self.dtype) for _ in range(2))
        self.gq, self.gk = (1 + 0.2 * torch.randn(D, generator=g) for _ in range(2))
        self.head = torch.randn((V, H * D), generator=g) * 0.5
        self.prefix = torch.randint(0, V, (PREFIX,), generator=g)
        self.prompts = [torch.randint(0, V, (n,), generator=g) for n in PROMPTS]
        n, width = len(PROMPTS), -(-(max(PROMPTS) + STEPS) // PAGE)
        pages = torch.randperm(n * width + -(-PREFIX // PAGE), generator=g).to(torch.int32)
        shape = (len(pages), G, PAGE, D) if heads_first else (len(pages), PAGE, G, D)
        k, v = (torch.full(shape, math.nan, dtype=self.dtype, device=DEV) for _ in range(2))
        if not heads_first:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        self.cache = serving.PagedCache(k, v)
        self.table = pages[:n * width].view(n, width).to(DEV)
        self.ptable = pages[n * width:].to(DEV)
        self.seq_len = torch.tensor(PROMPTS, dtype=torch.int32, device=DEV)
        self.freq = serving.rope_frequencies(D)
        self.dev = [t.to(DEV) for t in (self.tq, self.tk, self.tv, self.gq, self.gk, self.head)]
        self.set = [torch.tensor(x, dtype=torch.int32 if i == 1 else torch.float32, device=DEV)
                    for i, x in enumerate(SETTINGS)]

    def layer(self, ids, batch, attend=True):
        from paper_2609_17184_amd import serving
        tq, tk, tv, gq, gk, _ = self.dev
        q = serving.rope_append(tq[ids], tk[ids], tv[ids], self.cache, batch, self.freq, gq, gk, 1e-5)
        return serving.prefix_attention(q, self.cache, batch) if attend else None

    def logits(self, o):
        return (o.flatten(1).float()[:, None] * self.dev[5]).sum(-1)

    def start(self):
        """The prefix and the prompts; the attention output of the prompts' tokens."""
        from paper_2609_17184_amd import serving
        one = torch.tensor([PREFIX], dtype=torch.int32, device=DEV)
        self.layer(self.prefix.to(DEV), serving.Batch(one, self.ptable[None], torch.tensor([0, PREFIX], dtype=torch.int32,
                                                                                           device=DEV)), attend=False)
        starts = torch.tensor(np.cumsum([0] + PROMPTS), dtype=torch.int32, device=DEV)
        return self.layer(torch.cat(self.prompts).to(DEV),
                          serving.Batch(self.seq_len, self.table, starts, PREFIX, self.ptable))

    # ---- 64 bits

    def rot(self, x, gain, positions):
        """Heads [n, heads, D] and the bound of what the rotation mixes."""
        x = x.double()
        x = x * gain.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        a = (positions.double()[:, None] * 1e4 ** (-torch.arange(D // 2, dtype=torch.float64) * 2 / D))[:, None]
        u, w = x[..., :D // 2], x[..., D // 2:]
        mix = u.abs() + w.abs()
        return torch.cat([u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin()], -1), torch.cat([mix, mix], -1)

    def exact(self, ids):
        """Attention of the last token of the whole sequence `ids`, and its tolerance: the query and the keys are
        rounded once (h each, and 2^-19 of what is mixed), which moves a score by ds and a weight by exp(2 ds); weights
        and output are rounded once more each."""
        h, per = half(self.dtype), H // G
        pos = torch.arange(len(ids))
        K, mk = self.rot(self.tk[ids], self.gk, pos)
        q, mq = self.rot(self.tq[ids[-1:]], self.gq, pos[-1:])
        K, mk, W = (x.repeat_interleave(per, 1) for x in (K, mk, self.tv[ids].double()))
        s = (K * q).sum(-1) * D ** -0.5
        ds = ((mk * mq).sum(-1).amax(0) * D ** -0.5 * (2 * h + h * h + 2.0 ** -17))[:, None]
        p = torch.softmax(s, 0)[..., None]
        ref, mean = (p * W).sum(0), (p * W.abs()).sum(0)
        return ref, mean * (torch.expm1(2 * ds) + 2 * h) + ref.abs() * h + len(ids) * 2.0 ** -30 + 2.0 ** -25


def close(got, ref, tol):
    err = (got.cpu().double() - ref).abs()
    assert (err <= tol).all(), (err - tol).max()
    return (err / tol).max().item()


@pytest.mark.parametrize("dtype,heads_first", [("f16", True), ("bf16", False)])
def test_prompt_then_tokens(dtype, heads_first):
    from paper_2609_17184_amd import serving
    m = Loop(dtype, heads_first)
    n = len(PROMPTS)
    seqs = [torch.cat([m.prefix, p]) for p in m.prompts]
    o = m.start()
    worst, at = 0.0, 0
    for b, p in enumerate(PROMPTS):
        for i in range(p):
            worst = max(worst, close(o[at + i], *m.exact(seqs[b][:PREFIX + i + 1])))
        at += p
    last = torch.tensor(np.cumsum(PROMPTS) - 1, device=DEV)
    rng = np.random.default_rng(32)
    uniform = rng.random((STEPS + 1, n))
    u = torch.zeros(n, dtype=torch.float64, device=DEV)
    ids = torch.zeros(n, dtype=torch.int64, device=DEV)
    live = torch.ones(n, dtype=torch.int32, device=DEV)
    batch = serving.Batch(m.seq_len, m.table, None, PREFIX, m.ptable)

    def choose(o):
        z = m.logits(o)
        drawn = serving.sample(z, u, *m.set)
        ids.copy_(drawn[0].clamp(min=0))
        return z, drawn

    def step():
        m.seq_len.add_(live)
        o = m.layer(ids, batch)
        return (o, *choose(o))

    def check_draws(z, drawn, turn):
        f32 = lambda x: float(np.float32(x))
        for b in range(n):
            if not live[b]:
                continue
            t, k, p, mp = (s[b] for s in SETTINGS)
            token, prob, kept = draw(z[b].cpu().numpy(), uniform[turn, b], f32(t), k, f32(p), f32(mp))
            assert drawn[0][b].item() == token and drawn[2][b].item() == kept
            assert abs(drawn[1][b].item() - prob) <= 2.0 ** -26 + 2.0 ** -24 * prob
            seqs[b] = torch.cat([seqs[b], torch.tensor([token])])

    def end(turn):
        """The third sequence ends after the fourth token."""
        if turn == 4:
            live[2] = 0
            m.seq_len[2] = -1

    u.copy_(torch.tensor(uniform[0]))
    check_draws(*choose(o[last]), 0)
    saved = [t.clone() for t in (m.cache.k, m.cache.v, m.seq_len, ids, live)]
    history = []
    for turn in range(1, STEPS + 1):
        end(turn)
        u.copy_(torch.tensor(uniform[turn]))
        o, z, drawn = step()
        for b in range(n):
            if live[b]:
                worst = max(worst, close(o[b], *m.exact(seqs[b])))
        check_draws(z, drawn, turn)
        history.append([x.clone() for x in drawn])
    assert m.seq_len.tolist() == [p + STEPS if b != 2 else -1 for b, p in enumerate(PROMPTS)]
    log(f"[chain] {dtype}: worst {worst:.2f} of tolerance, {[len(s) for s in seqs]} positions")
    after = [m.cache.k.clone(), m.cache.v.clone()]

    # the same steps as one captured graph
    def rewind():
        for t, s in zip((m.cache.k, m.cache.v, m.seq_len, ids, live), saved):
            t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, _, drawn = step()
    for _ in range(2):
        rewind()
        for turn in range(1, STEPS + 1):
            end(turn)
            u.copy_(torch.tensor(uniform[turn]))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            keep = live.bool()
            for a, b in zip(drawn, history[turn - 1]):
                assert torch.equal(a[keep], b[keep])
        for a, b in zip((m.cache.k, m.cache.v), after):
            assert torch.equal(a.nan_to_num(7), b.nan_to_num(7))


def test_two_threads_share_a_batch():
    """Two threads on streams of their own, one batch and cache, different numbers of padding rows."""
    from paper_2609_17184_amd import serving
    c = Case(8, 2, 64, 16, "f16", [2, 1, 3], [30, 60, 17], 90, seed=33, extra=40)
    q = c.q.to(DEV)
    ref = {}                                  # (how the work is split follows the number of rows, and so do last bits)
    for rows in (6, 46):
        out, lse = serving.prefix_attention(q[:rows], c.cache, c.batch, return_lse=True)
        check_attention(c, 0.125, torch.cat([out, q[rows:]]), lse, torch.cat([out, q[rows:]]).cpu())
        ref[rows] = out[:6]
    z = torch.randn((5, 9000), device=DEV)
    u = torch.rand(5, dtype=torch.float64, device=DEV)
    tokens = serving.sample(z, u, 0.8, 40)[0]
    torch.cuda.synchronize()
    wrong = []

    def work(rows):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(60):
                out = serving.prefix_attention(q[:rows], c.cache, c.batch)
                if not torch.equal(out[:6], ref[rows]) or not torch.equal(serving.sample(z, u, 0.8, 40)[0], tokens):
                    wrong.append(rows)
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(rows,)) for rows in (6, 46)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
