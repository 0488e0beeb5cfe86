"""Attention under a window for batches of many sequences, whose tasks go to single waves, and behind a prefix that is worked
on for all of them at once."""
import math

import pytest
import torch

from gpu_common import log
from quantized_common import Quantized, behind_a_prefix, check_window, windowed
from serving_common import Case
from test_gpu_window import attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# heads, key/value heads, head_dim, page, type, tokens and own positions per sequence, prefix
BATCHES = [
    (16, 8, 64, 16, "bf16", [1] * 80, [i * 13 % 90 + 1 for i in range(80)], 133),
    (32, 8, 32, 16, "f16", [4] * 70, [i * 7 % 60 + 4 for i in range(70)], 50),       # 16 rows of a head each
    (32, 8, 32, 16, "bf16", [6] * 70, [i * 7 % 60 + 6 for i in range(70)], 50),      # 24 rows: two tiles of 16
    (32, 8, 32, 16, "f16", [8] * 65, [i * 5 % 50 + 8 for i in range(65)], 0),        # 32 rows
    (32, 8, 32, 16, "f16", [9] * 65, [i * 5 % 50 + 9 for i in range(65)], 20),       # 36 rows: blocks of many rows
    (55, 55, 96, 16, "f16", [1] * 12, [i * 31 % 200 + 1 for i in range(12)], 40),
    (8, 8, 128, 48, "bf16", [i % 4 for i in range(150)], [i * 11 % 300 + 3 for i in range(150)], 61),
    (16, 16, 32, 32, "f16", [1] * 200, [i * 37 % 900 + 1 for i in range(200)], 0),   # workgroups that take six tasks each
    (4, 4, 128, 32, "f16", [1] * 400, [i * 37 % 800 + 1 for i in range(400)], 0),
    (300, 1, 16, 16, "f16", [1, 2, 1], [1, 40, 30], 33),                             # more heads on one than a block has rows
    (47, 1, 32, 16, "bf16", [1] * 6, [9, 40, 1, 16, 33, 70], 900),
    (14, 2, 64, 16, "f16", [5, 0, 7, 1], [5, 3, 90, 200], 0),                        # heads that divide no block
]


@pytest.mark.parametrize("spec", BATCHES, ids=lambda s: "-".join(str(x) for x in s[:5]) + f"-{s[5][0]}")
@pytest.mark.parametrize("eight", [False, True])
def test_many_sequences(spec, eight):
    H, G, D, page, dt, new, lens, prefix = spec
    c = (Quantized if eight else Case)(H, G, D, page, dt, new, lens, prefix, seed=4)
    worst = max(check(c, *w) for w in [(0, 0), (20, 3), (100, 0)])
    log(f"[window] {spec[:5]} x {len(new)}, {'8' if eight else '16'} bits: worst {worst:.2f} of tolerance")


# heads, key/value heads, sequences, prefix: prefixes of few rows and of many, few chunks and many, own positions by
# workgroups and by waves, with and without a join of their own
BEHIND = [(8, 2, 3, 3001), (8, 2, 20, 9000), (16, 4, 40, 700), (2, 1, 500, 30000), (8, 2, 513, 9000), (8, 2, 513, 200), (64, 64, 20, 2500), (32, 8, 140, 5000)]


@pytest.mark.parametrize("shape", BEHIND, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("D,eight", [(16, False), (32, True)])
def test_behind_long_prefixes(shape, D, eight):
    H, G, B, P = shape
    c = (Quantized if eight else Case)(H, G, D, 32, "bf16" if D == 16 else "f16", [1] * B, [i * 7 % 90 + 1 for i in range(B)], P, seed=11)
    scale = D ** -0.5
    if B < 4:
        for a, b in zip(behind_a_prefix(c, scale), windowed(c, 0, 0, scale)):
            for x, y in zip(a[1:], b[1:]):
                torch.testing.assert_close(x, y, rtol=1e-12, atol=1e-12)
    out, lse = attend(c, 0, 0)
    worst = check_window(c, 0, 0, scale, out, lse, torch.full(c.q.shape, 3.0, dtype=c.dtype), behind_a_prefix(c, scale))
    log(f"[window] {shape} head_dim {D}, {'8' if eight else '16'} bits: worst {worst:.2f} of tolerance")


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("heads,kv", [(32, 8), (4, 1)])
def test_rows_that_see_nothing_behind_a_prefix(heads, kv, eight):
    """Sequences shorter than their tokens, without positions or none at all among many behind one prefix: the prefix's
    part is there for all rows, but reaches those that see something only."""
    new, lens = [2, 3, 1, 4, 1, 2] * 14, [1, 0, -1, 30, 9, 40] * 14
    c = (Quantized if eight else Case)(heads, kv, 64, 16, "bf16", new, lens, 77, seed=5, extra=3, first=1)
    check(c, 0, 0)
    out, lse = attend(c, 0, 0)
    t = c.starts[0]
    assert (out[t] == 0).all() and (lse[t] == -math.inf).all()        # place -1 of a sequence with one position
    assert (out[t + 1] != 0).any()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("many,prefix", [(10, 200), (10, 900), (90, 200), (90, 900)])
def test_values_that_are_not_finite_in_a_prefix_and_behind(many, prefix, eight):
    """NaN in the prefix reaches every row; NaN in one sequence's own positions reaches that sequence alone."""
    from paper_2609_17184_amd import serving
    c = (Quantized if eight else Case)(16, 8, 64, 16, "bf16", [1] * many, [20 + i for i in range(many)], prefix, seed=6)
    q = c.q.to(DEV)
    ref = serving.window_attention(q, c.cache, c.batch)
    vd = c.vd.view(torch.uint8) if eight else c.vd
    bad = 0x7F if eight else math.nan
    vd[c.tables[3][0], 5, 7, 9] = bad
    out = serving.window_attention(q, c.cache, c.batch)
    nan = torch.zeros(c.q.shape, dtype=torch.bool)
    nan[3, 10:12, 9] = True
    assert torch.equal(out.isnan().cpu(), nan)
    assert torch.equal(out[~nan.to(DEV)], ref[~nan.to(DEV)])
    vd[c.ptable[2], 5, 3, 9] = bad
    nan[:, 10:12, 9] = True
    assert torch.equal(serving.window_attention(q, c.cache, c.batch).isnan().cpu(), nan)
    c.batch.prefix_table[4] = c.n_pages
    assert serving.window_attention(q, c.cache, c.batch).isnan().all()


@pytest.mark.parametrize("eight", [False, True])
def test_captured_behind_a_prefix(eight):
    """The two launches of a prefix and of own positions captured and replayed while lengths change."""
    from paper_2609_17184_amd import serving
    c = (Quantized if eight else Case)(16, 8, 64, 16, "f16", [1] * 70, [60] * 70, 150, seed=7)
    q = c.q.to(DEV)
    serving.window_attention(q, c.cache, c.batch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = serving.window_attention(q, c.cache, c.batch, return_lse=True)
    for turn in range(4):
        c.batch.seq_len.copy_(torch.tensor([(i * 7 + turn * 11) % 60 + 1 for i in range(70)], dtype=torch.int32))
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, serving.window_attention(q, c.cache, c.batch, return_lse=True)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("many", [2, 80])
@pytest.mark.parametrize("dtype,eight,size", [("f16", False, 4e4), ("f16", True, 4e4), ("bf16", False, 1e10), ("bf16", True, 1e10), ("bf16", False, 1e15)])
def test_scores_too_large_for_their_differences(many, dtype, eight, size):
    """One position's key is the row's query, the others' are other sign patterns of its size: scores of size^2 * D, of which
    fp32 holds no differences as small as a softmax asks for.  All weight is that one position's."""
    from paper_2609_17184_amd import serving
    D, G, P = 64, 2, 45
    c = (Quantized if eight else Case)(4, G, D, 16, dtype, [3 if many == 2 else 1] * many, [37] * many, P, seed=8)
    g = torch.Generator().manual_seed(9)
    size = 2.0 ** math.floor(math.log2(size))
    signs = torch.randint(0, 2, c.k.shape, generator=g) * 2.0 - 1
    if eight:
        byte = torch.full(c.kb.shape, 127 + int(math.log2(size)), dtype=torch.uint8)
        c.kd.view(torch.uint8).copy_(signs.to(torch.float8_e4m3fn).view(torch.uint8))
        c.kb.view(torch.uint8).copy_(byte)
    else:
        c.kd.copy_(signs * size)
    want = torch.zeros(c.q.shape, dtype=torch.float64)
    for s in range(many):
        for i in range(c.new[s]):
            t = c.starts[s] + i
            for h in range(4):
                own = (7 * s + h) % 2
                j = (5 * s + 11 * h) % (P if not own else 34)
                page, at = (c.tables[s] if own else c.ptable)[j // 16], j % 16
                c.q[t, h] = signs[page, h // 2, at] * size
                want[t, h] = c.v[page, h // 2, at]
    out, lse = serving.window_attention(c.q.to(DEV), c.cache, c.batch, return_lse=True)
    torch.testing.assert_close(out.cpu().double(), want, rtol=2 * torch.finfo(c.dtype).eps, atol=0)
    score = size * size * D ** 0.5
    assert (lse.cpu().double() / score - 1).abs().max() < 2.0 ** -19


@pytest.mark.parametrize("new", [[3, 1], [60, 1], [1] * 130])
@pytest.mark.parametrize("byte,scale", [(63, 1e-30), (1, 1e-3), (250, 300.0)])
def test_factors_of_scores_at_fp32s_ends(new, byte, scale):
    """Key scales and a scale of the scores whose product leaves fp32, downwards or upwards (then with keys of 0): no score
    and no hidden position becomes NaN by it."""
    c = Quantized(16, 8, 32, 16, "bf16", new, [n + 40 for n in new], 21, seed=13)
    c.kb.view(torch.uint8)[c.kb.view(torch.uint8) != 255] = byte
    if byte == 250:
        c.kd.view(torch.uint8).zero_()
        c.kc.zero_()
    c.k = c.kc.nan_to_num(0.0) * 2.0 ** (byte - 127) * scale * 32 ** 0.5
    out, lse = attend(c, 30, 5, scale)
    check_window(c, 30, 5, 32 ** -0.5, out, lse, torch.full(c.q.shape, 3.0, dtype=c.dtype))


@pytest.mark.parametrize("D,dtype,eight", [(16, "bf16", False), (16, "f16", True), (128, "f16", False)])
def test_more_blocks_of_rows_than_workgroups(D, dtype, eight):
    """Prompts whose blocks of rows are more than the workgroups of a launch, which go on from one to the next: the same
    bits as from fewer of them at once."""
    from paper_2609_17184_amd import serving
    G, B, n = 64, 272, 50
    c = (Quantized if eight else Case)(G, G, D, 16, dtype, [n] * B, [n + i % 12 for i in range(B)], 0, seed=14)
    q = c.q.to(DEV)
    out, lse = serving.window_attention(q, c.cache, c.batch, 40, 3, return_lse=True)
    starts = torch.arange(69, dtype=torch.int32, device=DEV) * n
    for b in range(0, B, 68):
        part = serving.Batch(c.batch.seq_len[b:b + 68].contiguous(), c.batch.table[b:b + 68], starts)
        o, l = serving.window_attention(q[b * n:(b + 68) * n], c.cache, part, 40, 3, return_lse=True)
        assert torch.equal(o, out[b * n:(b + 68) * n]) and torch.equal(l, lse[b * n:(b + 68) * n])
    assert out.isfinite().all() and lse.isfinite().all()
