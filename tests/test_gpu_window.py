"""Attention under a window over 16-bit and 8-bit pages against a plain 64-bit implementation."""
import math
import threading

import pytest
import torch

from gpu_common import log
from quantized_common import Quantized, check_window
from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# heads, key/value heads, head_dim, page, type, tokens and own positions per sequence, prefix
BATCHES = [
    (16, 16, 128, 16, "f16", [1], [1], 0),
    (16, 16, 128, 16, "bf16", [1, 1, 1], [1, 40, 129], 77),
    (5, 1, 128, 32, "f16", [1] * 7, [3, 300, 16, 17, 31, 32, 33], 1),
    (28, 4, 128, 64, "bf16", [4, 1, 9, 2], [4, 64, 70, 200], 515),
    (6, 6, 96, 48, "f16", [3, 0, 2], [50, 0, 2], 100),
    (6, 3, 96, 16, "bf16", [40, 1], [140, 90], 21),
    (8, 2, 64, 128, "bf16", [1, 17], [129, 17], 64),
    (4, 2, 32, 16, "f16", [2, 2, 5], [500, 2, 37], 31),
    (3, 3, 16, 16, "bf16", [1, 2], [5, 65], 33),
    (32, 8, 64, 16, "f16", [40, 3], [40, 200], 0),
    (2, 1, 128, 1008, "f16", [1, 1], [1500, 20], 2000),
    (2, 1, 32, 16, "f16", [i % 3 for i in range(200)], [i * 7 % 50 + 2 for i in range(200)], 33),
    (4, 2, 128, 32, "bf16", [150, 70], [400, 70], 40),
]
WINDOWS = [(0, 0), (1, 0), (33, 4), (100, 50), (16, 16), (10000, 3)]


def make(spec, eight, **kw):
    H, G, D, page, dt, new, lens, prefix = spec
    return (Quantized if eight else Case)(H, G, D, page, dt, new, lens, prefix, **kw)


def attend(c, window, sinks, scale=None, before=None, **kw):
    from paper_2609_17184_amd import serving
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    lse = serving.window_attention(c.q.to(DEV), c.cache, c.batch, window, sinks, scale, out=out, return_lse=True, **kw)[1]
    return out, lse


def check(c, window, sinks, scale=None):
    out, lse = attend(c, window, sinks, scale)
    return check_window(c, window, sinks, c.D ** -0.5 if scale is None else scale, out, lse, torch.full(c.q.shape, 3.0, dtype=c.dtype))


@pytest.mark.parametrize("spec", BATCHES, ids=lambda s: "-".join(str(x) for x in s[:5]))
@pytest.mark.parametrize("eight,heads_first", [(False, True), (False, False), (True, True), (True, False)])
def test_windows(spec, eight, heads_first):
    """Every batch under every window, with NaN in all places of the cache that hold no position."""
    c = make(spec, eight, seed=4, heads_first=heads_first)
    worst = max(check(c, *w) for w in WINDOWS)
    log(f"[window] {spec[:5]} {'8' if eight else '16'} bits: worst {worst:.2f} of tolerance")
    if c.new == [1] * len(c.new):
        from paper_2609_17184_amd import serving
        single = serving.Batch(c.batch.seq_len, c.batch.table, None, c.prefix, c.batch.prefix_table)
        ref = serving.window_attention(c.q.to(DEV), c.cache, c.batch, 33, 4)
        assert torch.equal(serving.window_attention(c.q.to(DEV), c.cache, single, 33, 4), ref)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("D", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("tokens", [4, 5, 8, 9, 16, 17, 33, 64, 65, 100, 129])
def test_row_counts(tokens, D, eight):
    """Rows of a head's queries on either side of every block size, one token per sequence and all in one."""
    for new, lens in (([1] * tokens, [1 + 7 * i for i in range(tokens)]), ([tokens], [tokens + 150])):
        c = make((8, 2, D, 16, "f16" if tokens % 2 else "bf16", new, lens, 45), eight, seed=tokens)
        check(c, 70, 5)
        check(c, 0, 0)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (5000, 7), (700, 0)])
@pytest.mark.parametrize("new", [[1, 3], [1, 40], [2, 200]])
def test_long_sequences(new, window, sinks, eight):
    """Positions in many chunks, in tables with room for more."""
    c = make((4, 2, 64, 64, "bf16", new, [9000, 20011], 500), eight, seed=13, width=600)
    check(c, window, sinks)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("q_start", [True, False])
def test_padding_rows(q_start, eight):
    """Tokens of no sequence, sequences with seq_len < 0 or shorter than their tokens, before and behind the batch."""
    cls = Quantized if eight else Case
    if q_start:
        c = cls(4, 2, 32, 16, "f16", [2, 3, 4, 1], [-1, 2, 30, 0], 20, extra=5, first=2)
    else:
        c = cls(4, 2, 32, 16, "f16", [1, 1, 1, 1], [-1, 2, 30, 0], 20, extra=5, q_start=False)
    for w in WINDOWS:
        check(c, *w)


@pytest.mark.parametrize("eight", [False, True])
def test_rows_that_see_nothing(eight):
    c = make((4, 4, 64, 16, "f16", [2, 1, 3], [0, 5, 1], 0), eight, seed=2)
    out, lse = attend(c, 3, 1)
    check_window(c, 3, 1, 0.125, out, lse, out.cpu())
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_steep_scores(dtype, eight):
    """Scores that spread over hundreds, so that references rise late and most weights vanish."""
    c = make((4, 2, 64, 16, dtype, [1, 3, 40], [100, 900, 800], 70), eight, seed=6)
    c.q *= 20
    check(c, 500, 20, 0.5)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scales_far_apart(dtype):
    """Blocks whose scales differ by up to 2^20, in both orders: no weight of theirs leaves its type."""
    c = Quantized(4, 2, 64, 16, dtype, [1, 20], [800, 700], 70, seed=16, spread=3.0)
    check(c, 0, 0, 0.01)
    check(c, 300, 40, 0.01)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("new", [[6, 2], [70, 40]])
def test_hidden_positions_have_no_influence(new, eight):
    """Keys and values before the window and behind a token, whatever they hold: NaN, infinities, NaN scales, no page."""
    from paper_2609_17184_amd import serving
    lens = [300, 290]
    c = make((8, 2, 64, 16, "f16", new, lens, 40), eight, seed=9)
    q = c.q.to(DEV)
    ref, rlse = serving.window_attention(q, c.cache, c.batch, 64, 4, return_lse=True)
    see = []
    for b in range(2):
        # tokens at even distance see neither what is before position 120 of the sequence nor the last 3 positions
        n = new[b]
        see += [c.starts[b] + i for i in range(n) if c.prefix + lens[b] - n + i - 64 + 1 >= 40 + 120 and i < n - 3]
        for t in ([c.kd, c.vd] if not eight else [c.kd.view(torch.uint8), c.vd.view(torch.uint8)]):
            for place in list(range(0, 120)) + list(range(lens[b] - 3, lens[b])):
                if c.prefix + place < 4:
                    continue
                t[c.tables[b][place // 16], :, place % 16] = 0x7F if eight else (math.nan, math.inf, -math.inf)[place % 3]
    if eight:
        for b in range(2):
            for t in (c.kb, c.vb):
                for place in range(16, 96, 16):
                    t.view(torch.uint8)[c.tables[b][place // 16]] = 255
        c.batch.table[0, 1] = -1
    c.batch.table[1, 2] = c.n_pages
    c.batch.table[1, 3] = -1
    out, lse = serving.window_attention(q, c.cache, c.batch, 64, 4, return_lse=True)
    assert see
    err = (out[see].double() - ref[see].double()).abs().max().item()
    assert err <= torch.finfo(c.dtype).eps / 2 * ref[see].abs().max().item() and torch.equal(lse[see], rlse[see])
    last = [c.starts[b] + new[b] - 1 for b in range(2)]
    assert out[last].isnan().all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 20)])
def test_pages_outside_the_cache_make_nan(window, sinks, eight):
    """A visible page that is none of the cache's, or that the table does not hold: NaN for the rows that see it."""
    from paper_2609_17184_amd import serving
    c = make((4, 2, 64, 16, "f16", [1, 1, 1], [40, 40, 10], 50), eight, seed=1)
    q = c.q.to(DEV)

    def run():
        return serving.window_attention(q, c.cache, c.batch, window, sinks)
    ref = run()
    c.batch.table[0, 1] = c.n_pages
    c.batch.table[1, 2] = -1
    out = run()
    assert out[:2].isnan().all() and torch.equal(out[2], ref[2])
    c.batch.seq_len[2] = 16 * c.batch.table.shape[1] + 1
    assert run()[2].isnan().all()
    c.batch.seq_len[2] = 10
    c.batch.prefix_table[1] = -5             # positions 16 .. 31, first ones of which are sinks
    assert run().isnan().all()


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("new", [[1, 1], [40, 40]])
def test_nan_scales(which, new):
    """A visible block with a NaN scale makes the rows that see it NaN, in its head only."""
    from paper_2609_17184_amd import serving
    c = Quantized(4, 2, 64, 16, "bf16", new, [100, 100], 0, seed=3)
    q = c.q.to(DEV)
    ref = serving.window_attention(q, c.cache, c.batch, 30, 0)
    (c.kb if which == "k" else c.vb).view(torch.uint8)[c.tables[0][5], 1, 0] = 255      # positions 80 .. 95
    out = serving.window_attention(q, c.cache, c.batch, 30, 0)
    nan = torch.zeros(c.q.shape[:2], dtype=torch.bool)
    for i in range(new[0]):
        p = 100 - new[0] + i
        nan[i, 2:] = p >= 80 and p - 29 <= 95
    assert torch.equal(out.isnan().all(-1).cpu(), nan) and torch.equal(out.isnan().any(-1).cpu(), nan)
    keep = ~nan.to(DEV)
    err = (out[keep].double() - ref[keep].double()).abs().max().item()
    assert err <= torch.finfo(c.dtype).eps / 2 * ref.abs().max().item()


def test_nan_codes_reach_the_rows_that_see_them():
    from paper_2609_17184_amd import serving
    for new in ([1], [50]):
        c = Quantized(4, 2, 96, 16, "f16", new, [100], 0, seed=5)
        q = c.q.to(DEV)
        c.vd.view(torch.uint8)[c.tables[0][60 // 16], 0, 60 % 16, 7] = 0xFF
        out = serving.window_attention(q, c.cache, c.batch, 30, 2)
        nan = torch.zeros(c.q.shape, dtype=torch.bool)
        for i in range(new[0]):
            p = 100 - new[0] + i
            nan[i, :2, 7] = p >= 60 and p - 60 < 30
        assert torch.equal(out.isnan().cpu(), nan)


@pytest.mark.parametrize("eight", [False, True])
def test_a_row_stands_alone(eight):
    """The same sequence in other batches, other places and beside other lengths gives the same bits where the work is
    split alike."""
    from paper_2609_17184_amd import serving
    c = make((8, 2, 128, 16, "bf16", [1, 1, 1, 1], [700, 3, 450, 700], 0), eight, seed=17)
    c.q[3] = c.q[0]
    q = c.q.to(DEV)
    c.batch.table[3] = c.batch.table[0]
    out = serving.window_attention(q, c.cache, c.batch, 100, 3)
    assert torch.equal(out[0], out[3])
    c.batch.seq_len[1] = 40
    q[1:3].normal_()
    assert torch.equal(serving.window_attention(q, c.cache, c.batch, 100, 3)[[0, 3]], out[[0, 3]])


@pytest.mark.parametrize("eight", [False, True])
def test_large_offsets(eight):
    """Pages behind 2^31 elements of the cache."""
    from paper_2609_17184_amd import serving
    G, D, page = 8, 128, 16
    n_pages = 2 ** 31 // (G * D * page) + 40
    small = make((8, G, D, page, "f16", [1, 2], [33, 50], 64), eight, seed=11)
    ref = serving.window_attention(small.q.to(DEV), small.cache, small.batch, 40, 5)
    k, v = (torch.empty((n_pages, G, page, D), dtype=torch.uint8 if eight else torch.float16, device=DEV) for _ in range(2))
    shift = n_pages - small.n_pages
    k[shift:], v[shift:] = (t.view(torch.uint8) if eight else t for t in (small.kd, small.vd))
    if eight:
        ks, vs = (torch.zeros((n_pages, G, 1), dtype=torch.uint8, device=DEV) for _ in range(2))
        ks[shift:], vs[shift:] = small.kb.view(torch.uint8), small.vb.view(torch.uint8)
        cache = serving.QuantizedCache(k.view(small.kd.dtype), v.view(small.kd.dtype), ks.view(small.kb.dtype), vs.view(small.kb.dtype))
    else:
        cache = serving.PagedCache(k, v)
    batch = serving.Batch(small.batch.seq_len, small.batch.table + shift, small.batch.q_start, 64, small.batch.prefix_table + shift)
    assert torch.equal(serving.window_attention(small.q.to(DEV), cache, batch, 40, 5), ref)
    new = small.kn.to(DEV), small.vn.to(DEV)
    serving.rope_append(small.q.to(DEV), *new, cache, batch)
    serving.rope_append(small.q.to(DEV), *new, small.cache, small.batch)
    if eight:
        assert torch.equal(k[shift:], small.kd.view(torch.uint8)) and torch.equal(ks[shift:], small.kb.view(torch.uint8))


def test_strided_queries_and_outputs():
    """Queries that are a view of a fused projection, an output that is a view, two types over one 8-bit cache."""
    from paper_2609_17184_amd import serving
    c = Quantized(6, 2, 64, 16, "bf16", [1, 5, 30], [40, 70, 30], 20, seed=8)
    fused = torch.randn((36, 6 * 64 + 256), device=DEV).to(torch.bfloat16)
    q = fused[:, 128:128 + 384].view(36, 6, 64)
    q.copy_(c.q)
    room = torch.full((36, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    out = room[:, 1:7, 32:96]
    lse = serving.window_attention(q, c.cache, c.batch, 25, 2, out=out, return_lse=True)[1]
    check_window(c, 25, 2, 0.125, out, lse, out.cpu())
    room[:, 1:7, 32:96] = 3.0
    assert (room == 3).all()
    c.q = c.q.half()
    c.dtype = torch.float16
    check(c, 25, 2)


@pytest.mark.parametrize("eight", [False, True])
def test_streams_and_captured_steps(eight):
    """Captured once and replayed while lengths and inputs change, on a side stream, against the eager calls; two graphs
    that run one after the other."""
    from paper_2609_17184_amd import serving
    cases = [make((8, 2, 64, 16, "bf16", [1] * 3, [5, 600, 17], 90), eight, seed=s, width=60) for s in (20, 21)]
    freq = serving.rope_frequencies(64)
    stream = torch.cuda.Stream()
    work = []
    for c in cases:
        q, k, v = c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV)

        def step(c=c, q=q, k=k, v=v):
            r = serving.rope_append(q, k, v, c.cache, c.batch, freq)
            return serving.window_attention(r, c.cache, c.batch, 70, 4, return_lse=True)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = step()
        work.append((c, q, k, v, step, graph, outs))
    for turn in range(4):
        for c, q, k, v, step, graph, outs in work:
            c.batch.seq_len.copy_(torch.tensor([5, 600 - 100 * turn, 0 if turn == 1 else 17], dtype=torch.int32))
            q.normal_()
            k.normal_()
            v.normal_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for w in work:
                w[5].replay()
        torch.cuda.synchronize()
        for c, q, k, v, step, graph, outs in work:
            live = c.batch.seq_len > 0
            for a, b in zip(outs, step()):
                assert torch.equal(a[live], b[live])


def test_two_threads_share_a_cache():
    from paper_2609_17184_amd import serving
    c = Quantized(8, 2, 64, 16, "f16", [2, 1, 3], [300, 600, 17], 90, seed=33, extra=40)
    q = c.q.to(DEV)
    ref = {rows: serving.window_attention(q[:rows], c.cache, c.batch, 100, 3)[:6] for rows in (6, 46)}
    torch.cuda.synchronize()
    wrong = []

    def work(rows):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(60):
                if not torch.equal(serving.window_attention(q[:rows], c.cache, c.batch, 100, 3)[:6], ref[rows]):
                    wrong.append(rows)
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(rows,)) for rows in (6, 46)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_empty_batches_and_refusals():
    from paper_2609_17184_amd import serving
    c = Quantized(4, 2, 64, 16, "f16", [1, 1], [40, 17], 50, seed=1)
    none = torch.empty((0, 4, 64), dtype=c.dtype, device=DEV)
    out, lse = serving.window_attention(none, c.cache, c.batch, 5, return_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    nobody = serving.Batch(empty, torch.empty((0, 4), dtype=torch.int32, device=DEV), None, 50, c.batch.prefix_table)
    kept = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    serving.window_attention(c.q.to(DEV), c.cache, nobody, 5, out=kept)
    assert (kept == 3).all()
    q = c.q.to(DEV)
    for kw in (dict(window=-1), dict(sinks=-1)):
        with pytest.raises(ValueError):
            serving.window_attention(q, c.cache, c.batch, **kw)
    with pytest.raises(TypeError):
        serving.window_attention(q, c.cache, c.batch, 1.5)
    with pytest.raises(ValueError):
        serving.window_attention(q.float(), c.cache, c.batch, 5)
    with pytest.raises(ValueError):
        serving.prefix_attention(q, c.cache, c.batch)
    for table in (None, c.batch.prefix_table[:3]):
        with pytest.raises(ValueError):
            serving.window_attention(q, c.cache, serving.Batch(c.batch.seq_len, c.batch.table, None, 50, table))
    # a window beyond every number of positions
    assert torch.equal(serving.window_attention(q, c.cache, c.batch, 1 << 40, 1 << 50), serving.window_attention(q, c.cache, c.batch))
