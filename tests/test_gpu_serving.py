"""The serving operators on the GPU against plain 64-bit implementations: the append to the paged cache with norm and
rotation, and attention over a shared prefix and each sequence's own positions."""
import math

import pytest
import torch

from gpu_common import log
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
    (8, 2, 64, 128, "bf16", [1, 17], [129, 17], 64),
    (4, 2, 32, 16, "f16", [2, 2, 5], [500, 2, 37], 31),
    (3, 3, 16, 16, "bf16", [1, 2], [5, 65], 33),
    (32, 8, 64, 16, "f16", [40, 3], [40, 200], 0),      # more rows of a sequence than a block holds
    (2, 1, 128, 1008, "f16", [1, 1], [1500, 20], 2000),  # pages that divide nothing
    # more sequences than a wave looks at together, with a few tokens or many rows each
    (2, 1, 32, 16, "f16", [i % 3 for i in range(600)], [i * 7 % 50 + 2 for i in range(600)], 33),
    (32, 1, 16, 16, "bf16", [2] * 300, [i * 11 % 60 + 2 for i in range(300)], 20),
]


def half(dtype):
    return torch.finfo(dtype).eps / 2


def make(spec, **kw):
    H, G, D, page, dt, new, lens, prefix = spec
    return Case(H, G, D, page, dt, new, lens, prefix, **kw)


def check_append(c, rot, norms, eps, out, before):
    """Queries and the whole cache after an append: rounded once from fp32, whose own error is a few 2^-24 per
    operation (about 12 for the norm, 4 for the rotation, 2^-23 for the angle's sine and cosine): 2^-19 of the values
    that enter.  fp16's subnormals are spaced 2^-24."""
    freq = None if not rot else 1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    qn, kn = norms
    keys, values = c.k.clone().double(), c.v.clone().double()
    slack = torch.zeros_like(keys)
    got = out.cpu().double()
    done = torch.zeros(len(c.q), dtype=torch.bool)
    worst = 0.0
    for t, b, place in c.tokens():
        if place < 0:
            continue
        done[t] = True
        ref, mix = c.rotated(c.q[t], qn, eps, freq, c.prefix + place)
        tol = ref.abs() * half(c.dtype) + mix * 2.0 ** -19 + 2.0 ** -25
        err = (got[t] - ref).abs()
        assert (err <= tol).all(), (t, b, place, (err - tol).max())
        worst = max(worst, (err / tol).max().item())
        page, at = c.tables[b][place // c.page], place % c.page
        keys[page, :, at], mix = c.rotated(c.kn[t], kn, eps, freq, c.prefix + place)
        slack[page, :, at] = keys[page, :, at].abs() * half(c.dtype) + mix * 2.0 ** -19 + 2.0 ** -25
        values[page, :, at] = c.vn[t].double()
    kd, vd = c.kd.cpu().double(), c.vd.cpu().double()
    assert torch.equal(vd.nan_to_num(9e9), values.nan_to_num(9e9))
    assert torch.equal(kd.isnan(), keys.isnan())
    assert ((kd - keys).abs().nan_to_num(0) <= slack).all()
    assert torch.equal(out.cpu()[~done], before[~done]), "rows of padding stay as they were"
    return worst


def check_attention(c, scale, out, lse, before):
    """A weight is rounded to 16 bits (half a step), the output once more; the score's fp32 sum of D products is off by
    at most (D + 8) 2^-24 of the sum of their magnitudes, which moves a weight by as much; sums over n positions add
    n 2^-24, and weights below 2^-32 of the largest vanish."""
    got, glse = out.cpu().double(), lse.cpu().double()
    seen = torch.zeros(len(c.q), dtype=torch.bool)
    worst = 0.0
    for t, ref, rlse, mean, big in c.attention(scale):
        seen[t] = True
        n = c.prefix + max(c.lens) + 16
        ds = ((c.D + 8) * 2.0 ** -24 * big + n * 2.0 ** -24)[:, None]
        tol = mean * (half(c.dtype) + 2 * ds) + ref.abs() * half(c.dtype) + n * 2.0 ** -32 * 4 + 2.0 ** -25
        err = (got[t] - ref).abs()
        assert (err <= tol).all(), (t, (err - tol).max(), err.max())
        worst = max(worst, (err / tol).max().item())
        inf = rlse == -math.inf
        assert torch.equal(glse[t] == -math.inf, inf)
        lerr = (glse[t] - rlse).abs()[~inf]
        assert (lerr <= (2 * ds[:, 0] + rlse.abs() * 2.0 ** -22 + 2.0 ** -20)[~inf]).all(), (t, lerr.max())
    assert torch.equal(out.cpu()[~seen], before[~seen]), "rows of padding stay as they were"
    return worst


@pytest.mark.parametrize("spec", BATCHES, ids=lambda s: "-".join(str(x) for x in s[:5]))
@pytest.mark.parametrize("rot,norm", [("all", False), ("half", True), ("none", True)])
def test_append(spec, rot, norm):
    from paper_2609_17184_amd import serving
    c = make(spec, seed=3)
    r = {"all": c.D, "half": c.D // 2 // 16 * 16, "none": 0}[rot]
    g = torch.Generator().manual_seed(5)
    qn, kn = ((1 + 0.3 * torch.randn(c.D, generator=g)) if norm else None for _ in range(2))
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    before = out.cpu()
    freq = serving.rope_frequencies(r) if r else None
    got = serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, freq,
                              q_norm=None if qn is None else qn.to(DEV), k_norm=None if kn is None else kn.to(DEV),
                              eps=1e-5, out=out)
    assert got is out
    log(f"[append] {spec[:5]} rot {r} norm {norm}: worst {check_append(c, r, (qn, kn), 1e-5, out, before):.2f} of tolerance")


def test_append_far_positions_views_and_in_place():
    """Positions near 2^27, queries, keys and values as views of one fused row, queries rotated in place, positions
    outermost in the pages."""
    from paper_2609_17184_amd import serving
    c = Case(6, 2, 64, 16, "bf16", [1, 2], [4, 20], 0, heads_first=False, seed=8)
    c.prefix = 134217001
    c.batch._c.prefix_len = c.prefix
    fused = torch.cat([c.q.flatten(1), c.kn.flatten(1), c.vn.flatten(1)], 1).to(DEV)
    q, k, v = fused[:, :384].view(3, 6, 64), fused[:, 384:512].view(3, 2, 64), fused[:, 512:].view(3, 2, 64)
    serving.rope_append(q, k, v, c.cache, c.batch, serving.rope_frequencies(64), out=q)
    check_append(c, 64, (None, None), 0.0, q, q.cpu())
    assert torch.equal(fused[:, 384:].cpu(), torch.cat([c.kn.flatten(1), c.vn.flatten(1)], 1))


@pytest.mark.parametrize("q_start", [True, False])
def test_padding_rows(q_start):
    """Tokens of no sequence, sequences with seq_len < 0 or shorter than their tokens, before and behind the batch."""
    from paper_2609_17184_amd import serving
    if q_start:
        c = Case(4, 2, 32, 16, "f16", [2, 3, 4, 1], [-1, 2, 30, 0], 20, extra=5, first=2)
    else:
        c = Case(4, 2, 32, 16, "f16", [1, 1, 1, 1], [-1, 2, 30, 0], 20, extra=5, q_start=False)
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    before, q = out.cpu(), c.q.to(DEV)
    lse = serving.prefix_attention(q, c.cache, c.batch, out=out, return_lse=True)[1]
    check_attention(c, 32 ** -0.5, out, lse, before)
    out.fill_(3.0)
    serving.rope_append(q, c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, serving.rope_frequencies(32), out=out)
    check_append(c, 32, (None, None), 0.0, out, before)


@pytest.mark.parametrize("spec", BATCHES, ids=lambda s: "-".join(str(x) for x in s[:5]))
@pytest.mark.parametrize("heads_first", [True, False])
def test_attention(spec, heads_first):
    """Every batch with NaN in all places of the cache that hold no position."""
    from paper_2609_17184_amd import serving
    c = make(spec, seed=4, heads_first=heads_first)
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, out=out, return_lse=True)[1]
    w = check_attention(c, c.D ** -0.5, out, lse, torch.full(c.q.shape, 3.0, dtype=c.dtype))
    log(f"[attention] {spec}: worst {w:.2f} of tolerance")
    if c.new == [1] * len(c.new):
        single = serving.Batch(c.batch.seq_len, c.batch.table, None, c.prefix, c.batch.prefix_table)
        assert torch.equal(serving.prefix_attention(c.q.to(DEV), c.cache, single), out)


def test_attention_rows_that_see_nothing():
    from paper_2609_17184_amd import serving
    c = Case(4, 4, 64, 16, "f16", [2, 1, 3], [0, 5, 1], 0, seed=2)
    out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, return_lse=True)
    check_attention(c, 0.125, out, lse, out.cpu())
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()


def test_attention_steep_scores():
    """Scores that spread over hundreds, so that references rise late and most weights vanish."""
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 64, 16, "bf16", [1, 3], [100, 90], 700, seed=6)
    c.q *= 20
    out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, scale=0.5, return_lse=True)
    check_attention(c, 0.5, out, lse, out.cpu())


def test_attention_small_weights_beside_a_large_one():
    """One position far above many equal ones whose sum matters: fp16 weights keep the small ones."""
    from paper_2609_17184_amd import serving
    c = Case(2, 2, 32, 16, "f16", [1], [1], 6000, seed=7)
    c.q[:] = 1.0
    for t in (c.k, c.v):
        c.put(t, c.ptable, 0, torch.zeros((6000, 2, 32), dtype=c.dtype))
    c.put(c.v, c.ptable, 0, torch.ones((6000, 2, 32), dtype=c.dtype))
    top = torch.full((1, 2, 32), 20 * math.log(2) / 32).to(c.dtype)       # 2^20 times the weight of the others
    c.put(c.k, c.ptable, 3000, top)
    c.put(c.v, c.ptable, 3000, torch.zeros((1, 2, 32), dtype=c.dtype))
    c.put(c.k, c.tables[0], 0, torch.zeros((1, 2, 32), dtype=c.dtype))
    c.kd.copy_(c.k)
    c.vd.copy_(c.v)
    out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, scale=1.0, return_lse=True)
    _, ref, _, _, _ = next(iter(c.attention(1.0)))
    rel = ((out[0].cpu().double() - ref) / ref).abs().max().item()
    # the sum of 6000 equal fp16 weights: off by half a step each, the same way
    assert rel <= 2 * half(torch.float16) + 6000 * 2.0 ** -24, rel


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_attention_hidden_values_have_no_influence(bad):
    """The keys and values of a sequence's last tokens are not finite: earlier tokens do not see them."""
    from paper_2609_17184_amd import serving
    c = Case(8, 2, 64, 16, "f16", [6, 2], [45, 2], 40, seed=9)
    q = c.q.to(DEV)
    ref, rlse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    for t in (c.kd, c.vd):
        for place in (42, 43, 44):
            t[c.tables[0][place // 16], :, place % 16] = bad
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    see = [0, 1, 2, 6, 7]                     # tokens at 39, 40, 41 and the second sequence's
    err = (out[see].double() - ref[see].double()).abs().max().item()
    assert err <= half(c.dtype) * ref[see].abs().max().item() and torch.equal(lse[see], rlse[see])
    if bad == float("nan"):
        assert out[3:6].isnan().all()


@pytest.mark.parametrize("tokens", [4, 5, 8, 9, 16, 17, 33, 64, 65, 100])
@pytest.mark.parametrize("D", [16, 32, 64, 96, 128])
def test_attention_row_counts(tokens, D):
    """Rows of a head's queries on either side of every block size, one token per sequence and all in one."""
    from paper_2609_17184_amd import serving
    for new, lens in (([1] * tokens, [1 + 7 * i for i in range(tokens)]), ([tokens], [tokens + 150])):
        c = Case(8, 2, D, 16, "f16" if tokens % 2 else "bf16", new, lens, 333, seed=tokens)
        out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, return_lse=True)
        check_attention(c, D ** -0.5, out, lse, out.cpu())


@pytest.mark.parametrize("width,new", [(None, [1, 3]), (20000, [1, 3]), (20000, [1, 40])])
def test_attention_long_sequences(width, new):
    """Own positions in many chunks, in tables with room for more: chunks of every size, a short one behind them."""
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 64, 64, "bf16", new, [9000, 20011], 500, seed=13, width=width)
    out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, return_lse=True)
    check_attention(c, 0.125, out, lse, out.cpu())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_attention_long_prompt_hides_its_end(bad):
    """Blocks of many rows of one sequence, in which some rows see what others must not."""
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 128, 32, "bf16", [70, 40], [200, 40], 100, seed=12)
    q = c.q.to(DEV)
    ref, rlse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    check_attention(c, 128 ** -0.5, ref, rlse, ref.cpu())
    for t in (c.kd, c.vd):
        for b, first, n in ((0, 150, 200), (1, 20, 40)):
            for place in range(first, n):
                t[c.tables[b][place // 32], :, place % 32] = bad
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    see = list(range(20)) + list(range(70, 90))
    err = (out[see].double() - ref[see].double()).abs().max().item()
    assert err <= half(c.dtype) * ref[see].abs().max().item() and torch.equal(lse[see], rlse[see])


def test_attention_pages_outside_the_cache_make_nan():
    """A visible page that is none of the cache's, or that the table does not hold: NaN for the rows that see it."""
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 64, 16, "f16", [1, 1, 1], [40, 40, 10], 50, seed=1)
    q = c.q.to(DEV)
    ref = serving.prefix_attention(q, c.cache, c.batch)
    c.batch.table[0, 1] = c.n_pages
    c.batch.table[1, 2] = -1
    out = serving.prefix_attention(q, c.cache, c.batch)
    assert out[:2].isnan().all() and torch.equal(out[2], ref[2])
    c.batch.seq_len[2] = 16 * c.batch.table.shape[1] + 1
    assert serving.prefix_attention(q, c.cache, c.batch)[2].isnan().all()
    c.batch.seq_len[2] = 10
    c.batch.prefix_table[3] = -5
    assert serving.prefix_attention(q, c.cache, c.batch).isnan().all()


def test_append_pages_outside_the_cache_are_left_out():
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 64, 16, "f16", [1, 1, 1], [40, 17, 10], 0, seed=1)
    c.batch.table[0, 2] = c.n_pages
    c.batch.table[1, 1] = -1
    q = serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, serving.rope_frequencies(64))
    changed = (c.kd.cpu().nan_to_num(7) != c.k.nan_to_num(7)).any(-1).any(1).nonzero().tolist()
    assert changed == [[c.tables[2][0], 9]] and not q.isnan().any()


def test_empty_batches_and_short_prefix_tables():
    """No tokens, or no sequences: nothing happens.  A prefix table shorter than the prefix is refused."""
    from paper_2609_17184_amd import serving
    c = Case(4, 2, 64, 16, "f16", [1, 1], [40, 17], 50, seed=1)
    before = c.kd.clone()
    none = torch.empty((0, 4, 64), dtype=c.dtype, device=DEV)
    kv = torch.empty((0, 2, 64), dtype=c.dtype, device=DEV)
    assert serving.rope_append(none, kv, kv, c.cache, c.batch).shape == (0, 4, 64)
    out, lse = serving.prefix_attention(none, c.cache, c.batch, return_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    nobody = serving.Batch(empty, torch.empty((0, 4), dtype=torch.int32, device=DEV), None, 50, c.batch.prefix_table)
    kept = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, nobody, out=kept)
    serving.prefix_attention(c.q.to(DEV), c.cache, nobody, out=kept)
    assert (kept == 3).all() and torch.equal(c.kd.nan_to_num(7), before.nan_to_num(7))
    assert [len(x) for x in serving.sample(torch.empty((0, 100), device=DEV), torch.empty(0, dtype=torch.float64, device=DEV))] == [0] * 3
    for table in (None, c.batch.prefix_table[:3]):
        with pytest.raises(ValueError):
            serving.prefix_attention(c.q.to(DEV), c.cache, serving.Batch(c.batch.seq_len, c.batch.table, None, 50, table))


def test_attention_large_offsets():
    """Pages behind 2^31 elements of the cache."""
    from paper_2609_17184_amd import serving
    G, D, page = 8, 128, 16
    n_pages = 2 ** 31 // (G * D * page) + 40
    k = torch.empty((n_pages, G, page, D), dtype=torch.float16, device=DEV)
    v = torch.empty_like(k)
    small = Case(8, G, D, page, "f16", [1, 2], [33, 50], 64, seed=11)
    ref = serving.prefix_attention(small.q.to(DEV), small.cache, small.batch)
    shift = n_pages - small.n_pages
    k[shift:], v[shift:] = small.kd, small.vd
    batch = serving.Batch(small.batch.seq_len, small.batch.table + shift, small.batch.q_start, 64,
                          small.batch.prefix_table + shift)
    cache = serving.PagedCache(k, v)
    assert torch.equal(serving.prefix_attention(small.q.to(DEV), cache, batch), ref)
    serving.rope_append(small.q.to(DEV), small.kn.to(DEV), small.vn.to(DEV), cache, batch)
    serving.rope_append(small.q.to(DEV), small.kn.to(DEV), small.vn.to(DEV), small.cache, small.batch)
    assert torch.equal(k[shift:].nan_to_num(7), small.kd.nan_to_num(7))


def test_other_streams_and_captured_steps():
    """A step captured once and replayed while lengths, tables and inputs change, on a side stream, against the eager
    calls; two captured steps that run one after the other."""
    from paper_2609_17184_amd import serving
    cases = [Case(8, 2, 64, 16, "bf16", [1] * 3, [5, 60, 17], 90, seed=s, width=8) for s in (20, 21)]
    freq = serving.rope_frequencies(64)
    stream = torch.cuda.Stream()
    work = []
    for c in cases:
        q, k, v = c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV)

        def step(c=c, q=q, k=k, v=v):
            r = serving.rope_append(q, k, v, c.cache, c.batch, freq)
            return serving.prefix_attention(r, c.cache, c.batch, return_lse=True)
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
            c.batch.seq_len.copy_(torch.tensor([6 + turn, 61 + turn, 0 if turn == 1 else 18], dtype=torch.int32))
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
