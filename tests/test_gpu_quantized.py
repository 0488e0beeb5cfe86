"""The append to 8-bit pages against a plain 64-bit implementation."""
import math

import pytest
import torch

from gpu_common import log
from quantized_common import BLOCK, LEAST, Quantized, block_append, e4m3, exponent, stored

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# heads, key/value heads, head_dim, page, type, tokens and own positions per sequence, prefix
BATCHES = [
    (16, 16, 128, 16, "f16", [1], [1], 0),
    (16, 16, 128, 16, "bf16", [1, 1, 1], [1, 40, 129], 77),
    (5, 1, 128, 32, "f16", [1] * 7, [3, 300, 16, 17, 31, 32, 33], 1),
    (28, 4, 128, 64, "bf16", [4, 1, 9, 2], [4, 64, 70, 200], 515),
    (6, 6, 96, 48, "f16", [3, 0, 2, 40], [50, 0, 2, 47], 100),
    (8, 2, 64, 128, "bf16", [1, 17], [129, 17], 64),
    (4, 2, 32, 16, "f16", [2, 2, 5], [500, 2, 37], 31),
    (3, 3, 16, 16, "bf16", [1, 2, 33], [5, 65, 40], 33),
    (32, 8, 64, 16, "f16", [40, 3], [40, 200], 0),
    (55, 55, 96, 1008, "f16", [130, 20], [1100, 20], 0),
    (2, 1, 32, 16, "f16", [i % 3 for i in range(600)], [i * 7 % 50 + 2 for i in range(600)], 33),
]


def make(spec, **kw):
    H, G, D, page, dt, new, lens, prefix = spec
    return Quantized(H, G, D, page, dt, new, lens, prefix, **kw)


def check_append(c, rot, norms, eps, out, before, old):
    """Queries as in the 16-bit append: fp32's error is at most 2^-19 of what enters, and one rounding.  Values are not
    computed with, so their codes and scales are the definition's, bit for bit.  A key's code is off by half a step of
    e4m3 (2^-4 of itself, or half of the subnormals' 2^-9, times the scale) and fp32's error; its block's scale is that of
    the largest magnitude, which fp32's error may move across a border.  Everything else stays."""
    freq = None if not rot else 1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    qn, kn = norms
    got, done = out.cpu().double(), torch.zeros(len(c.q), dtype=torch.bool)
    rows = {}
    for t, b, place in c.tokens():
        if place < 0:
            continue
        done[t] = True
        ref, mix = c.rotated(c.q[t], qn, eps, freq, c.prefix + place)
        tol = ref.abs() * torch.finfo(c.dtype).eps / 2 + mix * 2.0 ** -19 + 2.0 ** -25
        assert ((got[t] - ref).abs() <= tol).all(), (t, b, place)
        rows.setdefault((b, place // BLOCK), []).append((t, place))
    assert torch.equal(out.cpu()[~done], before[~done]), "rows of padding stay as they were"
    vc, ve, kc, ke = c.vc.clone(), c.ve.clone(), c.kc.clone(), c.ke.clone()
    kgot, kb = stored(c.kd, c.kb, c.page), c.kb.view(torch.uint8).cpu().double() - 127
    touched = torch.zeros((c.n_pages, c.page), dtype=torch.bool)
    for (b, blk), group in rows.items():
        page, u, keep = c.tables[b][blk * BLOCK // c.page], blk % c.units, group[0][1] % BLOCK
        here = slice(u * BLOCK, (u + 1) * BLOCK)
        touched[page, here] = True
        block_append(vc[page, :, here], ve[page, :, u], keep, torch.stack([c.vn[t].double() for t, _ in group]))
        pairs = [c.rotated(c.kn[t], kn, eps, freq, c.prefix + place) for t, place in group]
        x, err = torch.stack([p[0] for p in pairs]), torch.stack([p[1] for p in pairs]) * 2.0 ** -19
        least, most = (exponent((x.abs() + s * err).clamp(min=0).amax((0, 2))) for s in (-1, 1))
        if keep:
            least, most = torch.maximum(least, ke[page, :, u]), torch.maximum(most, ke[page, :, u])
        e = kb[page, :, u]
        assert ((least <= e) & (e <= most)).all(), (b, blk)
        if keep:
            again = e4m3(kc[page, :, here][:, :keep] * (2.0 ** (ke[page, :, u] - e))[:, None, None]) * (2.0 ** e)[:, None, None]
            assert torch.equal(kgot[page, :, here][:, :keep], again)
        new, ref = kgot[page, :, here][:, keep:keep + len(group)], x.transpose(0, 1)
        step = torch.maximum(ref.abs() * 2.0 ** -4, (2.0 ** (e - 10))[:, None, None])
        assert ((new - ref).abs() <= step + err.transpose(0, 1) * (1 + 2.0 ** -4)).all(), (b, blk)
    held = touched[:, None, :, None].expand_as(vc) & vc.isfinite()
    vgot = c.vd.view(torch.uint8).cpu().contiguous().view(torch.float8_e4m3fn).double()
    assert torch.equal(vgot[held], vc[held])
    units = touched[:, ::BLOCK][:, None].expand_as(ve)
    assert torch.equal((c.vb.view(torch.uint8).cpu().double() - 127)[units], ve[units])
    for now, was in zip((c.kd, c.vd, c.kb, c.vb), old):                 # what is no block of the step's
        part = ~(touched[:, None, :, None] if now.dim() == 4 else touched[:, ::BLOCK][:, None]).expand(now.shape)
        assert torch.equal(now.view(torch.uint8).cpu()[part], was[part])


def append(c, rot, qn=None, kn=None, eps=1e-5, q=None, out=None):
    from paper_2609_17184_amd import serving
    q = c.q.to(DEV) if q is None else q
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV) if out is None else out
    before, old = out.cpu(), [t.view(torch.uint8).cpu().clone() for t in (c.kd, c.vd, c.kb, c.vb)]
    got = serving.rope_append(q, c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, serving.rope_frequencies(rot) if rot else None,
                              q_norm=None if qn is None else qn.to(DEV), k_norm=None if kn is None else kn.to(DEV), eps=eps, out=out)
    assert got is out
    check_append(c, rot, (qn, kn), eps, out, before, old)


@pytest.mark.parametrize("spec", BATCHES, ids=lambda s: "-".join(str(x) for x in s[:5]))
@pytest.mark.parametrize("rot,norm,heads_first", [("all", False, True), ("half", True, False), ("none", True, True)])
def test_append(spec, rot, norm, heads_first):
    c = make(spec, seed=3, heads_first=heads_first)
    g = torch.Generator().manual_seed(5)
    qn, kn = ((1 + 0.3 * torch.randn(c.D, generator=g)) if norm else None for _ in range(2))
    append(c, {"all": c.D, "half": c.D // 2 // 16 * 16, "none": 0}[rot], qn, kn)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_steps_of_growing_and_falling_sizes(dtype):
    """One sequence, steps of 1 to 20 tokens whose sizes rise and fall by up to 2^20: kept codes are rounded again exactly
    where the scale grows; and again from an earlier length (a rejected draft), whose block keeps its scale."""
    from paper_2609_17184_amd import serving
    c = make((2, 2, 64, 32, dtype, [1], [1], 0), seed=4, width=4)
    pages = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(6)
    codes, scale = torch.zeros((8, 2, BLOCK, 64), dtype=torch.float64), torch.full((8, 2), 0.0, dtype=torch.float64)
    k, v = (torch.zeros((3, 2, 32, 64), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros((3, 2, 2), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2))
    cache = serving.QuantizedCache(k, v, ks, vs)
    length = 0
    for step, (n, size) in enumerate([(1, 0), (3, 3), (1, 6), (14, -5), (1, 9), (2, -9), (20, 1), (1, 8), (-6, 0), (1, -4), (2, 2), (7, 3)]):
        if n < 0:
            length += n
            continue
        x = (torch.randn((n, 2, 64), generator=g) * 2.0 ** size).to(c.dtype)
        length += n
        batch = serving.Batch(torch.tensor([length], dtype=torch.int32, device=DEV), pages, torch.tensor([0, n], dtype=torch.int32, device=DEV))
        serving.rope_append(x.to(DEV), x.to(DEV), x.to(DEV), cache, batch)
        at = length - n
        rest = x.double()
        while len(rest):
            keep = at % BLOCK
            block_append(codes[at // BLOCK], scale[at // BLOCK], keep, rest[:BLOCK - keep])
            at, rest = at + len(rest[:BLOCK - keep]), rest[BLOCK - keep:]
        want = (codes * (2.0 ** scale)[..., None, None]).transpose(1, 2).reshape(-1, 2, 64)[:length]
        for t, s in ((k, ks), (v, vs)):
            got = stored(t, s, 32)[[2, 0, 1]].transpose(1, 2).reshape(-1, 2, 64)[:length]
            assert torch.equal(got, want), step


@pytest.mark.parametrize("dtype,size", [("bf16", 3e38), ("bf16", 1e-30), ("bf16", 1e-38), ("f16", 65504.0), ("f16", 6e-8), ("bf16", 0.0)])
@pytest.mark.parametrize("n", [1, 9])
def test_extreme_values(dtype, size, n):
    """The types' largest and smallest values, zeros; NaN and infinities become NaN and do not move the scale."""
    c = make((2, 2, 64, 16, dtype, [n], [n + 3], 0), seed=4)
    for t in (c.kn, c.vn):
        t.copy_((torch.rand(t.shape) * size).to(c.dtype))
        t[0, 0, :3] = torch.tensor([math.nan, math.inf, -math.inf])
        t[-1, 1, 5] = size
    from paper_2609_17184_amd import serving
    serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch)
    # (keys neither normalised nor rotated are stored as they are)
    for got, codes, exps, x in ((stored(c.kd, c.kb, 16), c.kc, c.ke, c.kn), (stored(c.vd, c.vb, 16), c.vc, c.ve, c.vn)):
        page = c.tables[0][0]
        block_append(codes[page], exps[page, :, 0], 3, x.double())
        want = codes[page, :, :3 + n] * (2.0 ** exps[page, :, 0])[:, None, None]
        a, b = got[page, :, :3 + n], want
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0), b.nan_to_num(0))
        assert (exps >= LEAST).all()


def test_far_positions_views_and_in_place():
    from paper_2609_17184_amd import serving
    c = make((6, 2, 64, 16, "bf16", [1, 2], [4, 20], 0), heads_first=False, seed=8)
    c.prefix = 134217001
    c.batch._c.prefix_len = c.prefix
    fused = torch.cat([c.q.flatten(1), c.kn.flatten(1), c.vn.flatten(1)], 1).to(DEV)
    q, k, v = fused[:, :384].view(3, 6, 64), fused[:, 384:512].view(3, 2, 64), fused[:, 512:].view(3, 2, 64)
    old = [t.view(torch.uint8).cpu().clone() for t in (c.kd, c.vd, c.kb, c.vb)]
    serving.rope_append(q, k, v, c.cache, c.batch, serving.rope_frequencies(64), out=q)
    check_append(c, 64, (None, None), 0.0, q, q.cpu(), old)


@pytest.mark.parametrize("q_start", [True, False])
def test_padding_rows(q_start):
    if q_start:
        c = Quantized(4, 2, 32, 16, "f16", [2, 3, 40, 1], [-1, 2, 60, 0], 20, extra=5, first=2)
    else:
        c = Quantized(4, 2, 32, 16, "f16", [1, 1, 1, 1], [-1, 2, 30, 0], 20, extra=5, q_start=False)
    append(c, 32)


def test_pages_outside_the_cache_are_left_out():
    from paper_2609_17184_amd import serving
    c = make((4, 2, 64, 16, "f16", [1, 1, 1], [40, 17, 10], 0), seed=1)
    c.batch.table[0, 2] = c.n_pages
    c.batch.table[1, 1] = -1
    old = [t.view(torch.uint8).clone() for t in (c.kd, c.kb)]
    q = serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, serving.rope_frequencies(64))
    changed = (c.kd.view(torch.uint8) != old[0]).any(-1).any(1).nonzero().tolist()
    assert [c.tables[2][0], 9] in changed and all(p == c.tables[2][0] for p, _ in changed) and not q.isnan().any()
    seq = c.batch.seq_len.clone()
    c.batch.seq_len[:] = 16 * c.batch.table.shape[1] + 1                # behind the tables' ends
    old = [t.view(torch.uint8).clone() for t in (c.kd, c.kb)]
    serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch)
    assert torch.equal(c.kd.view(torch.uint8), old[0]) and torch.equal(c.kb.view(torch.uint8), old[1])


def test_refusals():
    from paper_2609_17184_amd import serving
    c = make((4, 2, 64, 16, "f16", [1, 1], [40, 17], 0), seed=1)
    k, s = c.kd, c.kb
    bad = [(k, k.view(torch.uint8), s, s), (k, k[:, :1], s, s), (k, k, s[:-1], s[:-1]), (k, k, s.view(torch.uint8), s),
           (k.cpu(), k.cpu(), s.cpu(), s.cpu()), (k.half(), k.half(), s, s), (k, k, s, s.transpose(0, 1))]
    for args in bad:
        with pytest.raises(ValueError):
            serving.QuantizedCache(*args)
    q, n = c.q.to(DEV), c.kn.to(DEV)
    for args in ((q, n.bfloat16(), n.bfloat16()), (q.float(), n.float(), n.float()), (q, n, n[:1])):
        with pytest.raises(ValueError):
            serving.rope_append(*args, c.cache, c.batch)
    from paper_2609_17184_amd import LoopSpecError
    odd = torch.zeros((4, 2, 16, 72), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)[..., :64]
    scales = torch.zeros((4, 2, 1), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    cache = serving.QuantizedCache(odd, odd, scales, scales)           # strides of 72 bytes
    with pytest.raises(LoopSpecError):
        serving.rope_append(q, n, n, cache, c.batch)
    with pytest.raises(LoopSpecError):
        serving.window_attention(q, cache, c.batch)


def test_more_tokens_than_workgroups_of_one_token():
    """Over four million sequences of one token, most of them without positions: rows of padding stay as they are, and no
    launch is too large."""
    from paper_2609_17184_amd import serving
    T = (1 << 22) + 37
    at = [0, 5, 16, 1 << 22, T - 1]
    g = torch.Generator().manual_seed(12)
    lens = torch.full((T,), -1, dtype=torch.int32)
    tables = torch.full((T, 1), -1, dtype=torch.int32)
    for i, t in enumerate(at):
        lens[t], tables[t, 0] = 1 + 3 * i, i
    q, k, v = (torch.zeros((T, 1, 16), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    rows = [torch.randn((len(at), 1, 16), generator=g).to(torch.bfloat16) for _ in range(3)]
    for x, r in zip((q, k, v), rows):
        x[at] = r.to(DEV)
    codes = [torch.zeros((len(at), 1, 16, 16), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
    scales = [torch.zeros((len(at), 1, 1), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2)]
    out = torch.full_like(q, 3.0)
    serving.rope_append(q, k, v, serving.QuantizedCache(*codes, *scales), serving.Batch(lens.to(DEV), tables.to(DEV)), out=out)
    assert torch.equal(out[at].cpu(), rows[0])
    out[at] = 3.0
    assert (out == 3.0).all()
    for x, c, s in zip(rows[1:], codes, scales):
        got = stored(c, s, 16)
        for i in range(len(at)):
            e = exponent(x[i].double().abs().max().reshape(1)).item()
            if i == 0:
                assert torch.equal(got[i, 0, 0], e4m3(x[i, 0].double() * 2.0 ** -e) * 2.0 ** e)
            else:                             # (the positions below have the scale 2^-127, which grows to the new one's)
                assert torch.equal(got[i, 0, 3 * i], e4m3(x[i, 0].double() * 2.0 ** -e) * 2.0 ** e)
