"""8-bit pages and windows for the serving operators' tests, in 64 bits."""
import math

import torch

from serving_common import DT, Case

CODE, SCALE, BLOCK, LEAST = torch.float8_e4m3fn, torch.float8_e8m0fnu, 16, -64


def exponent(amax):
    """The smallest e >= LEAST with amax <= 448 * 2^e, amax a float64 tensor."""
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / 448))
    e = torch.where(amax > 448 * 2.0 ** e, e + 1, torch.where(amax <= 448 * 2.0 ** (e - 1), e - 1, e))
    return torch.where(amax > 0, e, LEAST).clamp(min=LEAST)


def e4m3(x):
    """Rounded to e4m3's values (ties to even); NaN where not finite."""
    step = 2.0 ** (torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6).nan_to_num(1.0, 1.0, 1.0))) - 3)
    return torch.where(x.isfinite(), torch.round(x / step) * step, math.nan)


def block_append(codes, scale, keep, x):
    """Rows x [n, G, D] behind the `keep` positions of a block: codes [G, 16, D] and scale exponents [G], float64, changed
    in place."""
    e = exponent(torch.where(x.isfinite(), x.abs(), 0.0).amax((0, 2)))
    if keep:
        e = torch.maximum(e, scale)
        codes[:, :keep] = e4m3(codes[:, :keep] * (2.0 ** (scale - e))[:, None, None])
    codes[:, keep:keep + len(x)] = e4m3(x.transpose(0, 1) * (2.0 ** -e)[:, None, None])
    scale.copy_(e)


def as_codes(x):
    return x.float().to(CODE)


class Quantized(Case):
    """The same batch over 8-bit pages.  Places without a position hold NaN codes, blocks without one a NaN scale."""

    def __init__(self, *args, spread=1.0, garbage=True, **kw):
        super().__init__(*args, **kw)
        from paper_2609_17184_amd import serving
        dev = "cuda:0"
        g = torch.Generator().manual_seed(kw.get("seed", 0) + 99)
        self.units = self.page // BLOCK
        made = []
        for name in ("k", "v"):
            x = getattr(self, name).double()                            # [pages, G, page, D]
            x = x * torch.exp(spread * torch.randn((self.n_pages, self.G, 1, 1), generator=g, dtype=torch.float64))
            x = x.reshape(self.n_pages, self.G, self.units, BLOCK, self.D)
            held = ~x.isnan().all(-1)
            e = exponent(torch.where(x.isfinite(), x.abs(), 0.0).amax((3, 4)))
            codes = e4m3(x * (2.0 ** -e)[..., None, None])
            value = (codes * (2.0 ** e)[..., None, None]).reshape(self.n_pages, self.G, self.page, self.D)
            setattr(self, name, value)
            byte = torch.where(held.any(-1), e + 127, 255 if garbage else 60).to(torch.uint8)
            codes = codes.reshape(self.n_pages, self.G, self.page, self.D)
            made.append((codes, e, byte))
        (self.kc, self.ke, kb), (self.vc, self.ve, vb) = made
        heads_first = kw.get("heads_first", True)

        def put(codes):
            codes = as_codes(codes)
            if heads_first:
                return codes.to(dev)
            return codes.view(torch.uint8).transpose(1, 2).contiguous().to(dev).transpose(1, 2).view(CODE)
        self.kd, self.vd = put(self.kc), put(self.vc)
        self.kb, self.vb = kb.to(dev).view(SCALE), vb.to(dev).view(SCALE)
        self.cache = serving.QuantizedCache(self.kd, self.vd, self.kb, self.vb)


def stored(codes, scale, page):
    """The values that codes and scales on the device stand for, float64 on the host."""
    c = codes.view(torch.uint8).cpu().contiguous().view(CODE).double()
    b = scale.view(torch.uint8).cpu().double()
    s = torch.where(b == 255, math.nan, 2.0 ** (b - 127)).repeat_interleave(BLOCK, 2)[..., None]
    return c * s


def windowed(c, window, sinks, scale):
    """Per token that is no padding: output [H, D], log-sum-exp [H], the weights' mean of |v| [H, D], the largest sum of
    |q| |k| [H], the largest |v| [H, 1]."""
    per = c.H // c.G
    kp, vp = c.get(c.k, c.ptable, c.prefix), c.get(c.v, c.ptable, c.prefix)
    for b, n in enumerate(c.new):
        length = c.lens[b]
        if length < 0 or not n:
            continue
        K = torch.cat([kp, c.get(c.k, c.tables[b], length)]).repeat_interleave(per, 1)
        V = torch.cat([vp, c.get(c.v, c.tables[b], length)]).repeat_interleave(per, 1)
        for i in range(n):
            t, place = c.starts[b] + i, length - n + i
            p = c.prefix + place
            j = torch.arange(len(K))
            see = (j <= p) & ((p - j < window) | (j < sinks)) if window else j <= p
            if place < 0 or not see.any():
                z = torch.zeros((c.H, c.D), dtype=torch.float64)
                yield t, z, torch.full((c.H,), -math.inf, dtype=torch.float64), z, z[:, 0], z[:, :1]
                continue
            k, v, q = K[see], V[see], c.q[t].double()
            s = (k * q).sum(-1) * scale
            w = torch.softmax(s, 0)[..., None]
            yield (t, (w * v).sum(0), torch.logsumexp(s, 0), (w * v.abs()).sum(0), (k.abs() * q.abs()).sum(-1).amax(0) * scale,
                   v.abs().amax((0, 2))[:, None])


def behind_a_prefix(c, scale):
    """The same without a window for batches of one token per sequence, whose sums over the prefix take too long one by one:
    all of them at once."""
    per, B, most = c.H // c.G, len(c.new), max(c.lens)
    q = c.q[c.first:c.first + B].double().reshape(B, c.G, per, c.D)
    own = [torch.zeros((B, most, c.G, c.D), dtype=torch.float64) for _ in "kv"]
    for b, n in enumerate(c.lens):
        for x, pages in zip(own, (c.k, c.v)):
            x[b, :n] = c.get(pages, c.tables[b], n)
    (kp, vp), (ko, vo) = (c.get(x, c.ptable, c.prefix) for x in (c.k, c.v)), own
    behind = torch.arange(most)[None] >= torch.tensor(c.lens)[:, None]
    rows = [[] for _ in range(5)]
    for g in range(c.G):
        # [positions, D] of the prefix and [B, positions, D] of each sequence
        both = lambda a, p, o: torch.cat([(a.reshape(-1, c.D) @ p[:, g].T).reshape(B, per, -1), a @ o[:, :, g].transpose(1, 2)], 2)  # noqa: E731
        mix = lambda w, p, o: (w[:, :, :c.prefix].reshape(B * per, -1) @ p[:, g]).reshape(B, per, c.D) + w[:, :, c.prefix:] @ o[:, :, g]  # noqa: E731
        s = both(q[:, g], kp, ko) * scale
        s[:, :, c.prefix:].masked_fill_(behind[:, None], -math.inf)
        big = both(q[:, g].abs(), kp.abs(), ko.abs()).amax(2) * scale
        w = torch.softmax(s, 2)
        top = torch.maximum(vp[:, g].abs().max(), vo[:, :, g].abs().amax((1, 2)))[:, None].expand(B, per)
        for to, x in zip(rows, (mix(w, vp, vo), torch.logsumexp(s, 2), mix(w, vp.abs(), vo.abs()), big, top)):
            to.append(x)
    ref, lse, mean, big, top = (torch.stack(x, 1).flatten(1, 2) for x in rows)
    for b in range(B):
        yield c.first + b, ref[b], lse[b], mean[b], big[b], top[b][:, None]


def check_window(c, window, sinks, scale, out, lse, before, rows=None):
    """A weight is rounded to 16 bits (half a step), the output once more; the score's fp32 sum of D products is off by at
    most (D + 8) 2^-24 of the sum of their magnitudes, which moves a weight by as much; sums over n positions add n 2^-24;
    weights (times their values' scale) below 2^-31 of the largest vanish.  fp16's subnormals are spaced 2^-24."""
    h = torch.finfo(c.dtype).eps / 2
    got, glse = out.cpu().double(), lse.cpu().double()
    seen = torch.zeros(len(c.q), dtype=torch.bool)
    worst = 0.0
    for t, ref, rlse, mean, big, most in rows or windowed(c, window, sinks, scale):
        seen[t] = True
        n = c.prefix + max(c.lens) + 16
        ds = ((c.D + 8) * 2.0 ** -24 * big + n * 2.0 ** -24)[:, None]
        tol = mean * (h + 2 * ds) + ref.abs() * h + n * 2.0 ** -30 * most + 2.0 ** -25
        err = (got[t] - ref).abs()
        assert (err <= tol).all(), (t, (err - tol).max(), err.max())
        worst = max(worst, (err / tol).max().item())
        inf = rlse == -math.inf
        assert torch.equal(glse[t] == -math.inf, inf), t
        lerr = (glse[t] - rlse).abs()[~inf]
        assert (lerr <= (2 * ds[:, 0] + rlse.abs() * 2.0 ** -22 + 2.0 ** -20)[~inf]).all(), (t, lerr.max())
    assert torch.equal(out.cpu()[~seen], before[~seen]), "rows of padding stay as they were"
    return worst
