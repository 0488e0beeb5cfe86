"""Batches over a paged cache for the serving operators' tests, and the operators in 64 bits."""
import math

import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


class Case:
    """A batch on the GPU with random pages.  new[b] tokens and lens[b] own positions per sequence; every place of
    the cache that holds none of the batch's positions is `hole`."""

    def __init__(self, H, G, D, page, dtype, new, lens, prefix, seed=0, hole=float("nan"), heads_first=True, extra=0,
                 q_start=True, width=None, first=0):
        from paper_2609_17184_amd import serving
        g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.D, self.page, self.dtype = H, G, D, page, DT[dtype]
        self.new, self.lens, self.prefix, self.first = list(new), list(lens), prefix, first
        B = len(new)
        own = [-(-max(n, 0) // page) for n in lens]
        npre = -(-prefix // page)
        perm = torch.randperm(npre + sum(own) + 2, generator=g).tolist()
        self.n_pages = len(perm)
        self.ptable = [perm.pop() for _ in range(npre)]
        self.tables = [[perm.pop() for _ in range(n)] for n in own]
        width = max(own + [1]) if width is None else width
        tab = torch.full((B, width + 3), -7, dtype=torch.int32)
        for b, t in enumerate(self.tables):
            tab[b, :min(len(t), width)] = torch.tensor(t[:width], dtype=torch.int32)
        shape = (self.n_pages, G, page, D) if heads_first else (self.n_pages, page, G, D)
        self.k, self.v = (torch.full(shape, hole, dtype=self.dtype) for _ in range(2))
        if not heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for table, n in [(self.ptable, prefix)] + list(zip(self.tables, lens)):
            for c in (self.k, self.v):
                self.put(c, table, 0, torch.randn((max(n, 0), G, D), generator=g).to(self.dtype))
        T = first + sum(new) + extra
        self.q = (torch.randn((T, H, D), generator=g) * 1.5).to(self.dtype)
        self.kn, self.vn = (torch.randn((T, G, D), generator=g).to(self.dtype) for _ in range(2))
        starts = [first]
        for n in new:
            starts.append(starts[-1] + n)
        self.starts = starts
        dev = "cuda:0"
        # (a transposed view keeps its strides on the way to the device)
        self.kd, self.vd = (c.transpose(1, 2).to(dev).transpose(1, 2) if not heads_first else c.to(dev)
                            for c in (self.k, self.v))
        self.cache = serving.PagedCache(self.kd, self.vd)
        self.batch = serving.Batch(torch.tensor(lens, dtype=torch.int32, device=dev), tab.to(dev)[:, :width],
                                   torch.tensor(starts, dtype=torch.int32, device=dev) if q_start else None, prefix,
                                   torch.tensor(self.ptable, dtype=torch.int32, device=dev) if prefix else None)

    def put(self, c, table, at, rows):
        for i, r in enumerate(rows):
            c[table[(at + i) // self.page], :, (at + i) % self.page] = r

    def get(self, c, table, n):
        if n <= 0:
            return torch.zeros((0, self.G, self.D), dtype=torch.float64)
        pages = c[torch.tensor(table[:-(-n // self.page)])].transpose(1, 2)
        return pages.reshape(-1, self.G, self.D)[:n].double()

    def tokens(self):
        """(token, sequence, own position) of every token that is no padding."""
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            for i in range(n):
                if length >= 0:
                    yield self.starts[b] + i, b, length - n + i

    def attention(self, scale):
        """Per token: output [H, D], log-sum-exp [H], and what the tolerances need: the weights' mean of |v| [H, D] and
        the largest sum of |q| |k| [H]."""
        per = self.H // self.G
        kp, vp = self.get(self.k, self.ptable, self.prefix), self.get(self.v, self.ptable, self.prefix)
        for t, b, place in self.tokens():
            n = max(place + 1, 0)
            K = torch.cat([kp, self.get(self.k, self.tables[b], n)]).repeat_interleave(per, 1)
            V = torch.cat([vp, self.get(self.v, self.tables[b], n)]).repeat_interleave(per, 1)
            q = self.q[t].double()
            if not len(K):
                z = torch.zeros((self.H, self.D), dtype=torch.float64)
                yield t, z, torch.full((self.H,), -math.inf, dtype=torch.float64), z, z[:, 0]
                continue
            s = (K * q).sum(-1) * scale                     # [positions, H]
            p = torch.softmax(s, 0)[..., None]
            yield (t, (p * V).sum(0), torch.logsumexp(s, 0), (p * V.abs()).sum(0),
                   (K.abs() * q.abs()).sum(-1).amax(0) * scale)

    def rotated(self, x, gain, eps, freq, position):
        """One token's heads [heads, D] in 64 bits, and the bound of |x_j| + |x_j'| of what the rotation mixes."""
        x = x.double()
        if gain is not None:
            x = x * gain.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        h = 0 if freq is None else len(freq)
        if not h:
            return x, x.abs()
        a = position * freq.double()
        u, w = x[:, :h], x[:, h:2 * h]
        mix = u.abs() + w.abs()
        return (torch.cat([u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin(), x[:, 2 * h:]], 1),
                torch.cat([mix, mix, x[:, 2 * h:].abs()], 1))
