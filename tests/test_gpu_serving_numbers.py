"""Numbers beyond 32 bits are taken for what they are, or refused."""
import pytest
import torch

from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_top_k_of_any_size():
    from paper_2609_17184_amd import serving
    z = torch.randn((4, 500), device=DEV)
    u = torch.rand(4, dtype=torch.float64, device=DEV)
    every = serving.sample(z, u)
    for k in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 2 ** 40 + 3, -2 ** 31 - 1, -2 ** 32 + 1):
        assert all(torch.equal(a, b) for a, b in zip(every, serving.sample(z, u, top_k=k))), k
    with pytest.raises((TypeError, ValueError)):
        serving.sample(z, u, top_k=1.5)


def test_sizes_beyond_32_bits_are_refused():
    from paper_2609_17184_amd import serving
    with pytest.raises((ValueError, serving.B.LoopSpecError)):
        serving.sample(torch.empty((1, 2 ** 32 + 5), dtype=torch.float16, device=DEV),
                       torch.zeros(1, dtype=torch.float64, device=DEV))
    c = Case(2, 2, 16, 16, "f16", [1], [1], 0)
    for n in (2 ** 32 + 8, 2 ** 31, -2 ** 32):
        with pytest.raises((ValueError, serving.B.LoopSpecError)):
            batch = serving.Batch(c.batch.seq_len, c.batch.table, None, n)
            serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, batch)
    wide = torch.empty((1, 2, 16), dtype=c.dtype, device=DEV)
    with pytest.raises((ValueError, serving.B.LoopSpecError)):
        serving.prefix_attention(wide.expand(2 ** 32 + 1, 2, 16), c.cache, c.batch, out=wide.expand(2 ** 32 + 1, 2, 16))
