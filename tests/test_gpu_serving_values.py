"""Attention over values of every magnitude that bf16 has: a weighted mean of finite values is finite."""
import pytest
import torch

from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("new,lens,prefix", [([1, 1, 3], [40, 1, 100], 2000), ([1] * 60, [2 + i for i in range(60)], 700),
                                             ([70, 40], [300, 60], 50)], ids=["few", "many", "prompts"])
def test_powers_of_two(new, lens, prefix):
    """Values times 2^k give outputs times 2^k, bit for bit: normal values below 2^7 and above 2^-20 or so, and weights
    within 60 octaves of the largest, stay normal numbers in every product and sum."""
    from paper_2609_17184_amd import serving
    c = Case(8, 2, 64, 16, "bf16", new, lens, prefix, seed=17)
    q = c.q.to(DEV)
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    v = c.vd.clone()
    for k in (-40, 100, 120):
        c.vd.copy_(v.float() * 2.0 ** k)
        o, s = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
        assert torch.equal(s, lse)
        assert torch.equal(o.double(), out.double() * 2.0 ** k), k


def test_equal_values_of_many_positions():
    """30000 positions of one weight and one value near the type's end: the mean is the value, within a rounded weight's
    half step and the output's."""
    from paper_2609_17184_amd import serving
    c = Case(2, 2, 32, 64, "bf16", [1], [1], 30000, seed=18)
    c.kd.zero_()
    c.vd.fill_(2.0 ** 126)
    out, lse = serving.prefix_attention(c.q.to(DEV), c.cache, c.batch, return_lse=True)
    assert ((out.double() / 2.0 ** 126 - 1).abs() <= 2 * torch.finfo(torch.bfloat16).eps / 2 + 30001 * 2.0 ** -24).all()
    # (an fp32 sum of 30001 equal terms, the logarithm and its fp32 result)
    assert ((lse.double() - torch.tensor(30001.0, dtype=torch.float64).log()).abs() <= 30001 * 2.0 ** -24 + 2.0 ** -18).all()
