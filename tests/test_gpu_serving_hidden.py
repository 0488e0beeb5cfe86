"""What attention rows must not see has no influence on them, bit for bit: blocks in which all of a wave's rows belong
to one token while the workgroup's positions go on to a later token's."""
import pytest
import torch

from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _same(c, q, out, lse, see):
    from paper_2609_17184_amd import serving
    o, s = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    assert torch.equal(o[see], out[see]) and torch.equal(s[see], lse[see])
    return o


@pytest.mark.parametrize("heads", [32, 48, 64, 96])
@pytest.mark.parametrize("D,tokens,length,prefix", [(128, 4, 134, 100), (64, 2, 65, 0), (16, 7, 520, 33), (96, 3, 3, 1)])
def test_last_token_of_many_heads(heads, D, tokens, length, prefix):
    """32 and more query heads to a key/value head: NaN and infinities in the last token's key and value, alone and
    together, and its page outside the cache, leave the earlier tokens as they were."""
    from paper_2609_17184_amd import serving
    c = Case(heads, 1, D, 32, "bf16" if heads == 48 else "f16", [tokens, 3], [length, 90], prefix, seed=heads + D)
    q = c.q.to(DEV)
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    assert not out.isnan().any()
    see = [i for i in range(tokens + 3) if i != tokens - 1]
    page, at = c.tables[0][(length - 1) // 32], (length - 1) % 32
    kept = [t[page, :, at].clone() for t in (c.kd, c.vd)]
    for bad in (float("nan"), float("inf"), float("-inf")):
        for which in ((c.kd,), (c.vd,), (c.kd, c.vd)):
            for t in which:
                t[page, :, at] = bad
            _same(c, q, out, lse, see)
            for t, old in zip((c.kd, c.vd), kept):
                t[page, :, at] = old
    if at == 0:                               # the last token begins a page of its own
        c.batch.table[0, (length - 1) // 32] = c.n_pages
        assert _same(c, q, out, lse, see)[tokens - 1].isnan().all()


@pytest.mark.parametrize("H,G,D,page,new,lens,prefix,first", [
    (8, 2, 64, 16, [6, 2], [45, 2], 40, 42), (4, 2, 128, 32, [70, 40], [200, 40], 100, 150), (16, 1, 32, 48, [5, 1], [700, 9], 0, 698),
    (6, 6, 96, 16, [40, 30], [1100, 30], 7, 1075)])
def test_last_tokens_of_few_heads(H, G, D, page, new, lens, prefix, first):
    """The first sequence's keys and values from position `first` on: bit for bit nothing for the tokens before it and
    the other sequence's."""
    from paper_2609_17184_amd import serving
    c = Case(H, G, D, page, "f16" if D < 96 else "bf16", new, lens, prefix, seed=9)
    q = c.q.to(DEV)
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    see = list(range(new[0] - (lens[0] - first))) + list(range(new[0], sum(new)))
    assert 0 < len(see) < sum(new)
    for bad in (float("nan"), float("inf"), float("-inf"), 60000.0):
        for t in (c.kd, c.vd):
            for place in range(first, lens[0]):
                t[c.tables[0][place // page], :, place % page] = bad
        _same(c, q, out, lse, see)
