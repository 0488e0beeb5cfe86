"""An attention row's bits are its own: another token's query, a padding row's, another sequence's keys change nothing
in it, on every path of the kernel (16 and 32 rows a wave, blocks of rows over the prefix and over own positions)."""
import pytest
import torch

from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# heads = key/value heads, head_dim, tokens and own positions per sequence, prefix; 64 heads leave a workgroup a chunk of
# 1024 positions of the prefix
PATHS = {
    "16 rows a wave": (64, 16, [1] * 9, [30 + i for i in range(9)], 8192),
    "32 rows a wave": (64, 16, [1] * 25, [30 + i for i in range(25)], 8192),
    "blocks of 64 rows": (64, 16, [1] * 60, [30 + i for i in range(60)], 8192),
    "blocks of 128 rows": (64, 16, [1] * 270, [2 + i % 30 for i in range(270)], 8192),
    "own positions": (4, 64, [6, 3], [120, 100], 0),
    "own positions, blocks": (8, 64, [60, 40], [900, 700], 20),
}


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_steep_row(path, dtype):
    """Keys whose first element rises every 32 positions, and queries that do not look at it, but for one in the second
    run: its largest score rises by some 18 octaves a tile of 32 positions."""
    from paper_2609_17184_amd import serving
    H, D, new, lens, prefix = PATHS[path]
    c = Case(H, H, D, 32, dtype, new, lens, prefix, seed=len(new), extra=2)
    for table in [c.ptable] + c.tables:
        if table:
            rise = (torch.arange(len(table) * 32) // 32).view(-1, 32) * 0.5
            c.kd[torch.tensor(table, device=DEV), :, :, 0] = rise[:, None].to(c.dtype).to(DEV)
    T, victim = sum(new), new[0] // 2
    q = c.q.to(DEV)
    q[:, :, 0] = 0
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    assert out[:T].isfinite().all()
    others = [t for t in range(T) if t != victim]
    q[victim, :, 0] = 200 * 8 * D ** -0.5
    q[T] = float("inf")
    q[T + 1] = 1000
    o, s = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    assert torch.equal(s[others], lse[others])
    assert torch.equal(o[others], out[others])
    assert not torch.equal(o[victim], out[victim])


def test_another_sequence():
    """Another sequence's keys, values, length and query."""
    from paper_2609_17184_amd import serving
    c = Case(64, 64, 16, 16, "f16", [1, 2, 1], [40, 50, 60], 8192, seed=3)
    q = c.q.to(DEV)
    out, lse = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    q[1:3] *= 100
    for t in (c.kd, c.vd):
        t[torch.tensor(c.tables[1], device=DEV)] *= 50
    c.batch.seq_len[1] = 35
    o, s = serving.prefix_attention(q, c.cache, c.batch, return_lse=True)
    assert torch.equal(o[[0, 3]], out[[0, 3]]) and torch.equal(s[[0, 3]], lse[[0, 3]])
