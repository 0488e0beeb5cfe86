"""NaN and infinities among the values that rows of a prompt see: they reach every row that sees them, in their column, and
no other.  Blocks of 128 rows share what they bring, and their rows do not see the same of it."""
import math

import pytest
import torch

from quantized_common import Quantized
from serving_common import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def positions(c, b):
    """Position (through the prefix) of every token of sequence b."""
    return torch.arange(c.new[b]) + c.prefix + c.lens[b] - c.new[b]


def visible(c, b, j, window, sinks):
    """Which tokens of sequence b see position j."""
    p = positions(c, b)
    see = (j <= p) & (p >= c.prefix)
    return see & ((p - j < window) | (torch.tensor(j) < sinks)) if window else see


def place(c, b, j):
    """Page and offset of position j as sequence b has it."""
    table, i = (c.ptable, j) if j < c.prefix else (c.tables[b], j - c.prefix)
    return table[i // c.page], i % c.page


def poison(c, eight, b, j, g, d, x):
    page, at = place(c, b, j)
    if eight:
        c.vd.view(torch.uint8)[page, g, at, d] = 0x7F       # (e4m3 has no infinities)
    else:
        c.vd[page, g, at, d] = x


def run(c, window, sinks):
    from paper_2609_17184_amd import serving
    return serving.window_attention(c.q.to(DEV), c.cache, c.batch, window, sinks).cpu()


def expect(want, c, b, j, g, d, x, window, sinks):
    """Add x to the outputs of the rows that see it, whose weights for it are positive."""
    per = c.H // c.G
    see = torch.zeros(len(c.q), dtype=torch.bool)
    for s in range(len(c.new)) if j < c.prefix else [b]:
        see[c.starts[s]:c.starts[s] + c.new[s]] = visible(c, s, j, window, sinks)
    want[see, g * per:(g + 1) * per, d] += x


def same(got, want):
    """Finite outputs bit for bit (a value that is not finite enters no other column), the others of one kind."""
    assert torch.equal(got.isnan(), want.isnan())
    fine = ~want.isnan()
    assert torch.equal(got[fine], want[fine])


# heads, key/value heads, head_dim, page, type, tokens and own positions per sequence, prefix
PROMPTS = {
    "50": (4, 2, 64, 16, "bf16", [50], [100], 0),
    "128": (2, 2, 128, 16, "f16", [128], [128], 0),
    "129": (8, 2, 96, 48, "f16", [129], [129], 0),
    "300": (3, 3, 32, 32, "bf16", [300], [310], 0),
    "prefix": (2, 1, 128, 16, "bf16", [150], [150], 40),
    "two": (4, 4, 16, 64, "f16", [130, 70], [200, 71], 21),
    "short": (2, 2, 64, 16, "f16", [129], [100], 0),
    "short-prefix": (2, 2, 64, 16, "bf16", [129], [90], 300),
    # rows of several tokens in blocks of 16, over a prefix with the other sequences' and alone
    "few": (8, 2, 64, 16, "bf16", [9], [100], 0),
    "few-short": (4, 2, 96, 32, "f16", [7, 3], [3, 130], 70),
    "together": (8, 2, 128, 16, "bf16", [3] * 20, [30] * 20, 700),
    "together-few": (4, 4, 32, 16, "f16", [2] * 5, [20] * 5, 900),
}


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 0), (100, 50)])
@pytest.mark.parametrize("name", PROMPTS)
def test_one_value(name, window, sinks, eight):
    """One at a time, at places on either side of every 16, 32 and 64 positions, in the prefix and in the sequence's own."""
    H, G, D, page, dt, new, lens, prefix = PROMPTS[name]
    c = (Quantized if eight else Case)(H, G, D, page, dt, new, lens, prefix, seed=7)
    clean = run(c, window, sinks)
    assert clean.isfinite().all()
    kept = c.vd.clone()
    n = prefix + lens[0]
    spots = sorted({x for o in (0, prefix) for m in (16, 32, 64) for k in range(n // m + 1) for x in (o + k * m - 1, o + k * m)}
                   | {10, n // 2, n - 1} & set(range(n)))
    for i, j in enumerate(x for x in spots if 0 <= x < n):
        x = math.nan if eight else (math.nan, math.inf, -math.inf)[i % 3]
        g, d = i % G, (5 * i + 3) % D
        poison(c, eight, 0, j, g, d, x)
        want = clean.clone()
        expect(want, c, 0, j, g, d, x, window, sinks)
        got = run(c, window, sinks)
        assert torch.equal(got.isnan(), want.isnan()), (j, i % 3)
        same(got, want)
        c.vd.copy_(kept)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (333, 20)])
@pytest.mark.parametrize("new,lens,prefix", [([300], [700], 0), ([100, 200], [90, 150], 2500)], ids=["own", "prefix"])
def test_many_values(new, lens, prefix, window, sinks, eight):
    """Every seventh position at once, more than a block of rows keeps a list of: in a column each of 32, so that rows differ
    in which of their columns are finite."""
    c = (Quantized if eight else Case)(2, 2, 32, 16, "bf16", new, lens, prefix, seed=8)
    clean = run(c, window, sinks)
    want = clean.clone()
    for b in range(len(new)):
        for j in range(prefix if b else 0, prefix + lens[b], 7):
            x = math.nan if eight or j % 5 == 0 else math.inf if j % 4 else -math.inf
            g, d = j // 7 % 2, j // 50 % 32
            poison(c, eight, b, j, g, d, x)
            expect(want, c, b, j, g, d, x, window, sinks)
    assert not want.isfinite().all() and want.isfinite().any()
    same(run(c, window, sinks), want)
