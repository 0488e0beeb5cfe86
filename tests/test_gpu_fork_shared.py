"""Rows that were shortened into pages they share: a fork gives every child pages of its own for what it appends next."""
import ctypes
import random

import pytest
import torch

from test_gpu_fork import KINDS, copied, layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference(lens, table, parent, refs, page, window, sinks, room):
    """(lens, table, refs, short, copies (source, page, positions)), from the counts and tables alone."""
    n_pages, width, given = len(refs), len(table[0]), list(refs)
    held_by = lambda p, x: sum(y == x for y in table[p])
    out, heirs, wants, later, short = [], set(), [], [], 0
    for n, row in zip(lens, table):
        for x in row:
            if n >= 0 and 0 <= x < n_pages:
                given[x] -= 1
    for j, p in enumerate(parent):
        row = [-1] * width
        if 0 <= p < len(lens) and lens[p] >= 0:
            n, heir = lens[p], p not in heirs
            heirs.add(p)
            held = min(-(-n // page), width)
            need = -(-(min(n, width * page) + room) // page) if room else held
            short += max(0, need - width)
            for i, x in enumerate(table[p]):
                ok = 0 <= x < n_pages
                gone = window and (i + 1) * page - 1 <= n - window and i * page >= sinks
                if ok and (i + 1) * page <= n:
                    row[i] = -1 if gone else x
                elif ok and heir and refs[x] == held_by(p, x):       # nobody else's
                    row[i] = x
                elif i < held:
                    if ok:
                        wants.append((j, i, x))
                        later += [x] if heir else []
                elif i < need:
                    wants.append((j, i, -1))
            out.append((n, row))
        else:
            out.append((-1, row))
        for x in row:
            if x >= 0:
                given[x] += 1
    # (a page that its own heir has a copy of is not given out in the same step)
    free = [x for x in range(n_pages) if given[x] == 0 and x not in later]
    copies = []
    for (j, i, source), x in zip(wants, free):
        out[j][1][i], given[x] = x, 1
        if source >= 0:
            copies.append((source, x, out[j][0] % page))
    return [n for n, _ in out], [r for _, r in out], given, short + max(0, len(wants) - len(free)), copies


def shared_batch(rng, n, page, n_pages, width):
    """Rows that begin with pages of the row before, and lengths that end anywhere in what they hold."""
    pages = list(range(n_pages))
    rng.shuffle(pages)
    lens, table = [], []
    for b in range(n):
        held = rng.randint(0, width - 1)
        row = [pages.pop() for _ in range(held)] + [-1] * (width - held)
        if b and rng.random() < 0.7:
            k = rng.randint(0, width)
            row[:k] = table[-1][:k]
        lens.append(rng.choice([-1, rng.randint(0, width * page), rng.randint(0, held * page)]))
        table.append(row)
    refs = [0] * n_pages
    for length, row in zip(lens, table):
        for x in row:
            if length >= 0 and x >= 0:
                refs[x] += 1
    return lens, table, refs


def check(lens, table, parent, refs, page, made, window=0, sinks=0, room=0):
    from paper_2609_17184_amd import serving
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    want = reference(lens, table, parent, refs, page, window, sinks, room)
    after = copied(made, want[4])
    got = serving.fork_pages(dev(lens), dev(table), dev(parent), dev(refs), [m[0] for m in made], 0, window, sinks, room)
    assert [t.tolist() for t in got] == [*want[:3], [want[3]]]
    now = [t.cpu() for _, raw, scales, _ in made for t in raw + scales]
    assert all(torch.equal(a, b) for a, b in zip(now, after))
    # the pages that a child appends to are its own
    for n, row in zip(want[0], want[1]):
        for i, x in enumerate(row):
            assert n < 0 or x < 0 or (i + 1) * page <= n or want[2][x] == sum(y == x for y in row)
    return want


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n,m", [(2, 2), (20, 30), (90, 120)])
@pytest.mark.parametrize("window,sinks,room", [(0, 0, 0), (0, 0, 20), (50, 7, 40)])
def test_random_sharing(n, m, window, sinks, room, seed):
    """Any sharing, in one workgroup and in several launches; enough pages, and too few."""
    rng = random.Random(seed)
    page, width = 16, 7
    n_pages = n * width + rng.choice([0, 3, m * width])
    lens, table, refs = shared_batch(rng, n, page, n_pages, width)
    parent = [rng.choice([i % n, rng.randrange(n), rng.randrange(n), -1]) for i in range(m)]
    check(lens, table, parent, refs, page, layers(torch.Generator().manual_seed(seed), n_pages, page, KINDS), window, sinks, room)


def test_both_holders_of_a_page_copy_it():
    """Two rows that end in one page and a third one's whole page: each heir has a copy, and the page, which nobody holds
    then or the third row, is none of those given out."""
    for third in ([], [32]):
        lens, table = [20, 25, *third], [[0, 1, -1], [2, 1, -1], [3, 1, -1]][:2 + len(third)]
        refs = [1, 2 + len(third), 1, len(third), 0, 0]
        made = layers(torch.Generator().manual_seed(2), 6, 16, KINDS)
        want = check(lens, table, list(range(len(lens))), refs, 16, made)
        assert want[2][1] == len(third)
        # with a single free page the second one's copy is not to be had
        want = check(lens, table, [1, 0, 2][:len(lens)], refs[:3] + [1, 0, 1], 16, made)
        assert want[3] == 1 and -1 in want[1][1][:2]


@pytest.mark.parametrize("rows", [1, 100])
def test_counts_in_place(rows):
    """The C call with refs_out = refs: the counts before the step decide."""
    from paper_2609_17184_amd import binding as B
    n, page = 2 * rows, 16
    lens, table = [20, 32] * rows, [[3 * (b // 2), 3 * (b // 2) + 1] for b in range(n)]
    n_pages = 3 * rows
    refs = [2 if x % 3 < 2 else 0 for x in range(n_pages)]
    parent = list(range(n))
    made = layers(torch.Generator().manual_seed(9), n_pages, page, KINDS[:1])
    want = reference(lens, table, parent, refs, page, 0, 0, 0)
    after = copied(made, want[4])
    d = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, table, parent, refs)]
    out = [torch.empty(s, dtype=torch.int32, device=DEV) for s in ((n,), (n, 2), (1,))]
    a = B.ForkArgs(n, n, page, n_pages, d[0].data_ptr(), d[1].data_ptr(), 2, 2, d[2].data_ptr(), d[3].data_ptr(), 0, 0, 0, 0,
                   out[0].data_ptr(), out[1].data_ptr(), 2, d[3].data_ptr(), out[2].data_ptr())
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    caches = (B.PagedCacheC * 1)(made[0][0]._c)
    rc = B.load_library().loopspec_fork_pages(ctypes.byref(a), caches, None, 1, ws.data_ptr(), 1 << 16, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and [t.tolist() for t in (out[0], out[1], d[3], out[2])] == [*want[:3], [want[3]]]
    assert all(torch.equal(t.cpu(), b) for t, b in zip(made[0][1], after))
    assert want[3] == 0 and want[2] == [2 if x % 3 == 0 else 1 for x in range(n_pages)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("cut", [5, 16, 21, 33])
def test_a_rejected_draft(cut, eight):
    """A row is forked at a page's end, one of the two loses its last tokens, is forked again at the shorter length and goes
    on: the other one's attention stays as it was, bit for bit, and its own is that of a row that was never shared."""
    from paper_2609_17184_amd import serving
    G, D, page, n, width = 2, 64, 16, 48, 6
    g = torch.Generator().manual_seed(3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)

    def cache():
        k, v = (torch.zeros((20, G, page, D), dtype=torch.uint8 if eight else torch.bfloat16, device=DEV) for _ in range(2))
        if not eight:
            return serving.PagedCache(k, v)
        s = [torch.full((20, G, 1), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2)]
        return serving.QuantizedCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), *s)
    draw = lambda m, heads: torch.randn((m, heads, D), generator=g).to(torch.bfloat16).to(DEV)
    old, new, q = [draw(n, 4), draw(n, G), draw(n, G)], [draw(20, 4), draw(20, G), draw(20, G)], draw(2, 4)

    def append(c, x, lens, table, starts):
        serving.rope_append(*x, c, serving.Batch(lens, table, i32(starts)))
    c = cache()
    start = serving.fork_pages(i32([0]), torch.full((1, width), -1, dtype=torch.int32, device=DEV), i32([0]), i32([0] * 20), [c], room=n)
    append(c, old, start[0] + n, start[1], [0, n])
    lens, table, refs, _ = serving.fork_pages(start[0] + n, start[1], i32([0, 0]), start[2], [c])
    before = serving.window_attention(q, c, serving.Batch(lens, table))
    lens[0] -= cut
    lens, table, refs, short = serving.fork_pages(lens, table, i32([0, 1]), refs, [c], room=20)
    assert short.item() == 0
    lens[0] += 20
    append(c, new, lens, table, [0, 20, 20])
    after = serving.window_attention(q, c, serving.Batch(lens, table))
    assert torch.equal(after[1], before[1])
    alone = cache()
    row = i32([[7, 3, 5, 11, 2, 9]])
    append(alone, old, i32([n]), row, [0, n])
    append(alone, new, i32([n - cut + 20]), row, [0, 20])
    assert torch.equal(serving.window_attention(q[:1], alone, serving.Batch(i32([n - cut + 20]), row))[0], after[0])
