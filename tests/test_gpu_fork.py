"""Forks of a batch's pages against a plain implementation on the host."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference(lens, table, parent, refs, n_pages, page, prefix, window, sinks, room, width=0):
    """(lens, table, refs, short, copies): copies lists (child, source page, page, positions)."""
    width, refs = len(table[0]) if table else width, list(refs)
    ok = lambda x: 0 <= x < n_pages
    for n, row in zip(lens, table):
        if n >= 0:
            for x in row:
                if ok(x):
                    refs[x] -= 1
    out, heirs, wants, short = [], set(), [], 0
    for j, p in enumerate(parent):
        row = [-1] * width
        if 0 <= p < len(lens) and lens[p] >= 0:
            n, heir = lens[p], p not in heirs
            heirs.add(p)
            held = min(-(-n // page), width)
            need = -(-(min(n, width * page) + room) // page) if room else held
            for i in range(width):
                first = prefix + i * page
                gone = window and first + page - 1 <= prefix + n - window and first >= sinks
                if ok(table[p][i]) and not gone and (heir or (i + 1) * page <= n):
                    row[i] = table[p][i]
                elif not heir and (i + 1) * page > n and i < held:
                    if ok(table[p][i]):
                        wants.append((j, i, table[p][i], n % page))
                elif held <= i < need and (not heir or not ok(table[p][i])):
                    wants.append((j, i, -1, 0))
            short += max(0, need - width)
            out.append((n, row))
        else:
            out.append((-1, row))
        for x in row:
            if ok(x):
                refs[x] += 1
    free = [x for x in range(n_pages) if refs[x] == 0]
    copies = []
    for (j, i, source, n), x in zip(wants, free):
        out[j][1][i], refs[x] = x, 1
        if source >= 0:
            copies.append((source, x, n))
    return [n for n, _ in out], [r for _, r in out], refs, short + max(0, len(wants) - len(free)), copies


def batch(rng, n, page, n_pages, width, most, shared=True, ahead=0):
    """Rows of random lengths whose pages are their own, but for common first ones; some rows are no sequence."""
    pages = list(range(n_pages))
    rng.shuffle(pages)
    lens, table = [], []
    for b in range(n):
        length = rng.choice([-1, 0, page, rng.randint(0, most), rng.randint(0, most), rng.randint(0, most)])
        row = [rng.choice([-1, -7, n_pages])] * width
        held = min(-(-max(length, 0) // page) + rng.randint(0, ahead), width)
        row[:held] = [pages.pop() for _ in range(held)]
        if shared and b and lens[-1] >= 0 and length > 0:
            k = rng.randint(0, min(length, lens[-1]) // page)
            row[:k] = table[-1][:k]
        lens.append(length)
        table.append(row)
    refs = [0] * n_pages
    for length, row in zip(lens, table):
        for x in row:
            if length >= 0 and 0 <= x < n_pages:
                refs[x] += 1
    return lens, table, refs


def layers(g, n_pages, page, kinds):
    """Caches of given (bits, heads, head_dim, heads first)."""
    from paper_2609_17184_amd import serving
    made = []
    for bits, G, D, heads_first in kinds:
        shape = (n_pages, G, page, D) if heads_first else (n_pages, page, G, D)
        raw = [torch.randint(0, 256, (*shape[:3], shape[3] * bits // 8), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
        k, v = (t.view(torch.float8_e4m3fn if bits == 8 else torch.float16) for t in raw)
        if not heads_first:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        if bits == 8:
            s = [torch.randint(0, 256, (n_pages, G, page // 16), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
            made.append((serving.QuantizedCache(k, v, *(t.view(torch.float8_e8m0fnu) for t in s)), raw, s, heads_first))
        else:
            made.append((serving.PagedCache(k, v), raw, [], heads_first))
    return made


def copied(made, copies):
    """The caches' bytes after the copies, on the host."""
    want = []
    for _, raw, scales, heads_first in made:
        for t in raw:
            t = t.cpu()
            for source, x, n in copies:
                a = (slice(None), slice(n)) if heads_first else (slice(n),)
                t[(x, *a)] = t[(source, *a)]
            want.append(t)
        for t in scales:
            t = t.cpu()
            for source, x, n in copies:
                t[x, :, :-(-n // 16)] = t[source, :, :-(-n // 16)]
            want.append(t)
    return want


def check(lens, table, parent, refs, n_pages, page, made, prefix=0, window=0, sinks=0, room=0, width=None):
    from paper_2609_17184_amd import serving
    dev = lambda x, shape=None: (torch.tensor(x, dtype=torch.int32) if shape is None else torch.tensor(x, dtype=torch.int32).view(shape)).to(DEV)
    width = len(table[0]) if table else width
    wide = torch.full((len(lens), width + 2), 5, dtype=torch.int32, device=DEV)
    wide[:, :width] = dev(table, (len(lens), width))
    want = reference(lens, table, parent, refs, n_pages, page, prefix, window, sinks, room, width)
    bytes_after = copied(made, want[4])
    given = dev(refs)
    got = serving.fork_pages(dev(lens, (len(lens),)), wide[:, :width], dev(parent, (len(parent),)), given, [m[0] for m in made],
                             prefix, window, sinks, room)
    assert got[0].tolist() == want[0]
    assert got[1].tolist() == want[1]
    assert got[2].tolist() == want[2] and given.tolist() == refs
    assert got[3].tolist() == [want[3]]
    now = [t.cpu() for _, raw, scales, _ in made for t in raw + scales]
    assert all(torch.equal(a, b) for a, b in zip(now, bytes_after))
    return got, want


KINDS = [(16, 2, 64, True), (8, 3, 96, True), (8, 2, 16, False), (16, 1, 128, False)]


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("window,sinks,room", [(0, 0, 0), (40, 5, 0), (1, 0, 7), (100, 20, 100), (0, 0, 33)])
def test_random_batches(window, sinks, room, seed):
    rng = random.Random(seed)
    page = rng.choice([16, 32, 48, 128])
    n, m, width = rng.randint(1, 40), rng.randint(1, 60), 12
    n_pages = n * (width + 2) + rng.choice([0, 3, 400])
    lens, table, refs = batch(rng, n, page, n_pages, width, page * (width - 2), ahead=2)
    parent = [rng.choice([rng.randrange(n), rng.randrange(n), rng.randrange(n), -1, n]) for _ in range(m)]
    check(lens, table, parent, refs, n_pages, page, layers(torch.Generator().manual_seed(seed), n_pages, page, KINDS),
          rng.choice([0, 21]), window, sinks, room)


@pytest.mark.parametrize("n,m", [(1, 1), (1, 300), (300, 1), (700, 600)])
def test_row_counts(n, m):
    rng = random.Random(n + m)
    lens, table, refs = batch(rng, n, 16, 5000, 6, 90)
    parent = [rng.randrange(n) for _ in range(m)]
    check(lens, table, parent, refs, 5000, 16, layers(torch.Generator().manual_seed(1), 5000, 16, KINDS[2:3]), room=5)


def test_short_pools():
    """Fewer free pages than wanted, none at all, and tables without room: counted, and -1 in the table."""
    rng = random.Random(3)
    for spare in (0, 1, 5):
        n_pages = 3 * 3 + spare
        lens, table = [40, 33, 48], [[0, 1, 2], [3, 4, 5], [6, 7, 8]]
        refs = [1] * 9 + [0] * spare
        made = layers(torch.Generator().manual_seed(2), n_pages, 16, KINDS[:2])
        (_, _, _, short), _ = check(lens, table, [0, 0, 0, 1, 1, 2], refs, n_pages, 16, made, room=16)
        assert short.item() > 0
        # without the second row's children its pages are there for the others
        check(lens, table, [0, 0, 0, 2, 2], refs, n_pages, 16, made)


def test_pages_of_a_window_run_dry():
    """Many steps of one batch: pages are taken as rows grow and given back behind the window; no page is lost."""
    from paper_2609_17184_amd import serving
    rng = random.Random(4)
    n_pages, page, width = 60, 16, 30
    made = layers(torch.Generator().manual_seed(3), n_pages, page, KINDS[1:2])
    lens, table, refs = [0, 0, 0], [[-1] * width for _ in range(3)], [0] * n_pages
    for step in range(40):
        parent = [0, 1, 2] if step % 7 else [rng.randrange(3) for _ in range(3)]
        got, want = check(lens, table, parent, refs, n_pages, page, made, window=50, sinks=10, room=11)
        assert want[3] == 0
        lens, table, refs = [n + 11 for n in want[0]], want[1], want[2]
        assert sum(refs) == sum(x >= 0 for row in table for x in row)


def test_counts_of_the_caller_keep_pages():
    """Pages that the caller counts for itself (a prefix's) are neither given out nor let go."""
    made = layers(torch.Generator().manual_seed(5), 12, 16, KINDS[:1])
    refs = [1, 1, 0, 0, 3, 2, 0, 0, 0, 1, 0, 1]                         # 4: twice more than by the table, 9 and 11: by no row
    check([20, 40], [[0, 1, -1], [4, 5, 5]], [1, 1, 5], refs, 12, 16, made)


def test_large_pages_and_many_caches():
    """Pages of 1008 positions and more caches than a launch describes."""
    rng = random.Random(5)
    kinds = [KINDS[i % 4] for i in range(19)]
    lens, table, refs = batch(rng, 3, 1008, 8, 2, 2016, shared=False)
    lens[0], table[0][0:2], refs = 1500, [6, 7], [0] * 8
    for length, row in zip(lens, table):
        for x in row:
            if length >= 0 and 0 <= x < 8:
                refs[x] += 1
    check(lens, table, [0, 0, 2], refs, 8, 1008, layers(torch.Generator().manual_seed(6), 8, 1008, kinds))


def test_empty_batches_and_refusals():
    from paper_2609_17184_amd import serving
    made = layers(torch.Generator().manual_seed(5), 6, 16, KINDS[:2])
    check([20, 5], [[0, 1], [2, -1]], [], [1, 1, 1, 0, 0, 4], 6, 16, made)          # all rows end
    check([], [], [0, -1], [0] * 6, 6, 16, made, width=3)                          # children of nobody
    caches = [m[0] for m in made]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    lens, table, parent, refs = i32(20, 5), i32(0, 1, 2, 3).view(2, 2), i32(0, 0), i32(1, 1, 1, 1, 0, 0)
    other = layers(torch.Generator().manual_seed(5), 7, 16, KINDS[:1])[0][0]
    for args in ((lens, table, parent, refs, []), (lens, table, parent, refs[:5], caches), (lens, table, parent, refs, [caches[0], other]),
                 (lens.long(), table, parent, refs, caches), (lens[:1], table, parent, refs, caches), (lens, table, parent.cpu(), refs, caches),
                 (lens, table[0], parent, refs, caches)):
        with pytest.raises(ValueError):
            serving.fork_pages(*args)
    for kw in (dict(window=-1), dict(sinks=-1), dict(room=-1), dict(prefix_len=-1)):
        with pytest.raises(ValueError):
            serving.fork_pages(lens, table, parent, refs, caches, **kw)
    from paper_2609_17184_amd import LoopSpecError
    with pytest.raises(LoopSpecError):
        serving.fork_pages(lens, table, parent, refs, caches, room=33)              # more than the table holds


def test_captured_forks():
    """A captured fork replayed while its batch changes, against the eager call; two graphs in turn."""
    from paper_2609_17184_amd import serving
    rng = random.Random(8)
    n_pages, page, width, n, m = 200, 32, 8, 6, 9
    work = []
    for s in range(2):
        made = layers(torch.Generator().manual_seed(s), n_pages, page, KINDS)
        dev = [torch.zeros(shape, dtype=torch.int32, device=DEV) for shape in ((n,), (n, width), (m,), (n_pages,))]
        args = (*dev, [x[0] for x in made], 3, 70, 9, 20)
        serving.fork_pages(*args)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = serving.fork_pages(*args)
        work.append((made, dev, args, graph, out))
    for turn in range(4):
        want = []
        for made, dev, args, graph, out in work:
            lens, table, refs = batch(rng, n, page, n_pages, width, 200)
            for d, x in zip(dev, (lens, table, [rng.randrange(n) for _ in range(m)], refs)):
                d.copy_(torch.tensor(x, dtype=torch.int32))
            ref = reference(lens, table, dev[2].tolist(), refs, n_pages, page, 3, 70, 9, 20)
            want.append((ref, copied(made, ref[4])))
        torch.cuda.synchronize()
        for w in work:
            w[3].replay()
        torch.cuda.synchronize()
        for (made, _, _, _, out), (ref, after) in zip(work, want):
            assert [t.tolist() for t in out] == [*ref[:3], [ref[3]]]
            assert all(torch.equal(t.cpu(), b) for t, b in zip([t for _, raw, sc, _ in made for t in raw + sc], after))


def test_counts_in_place():
    """The C call with refs_out = refs."""
    import ctypes
    from paper_2609_17184_amd import binding as B
    made = layers(torch.Generator().manual_seed(9), 10, 16, KINDS[:1])
    lens, table, parent, refs = [20, 30], [[0, 1], [2, 3]], [0, 0, 0], [1, 1, 1, 1] + [0] * 6
    want = reference(lens, table, parent, refs, 10, 16, 0, 0, 0, 0)
    d = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, table, parent, refs)]
    out = [torch.empty(s, dtype=torch.int32, device=DEV) for s in ((3,), (3, 2), (1,))]
    a = B.ForkArgs(2, 3, 16, 10, d[0].data_ptr(), d[1].data_ptr(), 2, 2, d[2].data_ptr(), d[3].data_ptr(), 0, 0, 0, 0,
                   out[0].data_ptr(), out[1].data_ptr(), 2, d[3].data_ptr(), out[2].data_ptr())
    ws = torch.empty(1024, dtype=torch.uint8, device=DEV)
    caches = (B.PagedCacheC * 1)(made[0][0]._c)
    rc = B.load_library().loopspec_fork_pages(ctypes.byref(a), caches, None, 1, ws.data_ptr(), 1024, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and [t.tolist() for t in (out[0], out[1], d[3], out[2])] == [*want[:3], [want[3]]]
