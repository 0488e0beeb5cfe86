"""Draws from logits on the GPU against a plain 64-bit implementation, row by row: tokens and kept counts equal,
probabilities within fp32's rounding."""
import math

import numpy as np
import pytest
import torch

from gpu_common import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def draw(z, u, t, k, p, m):
    """(token, probability, kept) of one row in 64 bits."""
    z = z.astype(np.float64)
    if np.isnan(z).any() or z.max() == np.inf or z.max() == -np.inf:
        return -1, 0.0, 0
    if not (0 <= t < np.inf and 0 < p <= 1 and 0 <= m <= 1 and 0 <= u < 1):
        return -1, 0.0, 0
    if t == 0:
        return int(z.argmax()), 1.0, 1
    w = np.exp((z - z.max()) / t)
    order = np.argsort(-z, kind="stable")
    order = order[np.isfinite(z[order])]
    if k > 0:
        order = order[:k]
    if p < 1:
        cum = np.cumsum(w[order])
        order = order[(cum - w[order]) < p * cum[-1]]
    order = np.sort(order[w[order] >= m])
    cum = np.cumsum(w[order])
    i = min(int(np.searchsorted(cum, u * cum[-1], side="right")), len(order) - 1)
    return int(order[i]), w[order[i]] / cum[-1], len(order)


def check(z, u, t, k, p, m):
    """Runs the batch and compares every row.  A weight is off by 2^-38.8 of itself, in a bin's sum by 2^-37 more, in
    the list's by 2^-45 of the row's largest weight, of which there are at most V <= 2^18: sums are off by 2^-27 of
    themselves (none is smaller than the largest weight), a probability by 2^-26 and fp32's half step."""
    from paper_2609_17184_amd import serving
    rows = len(z)

    def dev(x, kind):
        return torch.tensor(x, dtype=kind, device=DEV) if np.ndim(x) else x
    got = serving.sample(z.to(DEV), torch.tensor(u, dtype=torch.float64, device=DEV), dev(t, torch.float32),
                         dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32))
    token, prob, kept = (x.cpu().numpy() for x in got)
    zz = z.float().numpy()
    f32 = lambda x: np.broadcast_to(np.float32(x).astype(np.float64), (rows,))
    ref = [draw(*a) for a in zip(zz, u, f32(t), np.broadcast_to(k, (rows,)), f32(p), f32(m))]
    assert token.tolist() == [r[0] for r in ref]
    assert kept.tolist() == [r[2] for r in ref]
    err = np.abs(prob - np.array([r[1] for r in ref]))
    assert (err <= 2.0 ** -26 + 2.0 ** -24 * prob).all(), err.max()
    return ref


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 50, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (0.9, 200, 0.8, 0.01),
            (2.5, 0, 0.99, 0.0), (0.0, 5, 0.5, 0.5), (0.05, 0, 0.95, 0.0), (1.0, 1, 1.0, 0.0), (30.0, 0, 0.6, 0.0),
            (1.0, 0, 1e-6, 0.0), (1.0, 0, 1.0, 1.0), (1.0, 100000, 1.0, 0.0)]


@pytest.mark.parametrize("V", [1, 2, 63, 64, 1001, 4096, 49152, 130003, 262144])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_sizes(V, dtype):
    """Every combination of filters at every size, normal logits with a few peaks (16-bit types: many ties)."""
    rng = np.random.default_rng(V)
    rows = len(SETTINGS)
    z = rng.standard_normal((rows, V)) * 2.5
    z[:, rng.integers(0, V, 5)] += 6
    t, k, p, m = (np.array(x) for x in zip(*SETTINGS))
    ref = check(torch.tensor(z).to(DT[dtype]), rng.random(rows), t, k.astype(np.int32), p, m)
    log(f"[sample] V={V} {dtype}: kept {[r[2] for r in ref]}")


@pytest.mark.parametrize("setting", SETTINGS, ids=str)
def test_settings_for_all_rows(setting):
    """Numbers instead of tensors, many uniform numbers with the ends of the range, rows that share their logits."""
    rng = np.random.default_rng(1)
    z = (torch.tensor(rng.standard_normal(777)) * 3).float()
    u = np.concatenate([[0.0, 1 - 2.0 ** -53, 0.5, 2.0 ** -53], rng.random(300)])
    check(z[None].expand(len(u), -1), u, *setting)


def test_ties():
    """Equal logits: the cuts fall among them by id."""
    rng = np.random.default_rng(2)
    V = 5000
    z = np.zeros((6, V))
    z[1, ::3] = 1.0
    z[2] = np.round(rng.standard_normal(V))
    z[3] = -0.0
    z[3, ::2] = 0.0
    z[4, 17] = 8.0
    z[5] = np.where(rng.random(V) < 0.5, -np.inf, 2.0)
    for t, k, p, m in [(1.0, 700, 1.0, 0.0), (1.0, 0, 0.2999, 0.0), (0.5, 2500, 0.6001, 0.0), (1.0, 0, 1.0, 0.4)]:
        check(torch.tensor(z).float(), rng.random(6), t, k, p, m)


def test_wide_spread_and_odd_values():
    """Keys that need every round of the search: tiny differences, both signs, denormals, values near the ends of the
    type, geometric spacing."""
    rng = np.random.default_rng(3)
    V = 9001
    z = np.stack([1.0 + rng.random(V) * 1e-5, rng.standard_normal(V) * 1e-30, rng.standard_normal(V) * 1e-42,
                  rng.standard_normal(V) * 5e37, np.exp(rng.uniform(-80, 80, V)) * rng.choice([-1, 1], V),
                  rng.integers(-3, 3, V) + rng.random(V) * 1e-6, np.full(V, -3e38)]).astype(np.float32)
    for t, k, p, m in [(1.0, 3000, 1.0, 0.0), (1.0, 0, 0.7, 0.0), (1.0, 7000, 0.5, 0.0), (1e-30, 100, 1.0, 0.0),
                       (1e30, 4000, 0.9, 0.0), (1e-42, 0, 0.9, 0.0)]:
        check(torch.tensor(z), rng.random(len(z)), t, k, p, m)


@pytest.mark.parametrize("low", [-24.3, -27.7, -29.9, -40.0])
def test_flat_tail(low):
    """One logit and a vocabulary of equal ones far below, whose mass only counts together: the kept mass is top_p's
    within 2^-26 of the whole (sums are off by 2^-27), and no tie more than that."""
    from paper_2609_17184_amd import serving
    V = 262144
    p = np.float32(1 - 2.0 ** -24)
    z = torch.full((2, V), low)
    z[:, 100000] = 0.0
    w = math.exp(low)
    whole = 1 + (V - 1) * w
    token, prob, kept = serving.sample(z.to(DEV), torch.tensor([0.5, 0.9], dtype=torch.float64, device=DEV), 1.0, 0, float(p))
    assert token.tolist() == [100000] * 2
    for k, pr in zip(kept.tolist(), prob.tolist()):
        mass, before = 1 + (k - 1) * w, 1 + (k - 2) * w if k > 1 else 0.0     # with and without the last kept rank
        assert mass >= (float(p) - 2.0 ** -26) * whole and before < (float(p) + 2.0 ** -26) * whole
        assert abs(pr - 1 / mass) <= 2.0 ** -26 + 2.0 ** -24


def test_masked_rows():
    """-infinity is never kept; rows that cannot be drawn from give -1 and leave the others alone."""
    rng = np.random.default_rng(4)
    V = 3000
    z = rng.standard_normal((9, V)).astype(np.float32)
    z[0, 5:] = -np.inf
    z[1] = -np.inf
    z[2, 77] = np.nan
    z[3, V - 1] = np.inf
    z[4, :-1] = -np.inf
    z[5, ::2] = -np.inf
    z[6] = np.finfo(np.float32).min
    z[6, 100] = 0
    z[7, :] = np.finfo(np.float32).min
    for t, k, p, m in [(1.0, 0, 1.0, 0.0), (1.0, 10, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0)]:
        ref = check(torch.tensor(z), rng.random(9), t, k, p, m)
        assert [r[0] for r in ref[1:4]] == [-1] * 3


def test_settings_out_of_range():
    nan, inf = float("nan"), float("inf")
    t = np.array([-1.0, nan, inf, 1, 1, 1, 1, 1, 1, 1, 1, 1], np.float32)
    p = np.array([1, 1, 1, 0.0, -1, 1.5, nan, 1, 1, 1, 1, 1], np.float32)
    m = np.array([0, 0, 0, 0, 0, 0, 0, -0.1, 1.1, nan, 0, 0], np.float32)
    u = np.array([0.5] * 10 + [1.0, nan])
    rng = np.random.default_rng(5)
    check(torch.tensor(rng.standard_normal((12, 500))).float(), u, t, 0, p, m)


def test_strided_rows_and_one_missing_alignment():
    rng = np.random.default_rng(6)
    for dtype in DT:
        big = torch.tensor(rng.standard_normal((40, 1111)) * 3).to(DT[dtype])
        for off in (0, 1, 2, 3):
            check(big[:, off:1003 + off], rng.random(40), 0.9, 0, 0.95, 0.0)
            check(big[::2, off:1003 + off], rng.random(20), 1.0, 30, 1.0, 0.0)


def test_repeatable_and_independent_of_the_batch():
    from paper_2609_17184_amd import serving
    g = torch.Generator(device=DEV).manual_seed(0)
    z = torch.randn((300, 49152), generator=g, device=DEV) * 3
    u = torch.rand(300, generator=g, device=DEV, dtype=torch.float64)
    a = serving.sample(z, u, 0.9, 0, 0.95, 0.0)
    b = serving.sample(z, u, 0.9, 0, 0.95, 0.0)
    c = [torch.cat(x) for x in zip(*(serving.sample(z[i:i + 1], u[i:i + 1], 0.9, 0, 0.95, 0.0) for i in range(300)))]
    for x, y, w in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, w)


def test_law_of_the_draws():
    """40000 draws of a filtered distribution: chi-square with 99.9 % of its law below the bound."""
    from paper_2609_17184_amd import serving
    rng = np.random.default_rng(7)
    z = torch.tensor(rng.standard_normal(200) * 1.5).float()
    n = 40000
    u = rng.random(n)
    tok = serving.sample(z.to(DEV)[None].expand(n, -1), torch.tensor(u, device=DEV), 1.0, 20, 1.0, 0.0)[0].cpu().numpy()
    w = np.exp(z.double().numpy())
    keep = np.argsort(-w)[:20]
    exp = w[keep] / w[keep].sum() * n
    got = np.array([(tok == i).sum() for i in keep])
    assert got.sum() == n
    chi = ((got - exp) ** 2 / exp).sum()
    assert chi < 43.82, chi                    # 19 degrees of freedom


def test_captured_draw_follows_its_inputs():
    from paper_2609_17184_amd import serving
    rows, V = 6, 20011
    z = torch.randn((rows, V), device=DEV).to(torch.bfloat16)
    u = torch.rand(rows, device=DEV, dtype=torch.float64)
    top_p = torch.full((rows,), 0.9, device=DEV)
    call = lambda: serving.sample(z, u, 0.8, 100, top_p, 0.001)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for turn in range(4):
        z.normal_()
        u.uniform_()
        top_p.uniform_(0.3, 1.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, call()):
            assert torch.equal(a, b)
