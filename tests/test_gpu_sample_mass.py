"""Draws that are decided by weights as exact as 64 bits give them: equal logits, whose weights are equal numbers, and
close logits far from zero at low temperatures."""
import numpy as np
import pytest
import torch

from test_gpu_serving_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2, 4, 10, 64, 1000, 4096, 6000, 16384])
@pytest.mark.parametrize("spread", [False, True])
def test_equal_logits_at_the_border(n, spread):
    """n equal logits of all sizes, one after the other or over several shards, the others -infinity: halves and
    quarters of n as u's and top-p's border, of which a comparison of exact sums is on one side only."""
    V = n if not spread else max(4 * n, 3 * 4096 + 5)
    at = np.arange(n) if not spread else np.sort(np.random.default_rng(n).permutation(V)[:n])
    rows = np.float32([0.0, 0.3, -1.7, 5.1, 11.3, -23.9, 100.7, 1e-3, 777.7, 0.1])
    z = np.full((len(rows), V), -np.inf, np.float32)
    z[:, at] = rows[:, None]
    quarter = 0.25 if n % 4 == 0 else 0.5
    for t in (1.0, 0.7, 1e-4):
        for u in (0.5, quarter, 0.0):
            for k, p, m in [(0, 1.0, 0.0), (0, 0.5, 0.0), (0, quarter, 0.0), (0, 1.0, 1.0), (n // 2, 1.0, 0.0), (n - n % 2, 0.5, 0.0)]:
                check(torch.tensor(z), np.full(len(rows), u), t, k, p, m)


def test_close_logits_far_from_zero():
    """Neighbouring fp32 numbers near 1000 at T = 2e-5, three natural units apart, in two shards: u at every border of
    the kept masses, 2^-34 of it to either side (weights are off by 2^-36 of themselves)."""
    rng = np.random.default_rng(9)
    V, T = 5000, np.float32(2e-5)
    ids = np.array([3, 4, 700, 2000, 4095, 4096, 4500, 4999])
    zs, us = [], []
    for turn in range(12):
        step = np.spacing(np.float32(1000.0))
        z = np.full(V, -np.inf, np.float32)
        z[ids] = np.float32(1000.0 + turn * 1.37) + step * rng.integers(0, 3, len(ids)).astype(np.float32)
        w = np.exp((z[ids].astype(np.float64) - z.max()) / np.float64(T))
        cum = np.cumsum(w) / w.sum()
        for c in cum[:-1]:
            for side in (-1, 1):
                zs.append(z)
                us.append(c * (1 + side * 2.0 ** -34))
    z = torch.tensor(np.stack(zs))
    for k, p in ((0, 1.0), (len(ids), 1.0), (0, 0.9999999)):
        check(z, np.array(us), float(T), k, p, 0.0)
