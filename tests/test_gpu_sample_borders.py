"""Draws whose answer hangs on an exact border, against the plain 64-bit implementation."""
import numpy as np
import pytest
import torch

from test_gpu_serving_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k,p", [(0, 1.0), (3, 1.0), (0, 0.4), (4, 0.9)])
def test_min_p_of_one(k, p):
    """min_p = 1 keeps the largest logits alone, also where they lie just below a half octave."""
    rng = np.random.default_rng(8)
    tops = [2.0794413, 2.4260149, 2.7725885, 3.1190621]
    edges = np.float32(np.arange(-40, 60) * (np.log(2) / 2))
    for step in (-np.inf, np.inf):
        tops += edges.tolist() + np.nextafter(edges, np.float32(step)).tolist()
    tops = np.float32(tops)
    z = tops[:, None] - rng.uniform(0.01, 3, (len(tops), 400)).astype(np.float32)
    z[:, [7, 150, 151]] = tops[:, None]
    check(torch.tensor(z), rng.random(len(z)), 1.0, k, p, 1.0)
    check(torch.tensor(z), rng.random(len(z)), 1.0, k, p, 0.5)
