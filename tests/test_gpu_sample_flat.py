"""Draws from flat rows of a large vocabulary against the plain 64-bit implementation."""
import numpy as np
import pytest
import torch

from test_gpu_serving_sample import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,p", [(1.25, 0.95), (2.0, 0.9), (1.6, 0.99)])
def test_flat_rows_of_a_large_vocabulary(t, p):
    """Normal logits at high temperatures, whose boundary lists thousands (over 8192 at the second)."""
    rng = np.random.default_rng(10)
    z = torch.tensor(rng.standard_normal((3, 131072)) * 2.5).float()
    check(z, rng.random(3), t, 0, p, 0.0)
    check(z, rng.random(3), t, 60000, p, 1e-5)
