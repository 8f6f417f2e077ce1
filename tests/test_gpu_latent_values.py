"""The latent attention on values at the ends of bf16."""
import numpy as np
import pytest
import torch

from latent_shapes import ROUTES
from latent_util import LATENT, ROW, Shared, absorbed
from oracle.efim_oracle import bf16_to_f64, f64_to_bf16
from paper_2505_21889_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


@pytest.mark.parametrize("name", ["rows16", "rows32", "rows32_two_waves", "rows128"])
@pytest.mark.parametrize("size", [1e-30, 1e-35, 3e-37])
def test_absorbed_values_near_the_least_number(E, name, size):
    """Equal weights over values between `size` and twice that: their mean, down to where bf16's and fp32's normal numbers end."""
    heads, cached, new = ROUTES[name][:3]
    rng = np.random.default_rng(7)
    rows = f64_to_bf16((1.0 + rng.random((max(np.add(cached, new)), ROW))) * size)
    b = Shared(cached, new, rows, 8)
    got = bf16_to_f64(absorbed(E, b, W.gaussian_bf16(rng, (b.total, heads, ROW), 1.0)))
    values = bf16_to_f64(rows)[:, :LATENT]
    want = (np.cumsum(values, 0) / np.arange(1, len(values) + 1)[:, None])[b.visible() - 1]  # (scores below 1e-27 are zero)
    assert np.all(np.abs(got - want[:, None]) <= 2.0 ** -7 * want[:, None])
