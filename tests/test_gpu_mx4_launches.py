"""The attention over a 4-bit cache where a class takes several launches, all of which have parts to join."""
import numpy as np
import pytest

import mx4_batches as B
import mx4_util as X
from test_gpu_mx4 import E, _attend, _check  # noqa: F401 (E is a fixture)

pytestmark = pytest.mark.gpu


def _step(cached, new, heads, d, page=16, seed=0):
    """Caches of random codes and scales (in the slots of no row too)."""
    s = X.Step(cached, new, heads, d, page, seed=seed, filled=False)
    rng = np.random.default_rng(seed + 1)
    for cache in s.caches:
        cache[..., :page * (d // 2)] = rng.integers(0, 256, cache.shape[:-1] + (page * (d // 2),), dtype=np.uint8)
        cache[..., page * (d // 2):] = rng.integers(123, 127, cache.shape[:-1] + (page * (d // 32),), dtype=np.uint8)
    return s


@pytest.mark.parametrize("name", B.FEW)
def test_launches_of_few_rows(E, name):  # noqa: F811
    cached, new, heads, d = B.few(name)
    _check(E, _step(cached, new, heads, d, seed=1))


@pytest.mark.parametrize("d,page", [(128, 16), (64, 32)])
def test_launches_of_many_rows(E, d, page):  # noqa: F811
    """One in shares that end inside tiles, one in whole longer units; few rows between them."""
    cached, new, heads = B.many()
    s = _step(cached, new, heads, d, page, seed=2)
    _check(E, s)
    first = _attend(E, s)
    assert np.array_equal(first, _attend(E, s))
