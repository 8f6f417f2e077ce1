"""Batches over a 4-bit cache of which every launch of a class cuts tiles, so that partial results of one launch lie where those of the
launch in front of it lay (`test_mx4_launches.py` holds them to that)."""
import numpy as np

#: requests of few query rows: name -> (heads, new tokens of a request, up to, head dim); 2.x launches of 120
FEW = {"16 rows": ((4, 1), 4, 128), "32 rows": ((8, 1), 4, 128), "32 rows, head dim 64": ((4, 1), 8, 64)}


def few(name):
    """(cached, new, heads, head dim): 250 requests of about a thousand keys."""
    heads, most, d = FEW[name]
    rng = np.random.default_rng(most + d)
    cached, new = rng.integers(700, 1000, 250), rng.integers(1, most + 1, 250)
    new[[0, 100, 130, 245]] = most
    return cached, new, heads, d


def many():
    """(cached, new, heads): 140 requests of more than 32 query rows and about 3000 keys, one launch of 96 of them and one of the others,
    and 130 of few rows between them."""
    rng = np.random.default_rng(9)
    cached, new = rng.integers(2500, 3300, 270), rng.integers(17, 40, 270)
    few = rng.permutation(270)[:130]
    cached[few], new[few] = rng.integers(500, 1300, 130), rng.integers(0, 4, 130)
    return cached, new, (2, 1)
