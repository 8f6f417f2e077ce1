"""Each way through the latent attention: inputs that name the keys which went into a row, and the size of the error over
all of a request's rows, which a lost or doubled range of keys does not pass at any length."""
import numpy as np
import pytest
import torch

from latent_shapes import ROUTES
from latent_util import LATENT, ROW, Shared, absorbed, assert_close, attend, expanded, relative_error
from oracle.efim_oracle import bf16_to_f64, f64_to_bf16
from paper_2505_21889_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


def _marks(longest, columns):
    """Rows whose value marks the range of 32 keys in `columns` - 32 columns, and the key's place in it in 32 others."""
    at, rows = np.arange(longest), np.zeros((longest, ROW), np.uint16)
    rows[at, at // 32 % (columns - 32)] = 0x3F80
    rows[at, columns - 32 + at % 32] = 0x3F80
    return rows


def _shares(visible, columns):
    """Under equal weights: what part of the keys in front of `visible` has each mark."""
    at = np.arange(visible.max())
    upto = np.zeros((visible.max() + 1, columns))
    upto[at + 1, at // 32 % (columns - 32)] += 1
    upto[at + 1, columns - 32 + at % 32] += 1
    return np.cumsum(upto, 0)[visible] / visible[:, None]


def _counts(got_bits, visible, columns):
    """Weights are 1 and their sums exact; an output rounds once to bf16, 2^-8 at most, where it was split a binary16 value of each
    part as well, 2^-11 and a quotient in fp32.  A range lost is all of its mark, or half of it where two have the same."""
    got, want = bf16_to_f64(got_bits), _shares(visible, columns)[:, None]
    assert np.all(np.abs(got[..., :columns] - want) <= 2.0 ** -7 * want)
    assert np.all(got[..., columns:] == 0)


@pytest.mark.parametrize("name", ROUTES)
def test_absorbed_takes_every_key_once(E, name):
    heads, cached, new = ROUTES[name][:3]
    b = Shared(cached, new, _marks(max(np.add(cached, new)), LATENT), 1)
    _counts(absorbed(E, b, np.zeros((b.total, heads, ROW), np.uint16)), b.visible(), LATENT)


# Errors of the rows' norm: the output's rounding to bf16 and that of the weights, each 1.7e-3 of a number in the mean (2^-8 at most,
# evenly spread over a factor of two), with signs of their own: 2.4e-3 together; the bound is twice that.
BOUND = 5e-3


@pytest.mark.parametrize("name", ROUTES)
def test_absorbed_norm_of_the_error(E, name):
    heads, cached, new = ROUTES[name][:3]
    rng = np.random.default_rng(5)
    rows = W.gaussian_bf16(rng, (max(np.add(cached, new)), ROW), 1.0)
    b = Shared(cached, new, rows, 2)
    q = W.gaussian_bf16(rng, (b.total, heads, ROW), 1.0)
    got = absorbed(E, b, q).reshape(-1, LATENT)
    assert np.array_equal(got, absorbed(E, b, q).reshape(-1, LATENT)), "the same call gives the same bits"
    rows64, q64, seen = bf16_to_f64(rows), q.reshape(-1, ROW), np.repeat(b.visible(), heads)
    ends = np.cumsum(b.new) * heads
    for r in sorted({0, 1, len(new) // 2, len(new) - 1}):
        at = np.arange(ends[r] - new[r] * heads, ends[r])
        # of many rows: the first, the last, those around tiles' ends, and others
        some = at if len(at) <= 300 else np.unique(np.concatenate([at[:40], at[-40:], at[120:136], at[1150:1156], rng.choice(at, 200)]))
        keys = rows64[:b.keys[r]]
        want, size = attend(bf16_to_f64(q64[some]), seen[some], keys, keys[:, :LATENT])
        assert_close(got[some], want, size)
        assert relative_error(got[some], want) <= BOUND


EXPANDED = {  # heads, cached, new: two teams and one to a workgroup (more than 512 tiles of rows)
    "two_teams": (3, [100, 5000], [140, 300]),
    "two_teams_long": (1, [9000], [3]),
    "one_team": (48, [20, 4000], [1500, 130]),
}


@pytest.mark.parametrize("name", EXPANDED)
def test_expanded_takes_every_key_once(E, name):
    heads, cached, new = EXPANDED[name]
    b = Shared(cached, new, _marks(max(np.add(cached, new)), 128), 3)
    w = np.zeros((heads, 256, 512), np.uint16)
    w[:, 128 + np.arange(128), np.arange(128)] = 0x3F80  # values: the marks; keys: nothing
    _counts(expanded(E, b, np.zeros((b.total, heads, 192), np.uint16), w), b.visible(), 128)


@pytest.mark.parametrize("name", EXPANDED)
def test_expanded_norm_of_the_error(E, name):
    heads, cached, new = EXPANDED[name]
    rng = np.random.default_rng(6)
    rows = W.gaussian_bf16(rng, (max(np.add(cached, new)), ROW), 1.0)
    b = Shared(cached, new, rows, 4)
    q, w = W.gaussian_bf16(rng, (b.total, heads, 192), 1.0), W.gaussian_bf16(rng, (heads, 256, 512), 512 ** -0.5)
    got, rows64 = expanded(E, b, q, w), bf16_to_f64(rows)
    start = 0
    for c, n in zip(cached, new):
        some = start + np.unique(np.concatenate([np.arange(min(n, 140)), rng.integers(0, n, 60), [n - 1]]))
        for h in sorted({0, heads // 2, heads - 1}):
            w64 = bf16_to_f64(w[h])
            keep = bf16_to_f64(f64_to_bf16(rows64[:c + n, :LATENT] @ w64.T))
            keys = np.concatenate([keep[:, :128], rows64[:c + n, LATENT:]], 1)
            want, size = attend(bf16_to_f64(q[some, h]), b.visible()[some], keys, keep[:, 128:])
            # (a key that fp32 sums round to the other neighbour moves its scores by 2^-8 of one product: 2e-3 of the values' size)
            assert_close(got[some, h], want, size, more=2e-3)
            assert relative_error(got[some, h], want) <= BOUND
        start += n
