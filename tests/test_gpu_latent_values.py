"""The latent attention on values at the ends of bf16: what a row that sees an infinite key gets, by the definition in 64 bits,
wherever the key lies, what a row that does not see it gets, and values so small that their parts' scale is at the end of fp32."""
import numpy as np
import pytest
import torch

from latent_shapes import ROUTES
from latent_util import LATENT, ROW, Shared, absorbed, assert_close, attend, expanded
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


def _places(cached, new):
    """Of request 0: a key of its first range, one in the middle, the last in the cache, and of the new ones the first, the last but
    one and the last."""
    c, n = cached[0], new[0]
    return sorted({3, c // 2, c // 2 + 33, max(c - 1, 0), c, c + n - 2, c + n - 1} & set(range(c + n)))


def _check(got, clean, sees, above, columns, want, size):
    """got, clean, want, size [rows, d]; sees, above [rows]: whether the row sees the infinite key, and has it for its maximum.
    columns: of the values, those that are infinite in the key."""
    assert np.array_equal(got[~sees], clean[~sees]), "rows that do not see the key"
    assert np.all(np.isnan(bf16_to_f64(got[sees & above]))), "infinity less infinity"
    below = sees & ~above
    assert np.all(np.isnan(bf16_to_f64(got[below][:, columns]))), "no weight times infinity"
    others = np.setdiff1d(np.arange(got.shape[1]), columns)
    if len(others) and below.any():
        assert_close(got[below][:, others], want[below][:, others], size[below][:, others])


@pytest.mark.parametrize("column", [7, 300, 530])
@pytest.mark.parametrize("name", ["rows16", "rows32", "rows32_two_waves", "rows128", "rows128_even"])
def test_absorbed_one_infinity_in_a_key(E, name, column):
    """A score of minus infinity is no weight, and no weight times an infinite value is no number: in its column alone."""
    heads, cached, new = ROUTES[name][:3]
    rng = np.random.default_rng(9)
    rows = W.gaussian_bf16(rng, (max(np.add(cached, new)), ROW), 1.0)
    q = W.gaussian_bf16(rng, (sum(new), heads, ROW), 1.0)
    b = Shared(cached, new, rows, 10)
    visible = np.repeat(b.visible(), heads)
    # rows of request 0, and in front of its end those that see its last keys
    at = np.unique(np.concatenate([np.arange(new[0] * heads)[-80:], rng.integers(0, new[0] * heads, 60)]))
    q[:, :, column] = np.where(q[:, :, column] & 0x7FFF == 0, 0x3F80, q[:, :, column])
    clean = absorbed(E, b, q).reshape(-1, LATENT)
    q64 = bf16_to_f64(q).reshape(-1, ROW)
    for key in _places(cached, new):
        for bits in (0x7F80, 0xFF80):
            bad = rows.copy()
            bad[key, column] = bits
            got = absorbed(E, Shared(cached, new, bad, 10), q).reshape(-1, LATENT)
            sees, above = visible > key, (q64[:, column] > 0) == (bits == 0x7F80)
            keys = np.where(np.arange(len(rows))[:, None] == key, 0.0, bf16_to_f64(rows))[:cached[0] + new[0]]
            alone = visible[at] > 1  # (a row with no other key has no number anywhere)
            want, size = attend(q64[at[alone]], visible[at[alone]], keys, keys[:, :LATENT], without=[key])
            _check(got[at[alone]], clean[at[alone]], sees[at[alone]], above[at[alone]], [column] if column < LATENT else [], want, size)
            # every row of every request: what is a number
            nan = np.isnan(bf16_to_f64(got))
            expect = np.zeros_like(nan)
            expect[sees & (above | (visible == 1))] = True
            if column < LATENT:
                expect[sees, column] = True
            assert not np.any(nan != expect), (key, bits)


@pytest.mark.parametrize("heads,cached,new", [(3, [100], [140]), (2, [0], [300]), (48, [20], [1500])])
def test_expanded_one_infinity_in_a_key(E, heads, cached, new):
    """In the latent: keys and values of the token are infinite throughout.  In the rotated part: its scores alone."""
    rng = np.random.default_rng(11)
    rows = W.gaussian_bf16(rng, (cached[0] + new[0], ROW), 1.0)
    q, w = W.gaussian_bf16(rng, (new[0], heads, 192), 1.0), W.gaussian_bf16(rng, (heads, 256, 512), 512 ** -0.5)
    column = 5
    # what column 5 of a latent gives to its keys has the sign of the query's element, or in odd rows the other one
    sign = np.where(np.arange(new[0]) % 2, -1.0, 1.0)
    q64, w64 = bf16_to_f64(q), bf16_to_f64(w)
    q64[:, :, :128] = sign[:, None, None] * (np.abs(q64[:, :, :128]) + 0.01)
    q64[:, :, 131] = sign[:, None] * (np.abs(q64[:, :, 131]) + 0.01)
    w64[:, :128, column] = np.abs(w64[:, :128, column]) + 0.01
    w64[:, 128:, column] += np.where(w64[:, 128:, column] < 0, -0.01, 0.01)
    q, w = f64_to_bf16(q64), f64_to_bf16(w64)
    q64, w64 = bf16_to_f64(q), bf16_to_f64(w)
    b = Shared(cached, new, rows, 12)
    visible, clean = b.visible(), expanded(E, b, q, w)
    at = np.unique(np.concatenate([np.arange(new[0])[-40:], rng.integers(0, new[0], 30)]))
    at = at[visible[at] > 1]
    for key in _places(cached, new):
        for where in (column, LATENT + 3):
            for bits in (0x7F80, 0xFF80):
                bad = rows.copy()
                bad[key, where] = bits
                got = expanded(E, Shared(cached, new, bad, 12), q, w)
                sees, above = visible > key, (sign > 0) == (bits == 0x7F80)
                nan = np.isnan(bf16_to_f64(got))
                expect = sees & (above | (where == column) | (visible == 1))
                assert not np.any(nan != expect[:, None, None]), (key, where, bits)
                for h in sorted({0, heads - 1}):
                    keep = bf16_to_f64(f64_to_bf16(bf16_to_f64(rows[:, :LATENT]) @ w64[h].T))
                    keys = np.concatenate([keep[:, :128], bf16_to_f64(rows[:, LATENT:])], 1)
                    want, size = attend(q64[at, h], visible[at], keys, keep[:, 128:], without=[key])
                    _check(got[at, h], clean[at, h], sees[at], above[at], np.arange(128) if where == column else [], want, size)


@pytest.mark.parametrize("name", ["rows16", "rows32", "rows32_two_waves", "rows128", "rows128_even"])
def test_absorbed_queries_that_are_no_numbers_keep_to_themselves(E, name):
    """Runs of query rows, some of them whole waves': the other rows keep their bits."""
    heads, cached, new = ROUTES[name][:3]
    rng = np.random.default_rng(13)
    b = Shared(cached, new, W.gaussian_bf16(rng, (max(np.add(cached, new)), ROW), 1.0), 14)
    q = W.gaussian_bf16(rng, (b.total, heads, ROW), 1.0)
    clean = absorbed(E, b, q).reshape(-1, LATENT)
    bad = np.arange(len(clean)) % 89 < 37
    for bits in (0x7FC0, 0xFF80):
        q2 = q.copy().reshape(-1, ROW)
        q2[bad] = bits
        got = absorbed(E, b, q2.reshape(q.shape)).reshape(-1, LATENT)
        assert np.array_equal(got[~bad], clean[~bad]) and np.all(np.isnan(bf16_to_f64(got[bad])))


@pytest.mark.parametrize("heads,cached,new", [(3, [100, 7], [140, 300]), (48, [20, 900], [1500, 200])])
def test_expanded_rows_that_are_no_numbers_keep_to_themselves(E, heads, cached, new):
    """Runs of query rows; a new token's latent, which the rows in front of it do not see."""
    rng = np.random.default_rng(15)
    rows = W.gaussian_bf16(rng, (max(np.add(cached, new)), ROW), 1.0)
    q, w = W.gaussian_bf16(rng, (sum(new), heads, 192), 1.0), W.gaussian_bf16(rng, (heads, 256, 512), 512 ** -0.5)
    b = Shared(cached, new, rows, 16)
    clean, visible = expanded(E, b, q, w), b.visible()
    bad = np.arange(sum(new)) % 89 < 37
    for bits in (0x7FC0, 0xFF80):
        q2, rows2 = q.copy(), rows.copy()
        q2[bad] = bits
        got = expanded(E, b, q2, w)
        assert np.array_equal(got[~bad], clean[~bad]) and np.all(np.isnan(bf16_to_f64(got[bad])))
        for key in (cached[0] + 33, cached[0] + new[0] - 1):
            rows2[key] = bits
            got = expanded(E, Shared(cached, new, rows2, 16), q, w)
            seen = visible > np.nonzero((rows2 != rows).any(1))[0].min()
            assert np.array_equal(got[~seen], clean[~seen]) and np.all(np.isnan(bf16_to_f64(got[seen])))
            rows2 = rows.copy()
