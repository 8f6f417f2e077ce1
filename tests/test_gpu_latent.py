"""The latent cache against fp64: append, absorbed attention, expanded attention, and the two forms against each other."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as S
from oracle.efim_oracle import bf16_to_f64, f64_to_bf16
from paper_2505_21889_amd import workloads as W

import gpu_util as U

pytestmark = pytest.mark.gpu

SCALE = 192 ** -0.5
ROW = 576


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


class Batch:
    """A ragged batch over a latent cache: shuffled pages, every slot behind a request's keys and every unused page poison."""

    def __init__(self, cached, new, heads, page, seed, sigma=1.0):
        rng = self.rng = np.random.default_rng(seed)
        self.cached, self.new = np.asarray(cached, np.int32), np.asarray(new, np.int32)
        self.heads, self.page, self.total = heads, page, int(np.sum(new))
        self.table, self.pages = W.make_block_table(self.cached, self.new, page, rng)
        self.cache = np.full((self.pages, page, ROW), W.POISON_BITS, np.uint16)
        for r, (c, n) in enumerate(zip(cached, new)):
            at = np.arange(c + n)
            self.cache[self.table[r][at // page], at % page] = W.gaussian_bf16(rng, (c + n, ROW), sigma)
        self.table_dev = torch.from_numpy(self.table).cuda()

    def desc(self, E):
        return E.BatchDesc(self.cached, self.new, self.table_dev, self.heads, 1, ROW, self.page, self.pages)

    def gaussian(self, *shape, sigma=1.0):
        return W.gaussian_bf16(self.rng, shape, sigma)


def _workspace(nbytes):
    return torch.full((max(nbytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN patterns: nothing is taken from it


def _absorbed(E, b, q, cache=None, scale=SCALE):
    desc = b.desc(E)
    qd, cd = U.dev_bits(q), U.dev_bits(b.cache if cache is None else cache)
    out = torch.full((b.total, b.heads, 512), 0x7FC1, dtype=torch.int16, device="cuda")
    nbytes = E.efim_latent_workspace_bytes(desc)
    E.efim_latent_attention(desc, qd, cd, out, scale, _workspace(nbytes), nbytes)
    torch.cuda.synchronize()
    return U.host_bits(out)


def _expanded(E, b, q, w, scale=SCALE):
    desc = b.desc(E)
    qd, cd, wd = U.dev_bits(q), U.dev_bits(b.cache), U.dev_bits(w)
    out = torch.full((b.total, b.heads, 128), 0x7FC1, dtype=torch.int16, device="cuda")
    nbytes = E.efim_latent_expanded_workspace_bytes(desc)
    E.efim_latent_attention_expanded(desc, qd, cd, wd, out, scale, _workspace(nbytes), nbytes)
    torch.cuda.synchronize()
    return U.host_bits(out)


def _close(got_bits, want, size, more=0.0):
    """size: the mean magnitude of the values under the softmax's weights.  A weight is rounded to bf16 (at most 2^-8 of it)
    in the sum and in the normaliser, the output once more; fp32 scores of 576 products and the exponential: 1e-3 of size."""
    got = bf16_to_f64(got_bits)
    assert np.all(np.isfinite(got))
    worst = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 1e-3 + more) * size)
    assert np.all(worst <= 0), "bound passed by %.3e" % worst.max()


# --- append ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("cached,new,heads,page,inter,pad", [
    ([0], [1], 1, 16, 0, 0),
    ([5, 0, 31, 16000], [3, 0, 40, 9], 16, 8, 1, 8),
    ([100, 255], [1, 130], 33, 256, 0, 64),
    ([7] * 80, [2] * 80, 4, 32, 0, 0),
    ([1] * 400, [1] * 400, 2, 16, 1, 0),
])
def test_append_against_fp64(E, cached, new, heads, page, inter, pad):
    b = Batch(cached, new, heads, page, 51 + heads)
    before = b.cache.copy()
    kv, q = b.gaussian(b.total, ROW + pad, sigma=3.0), b.gaussian(b.total, heads, 192)
    weight, inv_freq, eps = b.gaussian(512), 1e4 ** (-2.0 * np.arange(32) / 64), 1e-6
    qd, kvd, cd = U.dev_bits(q), U.dev_bits(kv), U.dev_bits(b.cache)
    q_abs = torch.full((b.total, heads, ROW), 0x7FC1, dtype=torch.int16, device="cuda")
    # from a slice of the projection into a slice of the absorbed queries
    E.efim_latent_append(b.desc(E), qd[:, :, 128:], 192, q_abs[:, :, 512:], ROW, kvd, ROW + pad, U.dev_bits(weight), eps, cd, inv_freq, inter)
    torch.cuda.synchronize()
    got_q, got = U.host_bits(q_abs), U.host_bits(cd)
    assert np.all(got_q[:, :, :512] == 0x7FC1) and np.array_equal(U.host_bits(qd), q)
    req, pos = S.positions(b.cached, b.new)
    want_q = S.rotate(bf16_to_f64(q[:, :, 128:]), pos, inv_freq, inter)
    raw = bf16_to_f64(kv[:, :ROW])
    want = np.concatenate([S.rms_norm(raw[:, :512], bf16_to_f64(weight), eps), S.rotate(raw[:, None, 512:], pos, inv_freq, inter)[:, 0]], 1)
    at, slot = b.table[req, pos // page], pos % page
    for have, ref in ((got_q[:, :, 512:], want_q), (got[at, slot][:, :512], want[:, :512]), (got[at, slot][:, 512:], want[:, 512:])):
        # one rounding to bf16, fp32 arithmetic in front of it
        assert np.all(np.abs(bf16_to_f64(have) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * np.abs(ref).max(-1, keepdims=True))
    got[at, slot], before[at, slot] = 0, 0
    assert np.array_equal(got, before), "no other slot changes"
    # in place, and keys only
    cd2, cd3 = U.dev_bits(b.cache), U.dev_bits(b.cache)
    qd2 = qd.clone()
    E.efim_latent_append(b.desc(E), qd2[:, :, 128:], 192, qd2[:, :, 128:], 192, kvd, ROW + pad, U.dev_bits(weight), eps, cd2, inv_freq, inter)
    E.efim_latent_append(b.desc(E), None, 0, None, 0, kvd, ROW + pad, U.dev_bits(weight), eps, cd3, inv_freq, inter)
    torch.cuda.synchronize()
    assert torch.equal(cd2, cd) and torch.equal(cd3, cd)
    assert np.array_equal(U.host_bits(qd2)[:, :, 128:], got_q[:, :, 512:]) and np.array_equal(U.host_bits(qd2)[:, :, :128], q[:, :, :128])


def test_append_without_weight(E):
    b = Batch([3], [5], 2, 16, 8)
    kv = b.gaussian(b.total, ROW)
    kv[1, :512] = 0
    ones = np.full(512, 0x3F80, np.uint16)
    outs = []
    for w in (None, U.dev_bits(ones)):
        cd = U.dev_bits(b.cache)
        E.efim_latent_append(b.desc(E), None, 0, None, 0, U.dev_bits(kv), ROW, w, 1e-6, cd, np.ones(32), 0)
        torch.cuda.synchronize()
        outs.append(U.host_bits(cd))
    assert np.array_equal(*outs)
    assert np.all(outs[0][b.table[0, 0], 4, :512] == 0)


# --- attention -------------------------------------------------------------------------------------------------------------


LENGTHS = [
    ([0], [1]),                                   # one key
    ([0, 1, 30, 31, 32, 33], [1, 1, 1, 1, 1, 1]),  # around a key tile
    ([127, 128, 129, 640], [1, 1, 1, 1]),
    ([500, 0, 63], [2, 5, 0]),                    # a request without new tokens
    ([0, 200, 5], [40, 17, 3]),
    ([1000, 96], [9, 33]),
]


@pytest.mark.parametrize("cached,new", LENGTHS)
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 8), (16, 64), (28, 16), (128, 256)])
def test_absorbed_against_fp64(E, cached, new, heads, page):
    if heads * sum(new) * (max(cached) + max(new)) > 4000000:
        heads = 16
    b = Batch(cached, new, heads, page, 100 + heads)
    q = b.gaussian(b.total, heads, ROW)
    got = _absorbed(E, b, q)
    want, size = S.latent_attention(b.cached, b.new, b.table, page, bf16_to_f64(q), b.cache, SCALE)
    _close(got, want, size)
    assert np.array_equal(got, _absorbed(E, b, q)), "the same call gives the same bits"


@pytest.mark.parametrize("heads,new", [(16, 1), (4, 8), (16, 2), (1, 32), (17, 1), (33, 1), (16, 40)])
def test_absorbed_split_over_long_contexts(E, heads, new):
    """Few rows behind long contexts: ranges of keys on many workgroups, joined; 17 and 33 rows leave most of a tile empty."""
    b = Batch([5000, 2049], [new, new], heads, 16, 7 + heads)
    assert E.efim_latent_workspace_bytes(b.desc(E)) > 256, "the case is meant to split"
    q = b.gaussian(b.total, heads, ROW)
    want, size = S.latent_attention(b.cached, b.new, b.table, 16, bf16_to_f64(q), b.cache, SCALE)
    _close(_absorbed(E, b, q), want, size)


@pytest.mark.parametrize("cached,new", [
    ([9000, 5, 700, 64], [1, 1, 1, 1]),            # parts of one tile each, from one key tile to many
    ([9000, 0, 700, 64, 2000], [2, 9, 3, 16, 7]),  # several tiles of a request
    ([3000] * 30, [1] * 30),                       # as many parts for each
    ([100 * r for r in range(60)], [1 + r % 3 for r in range(60)]),
    ([0, 0, 4000], [40, 1, 1]),                    # first tiles of fewer key tiles than others have parts
])
@pytest.mark.parametrize("heads", [4, 16, 48])
def test_absorbed_dealt_over_tiles_of_different_lengths(E, cached, new, heads):
    b = Batch(cached, new, heads, 32, 170 + heads)
    q = b.gaussian(b.total, heads, ROW)
    got = _absorbed(E, b, q)
    want, size = S.latent_attention(b.cached, b.new, b.table, 32, bf16_to_f64(q), b.cache, SCALE)
    _close(got, want, size)
    assert np.array_equal(got, _absorbed(E, b, q)), "the same call gives the same bits"


@pytest.mark.parametrize("heads", [16, 32, 64])
def test_absorbed_scores_that_grow_and_sharp_weights(E, heads):
    """Keys whose scores grow along the context move the running reference in almost every tile; large queries leave one weight."""
    b = Batch([700, 300], [1, 2], heads, 16, 77)
    q = b.gaussian(b.total, heads, ROW)
    cache = b.cache.copy()
    for r, (c, n) in enumerate(zip(b.cached, b.new)):
        at = np.arange(c + n)
        rows = bf16_to_f64(cache[b.table[r][at // 16], at % 16]) * (0.05 * at[:, None] + 0.1)
        cache[b.table[r][at // 16], at % 16] = f64_to_bf16(rows)
    for scale in (SCALE, 20 * SCALE, 1e-3):
        want, size = S.latent_attention(b.cached, b.new, b.table, 16, bf16_to_f64(q), cache, scale)
        # scores reach some thousands of units here: fp32 leaves 2^-24 of the largest partial sum of an exponent
        top = scale * 4.0 * 36.0 * ROW
        _close(_absorbed(E, b, q, cache, scale), want, size, more=2.0 ** -22 * top)


def test_more_requests_than_a_launch_takes(E):
    rng = np.random.default_rng(3)
    cached, new = rng.integers(0, 60, 300), rng.integers(0, 3, 300)
    b = Batch(cached, new, 4, 16, 9)
    q = b.gaussian(b.total, 4, ROW)
    want, size = S.latent_attention(b.cached, b.new, b.table, 16, bf16_to_f64(q), b.cache, SCALE)
    _close(_absorbed(E, b, q), want, size)
    qe, w = b.gaussian(b.total, 4, 192), b.gaussian(4, 256, 512, sigma=512 ** -0.5)
    want, size = S.latent_attention_expanded(b.cached, b.new, b.table, 16, bf16_to_f64(qe), b.cache, bf16_to_f64(w), SCALE)
    _close(_expanded(E, b, qe, w), want, size, more=2e-3)


# (expanded keys that fp32 sums round to the other neighbour than fp64 sums do: a score then moves by 2^-8 of one product,
# 2e-3 of the values' size)
@pytest.mark.parametrize("cached,new", LENGTHS + [([0], [300]), ([64, 3], [129, 260])])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 8), (16, 64)])
def test_expanded_against_fp64(E, cached, new, heads, page):
    b = Batch(cached, new, heads, page, 200 + heads)
    q, w = b.gaussian(b.total, heads, 192), b.gaussian(heads, 256, 512, sigma=512 ** -0.5)
    got = _expanded(E, b, q, w)
    want, size = S.latent_attention_expanded(b.cached, b.new, b.table, page, bf16_to_f64(q), b.cache, bf16_to_f64(w), SCALE)
    _close(got, want, size, more=2e-3)
    assert np.array_equal(got, _expanded(E, b, q, w)), "the same call gives the same bits"


def test_expanded_many_row_tiles(E):
    """Enough rows and heads for the larger row tile."""
    b = Batch([0, 40], [2050, 700], 48, 16, 31)
    q, w = b.gaussian(b.total, 48, 192), b.gaussian(48, 256, 512, sigma=512 ** -0.5)
    got = bf16_to_f64(_expanded(E, b, q, w))
    heads = [0, 17, 47]  # (all are 40 s of fp64)
    want, size = S.latent_attention_expanded(b.cached, b.new, b.table, 16, bf16_to_f64(q)[:, heads], b.cache, bf16_to_f64(w)[heads], SCALE)
    _close(f64_to_bf16(got[:, heads]), want, size, more=2e-3)
    assert np.all(np.isfinite(got))


def test_the_two_forms_agree(E):
    """Absorbed queries and expanded outputs formed in fp64: the forms differ by the roundings of the operands alone."""
    b = Batch([130, 12], [20, 64], 8, 16, 61)
    q, w = b.gaussian(b.total, 8, 192), b.gaussian(8, 256, 512, sigma=512 ** -0.5)
    q64, w64 = bf16_to_f64(q), bf16_to_f64(w)
    absorbed = np.concatenate([np.einsum("thj,hjc->thc", q64[..., :128], w64[:, :128]), q64[..., 128:]], -1)
    latent = bf16_to_f64(_absorbed(E, b, f64_to_bf16(absorbed)))
    one = np.einsum("thc,hjc->thj", latent, w64[:, 128:])
    two = bf16_to_f64(_expanded(E, b, q, w))
    exact, _ = S.latent_attention_expanded(b.cached, b.new, b.table, 16, q64, b.cache, w64, SCALE, round_expanded=False)
    for x in (one, two):
        assert np.linalg.norm(x - exact) <= 1e-2 * np.linalg.norm(exact)


def test_rows_beyond_four_gigabytes(E):
    """Pages whose byte offsets pass 32 bits."""
    page, heads = 256, 16
    pages = (5 << 30) // (page * ROW * 2)
    cached, new = np.array([600], np.int32), np.array([3], np.int32)
    b = Batch(cached, new, heads, page, 71)
    far = pages - 1 - np.arange(b.table.shape[1])
    cache = torch.empty((pages, page, ROW), dtype=torch.int16, device="cuda")
    cache[torch.from_numpy(far).cuda()] = U.dev_bits(b.cache[b.table[0]])
    table = torch.from_numpy(far[None].astype(np.int32)).cuda()
    desc = E.BatchDesc(cached, new, table, heads, 1, ROW, page, pages)
    q, qe, w = b.gaussian(3, heads, ROW), b.gaussian(3, heads, 192), b.gaussian(heads, 256, 512, sigma=512 ** -0.5)
    out = torch.zeros(3, heads, 512, dtype=torch.int16, device="cuda")
    oute = torch.zeros(3, heads, 128, dtype=torch.int16, device="cuda")
    nbytes = E.efim_latent_workspace_bytes(desc)
    E.efim_latent_attention(desc, U.dev_bits(q), cache, out, SCALE, _workspace(nbytes), nbytes)
    nbytes = E.efim_latent_expanded_workspace_bytes(desc)
    E.efim_latent_attention_expanded(desc, U.dev_bits(qe), cache, U.dev_bits(w), oute, SCALE, _workspace(nbytes), nbytes)
    kv = b.gaussian(3, ROW)
    torch.cuda.synchronize()
    assert np.array_equal(U.host_bits(out), _absorbed(E, b, q))
    assert np.array_equal(U.host_bits(oute), _expanded(E, b, qe, w))
    E.efim_latent_append(desc, None, 0, None, 0, U.dev_bits(kv), ROW, None, 1e-6, cache, np.ones(32), 0)
    near = U.dev_bits(b.cache)
    E.efim_latent_append(b.desc(E), None, 0, None, 0, U.dev_bits(kv), ROW, None, 1e-6, near, np.ones(32), 0)
    torch.cuda.synchronize()
    assert np.array_equal(U.host_bits(cache[torch.from_numpy(far).cuda()]), U.host_bits(near)[b.table[0]])


def test_infinities_and_nan_behind_the_causal_limit(E):
    """A later new token's row full of NaN or infinities leaves the rows that do not see it as they are."""
    b = Batch([70], [12], 16, 16, 91)
    q, qe, w = b.gaussian(12, 16, ROW), b.gaussian(12, 16, 192), b.gaussian(16, 256, 512, sigma=512 ** -0.5)
    clean, clean_e = _absorbed(E, b, q), _expanded(E, b, qe, w)
    for bits in (0x7F80, 0xFF80, 0x7FC0):
        at = 70 + 11
        b.cache[b.table[0, at // 16], at % 16] = bits
        assert np.array_equal(_absorbed(E, b, q)[:11], clean[:11])
        assert np.array_equal(_expanded(E, b, qe, w)[:11], clean_e[:11])


def test_query_rows_that_are_no_numbers_keep_to_themselves(E):
    """Whole runs of a wave's query rows, and runs that cross tiles, in requests whose other rows see the same keys."""
    cached, new, heads = [5, 700, 40], [400, 300, 150], 4
    b = Batch(cached, new, heads, 16, 47)
    q, w = b.gaussian(b.total, heads, ROW), b.gaussian(heads, 256, 512, sigma=512 ** -0.5)
    short = np.ascontiguousarray(q[:, :, :192])
    clean = _absorbed(E, b, q), _expanded(E, b, short, w)
    bad = np.zeros(b.total, bool)
    for lo, hi in ((0, 70), (128, 256), (310, 401), (500, 564), (700, 849)):
        bad[lo:hi] = True
    for value in (0x7FC0, 0x7F80):
        q2, short2 = q.copy(), short.copy()
        q2[bad], short2[bad] = value, value
        for got, want in zip((_absorbed(E, b, q2), _expanded(E, b, short2, w)), clean):
            assert np.array_equal(got[~bad], want[~bad])
            assert not np.any(np.isfinite(bf16_to_f64(got[bad])))


def test_streams_and_graph_replays(E):
    """A side stream, and a captured graph replayed between eager work: append, both attentions."""
    b = Batch([900, 33], [3, 4], 16, 16, 13)
    kv, q, qe = U.dev_bits(b.gaussian(b.total, ROW)), U.dev_bits(b.gaussian(b.total, 16, ROW)), U.dev_bits(b.gaussian(b.total, 16, 192))
    w, cache = U.dev_bits(b.gaussian(16, 256, 512, sigma=512 ** -0.5)), U.dev_bits(b.cache)
    outs = [torch.zeros(b.total, 16, n, dtype=torch.int16, device="cuda") for n in (512, 128)]
    q_out, desc = torch.zeros(b.total, 16, 64, dtype=torch.int16, device="cuda"), b.desc(E)
    sizes = E.efim_latent_workspace_bytes(desc), E.efim_latent_expanded_workspace_bytes(desc)
    spaces = [_workspace(n) for n in sizes]
    freq = 1e4 ** (-2.0 * np.arange(32) / 64)

    def step(stream):
        E.efim_latent_append(desc, qe[:, :, 128:], 192, q_out, 64, kv, ROW, None, 1e-6, cache, freq, 0, stream)
        E.efim_latent_attention(desc, q, cache, outs[0], SCALE, spaces[0], sizes[0], stream)
        E.efim_latent_attention_expanded(desc, qe, cache, w, outs[1], SCALE, spaces[1], sizes[1], stream)

    def results():
        torch.cuda.synchronize()
        return [x.clone() for x in (*outs, q_out, cache)]

    step(None)
    want = results()
    side = torch.cuda.Stream()
    for x in (*outs, q_out):
        x.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    assert all(torch.equal(x, y) for x, y in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for k in range(4):
        for x in (*outs, q_out, *spaces):
            x.fill_(k)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(results(), want)), "replay %d" % k
        kv2 = kv.roll(k + 1, 0)
        (kv2.float() * 2).sum().item()  # the program's own work in between
