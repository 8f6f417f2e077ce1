"""The 4-bit cache on the device: append against the oracle bit for bit, attention against fp64 within what its roundings allow."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from oracle.efim_oracle import bf16_to_f64
from paper_2505_21889_amd import workloads as W

import gpu_util as U
import mx4_util as X

pytestmark = pytest.mark.gpu

FREQ = 1.0e6 ** (-np.arange(64) / 64.0)


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# --- append ------------------------------------------------------------------------------------------------------------


def _append(E, s, inv_freq, rotary, inter, in_place=False, with_q=True, stored=True, stream=None):
    table = _dev(s.table)
    q = U.dev_bits(s.q) if with_q else None
    q_out = None if not with_q else q if in_place else torch.full(q.shape, 0x7FC1, dtype=torch.int16, device="cuda")
    k, v = U.dev_bits(s.k), U.dev_bits(s.v)
    back = [torch.full(k.shape, 0x7FC1, dtype=torch.int16, device="cuda") for _ in range(2)] if stored else [None, None]
    caches = [_dev(c) for c in s.caches]
    E.efim_rope_append_mx4(s.desc(E, table), q, q_out, k, v, *caches, *back, inv_freq, rotary, inter, stream=stream)
    torch.cuda.synchronize()
    if with_q and not in_place:
        assert np.array_equal(U.host_bits(q), s.q), "the raw queries are read only"
    return (U.host_bits(q_out) if with_q else None, *(c.cpu().numpy() for c in caches),
            *(None if b is None else bf16_to_f64(U.host_bits(b)) for b in back))


def _check_append(E, s, inv_freq, rotary, inter, **how):
    got = _append(E, s, inv_freq, rotary, inter, **how)
    want = [c.copy() for c in s.caches]
    q, k, v = M.append(s.cached, s.new, s.table, s.page, s.q if got[0] is not None else None, s.k, s.v, *want, inv_freq[:rotary // 2], inter)
    assert np.array_equal(got[1], want[0]) and np.array_equal(got[2], want[1])  # every byte of the caches
    if q is not None:
        assert np.array_equal(got[0], q)
    if got[3] is not None:
        assert np.array_equal(got[3], k, equal_nan=True) and np.array_equal(got[4], v, equal_nan=True)


@pytest.mark.parametrize("inter", [0, 1])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (128, 48), (128, 16), (64, 64), (64, 32), (64, 16), (64, 48)])
def test_append_is_the_definition_bit_for_bit(E, d, rotary, inter):
    for page in (8, 16, 256):
        _check_append(E, X.Step([10, 0, 255, 77], [5, 17, 0, 1], (6, 2), d, page, seed=rotary + page), FREQ, rotary, inter)


@pytest.mark.parametrize("heads", [(1, 1), (28, 4), (32, 32), (7, 7), (64, 1)])
def test_append_head_layouts_in_place_and_keys_only(E, heads):
    s = X.Step([100, 3], [3, 9], heads, 128, 16, seed=heads[0])
    _check_append(E, s, FREQ, 128, 0, in_place=True)
    _check_append(E, s, FREQ, 128, 1, with_q=False)
    _check_append(E, s, FREQ, 128, 0, stored=False)


def test_append_more_requests_than_a_launch_takes(E):
    rng = np.random.default_rng(5)
    _check_append(E, X.Step(rng.integers(0, 40, 800), rng.integers(0, 3, 800), (2, 1), 64, 8, seed=6), FREQ, 64, 0)


def test_append_every_bf16_number_and_blocks_that_are_not_finite(E):
    """All 65536 patterns as values, in blocks of neighbours (so of one exponent), of mixed ones and with signs turned."""
    every = np.arange(65536, dtype=np.uint16)
    rows = np.concatenate([every, np.random.default_rng(1).permutation(every), (every[::-1] * 40503) & 0xFFFF]).reshape(-1, 2, 128)
    s = X.Step([0], [len(rows)], (2, 2), 128, 16, seed=2, filled=False)
    s.v = rows.copy()
    s.k = rows.copy()  # at the first position the angle is zero; elsewhere nothing below is rotated but the first 16 elements
    # finite elements only where they are rotated: products of infinities there are the rotation's, not the rounding's, matter
    s.k[:, :, :16] = W.gaussian_bf16(np.random.default_rng(3), (len(rows), 2, 16), 1.0)
    _check_append(E, s, FREQ, 16, 0)


def test_append_scales_at_the_borders(E):
    """Largest elements next to 7 2^s, at the ends of the scales' range, and blocks of zeros with signs."""
    rng = np.random.default_rng(4)
    rows = W.gaussian_bf16(rng, (64, 1, 128), 1e-3)
    for i, top in enumerate([0x40E0, 0x40E1, 0x40DF, 0x4100, 0x7F7F, 0x7F60, 0x7F61, 0x0001, 0x0080, 0x0260, 0x0261, 0x01FF, 0x8000, 0x0000]):
        rows[i, 0, 32:64] = 0x8000 if top in (0, 0x8000) else 0
        rows[i, 0, 40] = top
        rows[i, 0, 70] = top | 0x8000
    s = X.Step([0], [64], (1, 1), 128, 16, seed=5, filled=False)
    s.v = rows
    _check_append(E, s, FREQ, 128, 0)


# --- attention ---------------------------------------------------------------------------------------------------------


def _attend(E, s, scale=0.0, stream=None):
    out = torch.full((s.total, s.hq, s.d), 0x7FC1, dtype=torch.int16, device="cuda")  # no numbers: unwritten rows show
    desc = s.desc(E, _dev(s.table))
    size = E.efim_mx4_workspace_bytes(desc)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    E.efim_extend_attention_mx4(desc, U.dev_bits(s.q), _dev(s.caches[0]), _dev(s.caches[1]), out, scale, ws, size, stream=stream)
    torch.cuda.synchronize()
    return U.host_bits(out)


def _check(E, s, scale=0.0):
    got = bf16_to_f64(_attend(E, s, scale))
    out, size, reach, keys = M.attention(s.cached, s.new, s.table, s.page, s.q, *s.caches, scale or s.d ** -0.5)
    off = np.abs(got - out) / X.attention_bound(out, size, reach, keys, s.d)
    assert off.max() <= 1.0, off.max()
    return got


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys", [1, 2, 31, 32, 33, 127, 128, 129, 255, 257, 1000, 4097])
def test_one_new_token(E, keys, d):
    for heads in ((1, 1), (8, 2), (7, 1)):
        _check(E, X.Step([keys - 1], [1], heads, d, seed=keys))


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_that_end_inside_tiles(E, page, d):
    _check(E, X.Step([130, 7, 61, 0, 300], [1, 2, 4, 1, 3], (8, 2), d, page, seed=page))
    _check(E, X.Step([130, 0, 61], [70, 33, 129], (4, 1), d, page, seed=page + 1))


@pytest.mark.parametrize("rows", [(1, 16), (16, 1), (17, 1), (4, 4), (4, 5), (2, 16), (32, 1), (33, 1), (1, 33), (1, 64), (5, 7), (127, 1), (129, 1), (65, 2)])
def test_rows_of_every_kernel_and_their_borders(E, rows):
    """Numbers of new tokens and heads of a group on both sides of 16, 32 and 128 query rows."""
    n, g = rows
    for d in (64, 128):
        _check(E, X.Step([0, 200, 513], [n, n, n], (2 * g, 2), d, seed=n * g))


def test_a_step_that_mixes_everything(E):
    _check(E, X.Step([900, 0, 0, 250, 64, 63, 1, 0, 2000], [1, 300, 0, 40, 1, 8, 16, 1, 0], (12, 4), 128, seed=11))
    _check(E, X.Step([900, 0, 0, 250, 64, 63, 1, 0, 2000], [1, 300, 0, 40, 1, 8, 16, 1, 0], (12, 4), 64, 8, seed=12))


def test_more_requests_than_a_launch_takes(E):
    rng = np.random.default_rng(3)
    new = rng.choice([0, 1, 2, 40], 230)
    _check(E, X.Step(rng.integers(0, 200, 230), new, (4, 1), 64, seed=4))


def test_long_contexts_are_cut_and_joined(E):
    """One request: its keys go to many workgroups, in both kernels."""
    _check(E, X.Step([20000], [1], (4, 1), 128, seed=21))
    _check(E, X.Step([9000], [40], (4, 2), 128, 64, seed=22))
    _check(E, X.Step([30000, 5], [6, 6], (8, 2), 64, seed=23))


def test_whole_tiles_units_and_even_shares(E):
    """The ways in which tiles of many rows are dealt: more tiles than places, a unit for each place, shares that end inside tiles."""
    rng = np.random.default_rng(7)
    _check(E, X.Step(rng.integers(0, 200, 9), rng.integers(33, 150, 9), (64, 64), 64, seed=61))
    _check(E, X.Step([3000, 0, 700], [150, 40, 65], (8, 2), 128, seed=62))
    _check(E, X.Step(rng.integers(2600, 3300, 12), rng.integers(33, 60, 12), (16, 16), 64, seed=63))
    _check(E, X.Step(rng.integers(2600, 3300, 12), rng.integers(33, 60, 12), (16, 16), 128, 8, seed=64))


@pytest.mark.parametrize("new,heads", [(2, (4, 2)), (40, (4, 2)), (40, (64, 32))])
def test_blocks_that_are_no_numbers_far_back(E, new, heads):
    """In keys and values whose parts are joined: the rows that see them lose them, and those in front do not."""
    s = X.Step([2900, 2800], [new, new], heads, 64, seed=71)
    for r, token, head, block in ((0, 1500, 0, 1), (0, 2900 + new - 1, 1, 0)):
        page = s.table[r, token // s.page]
        s.caches[1][page, head, s.page * 32 + token % s.page * 2 + block] = M.NAN_BYTE
    got = bf16_to_f64(_attend(E, s)).reshape(2, new, heads[1], -1, 64)
    assert np.isnan(got[0, :, 0, :, 32:]).all() and np.isnan(got[0, -1, 1, :, :32]).all()
    got[0, :, 0, :, 32:] = got[0, -1, 1, :, :32] = 0.0
    assert not np.isnan(got).any()


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(E, seed):
    rng = np.random.default_rng(900 + seed)
    heads = [(4, 4), (28, 4), (8, 1), (32, 8), (64, 1), (6, 2)][rng.integers(6)]
    batch, long = int(rng.integers(1, 12)), int(rng.choice([5, 70, 600, 3000]))
    new = rng.integers(0, rng.choice([2, 6, 40, 120]), batch)
    _check(E, X.Step(rng.integers(0, long, batch), new + (new.sum() == 0), heads, int(rng.choice([64, 128])), int(rng.choice([8, 16, 32, 256])), seed=seed))


def test_a_whole_prompt(E):
    _check(E, X.Step([0], [1100], (4, 1), 128, seed=31))
    _check(E, X.Step([0, 700], [520, 333], (3, 3), 64, seed=32))


@pytest.mark.parametrize("scale", [1e-4, 0.5, 3.0])
def test_scales_and_scores_that_rise(E, scale):
    """Scores that rise along the context move every row's reference again and again."""
    for new in (1, 50):
        s = X.Step([700], [new], (4, 1), 128, seed=41)
        _check(E, s, scale)
        t = np.arange(700 + new)
        rows = W.gaussian_bf16(np.random.default_rng(5), (len(t), 1, 128), 1.0)
        up = bf16_to_f64(rows) * (0.02 * t)[:, None, None]
        codes, scales = M.quantise(M.f64_to_bf16(up))
        M.put(s.caches[0], s.page, 128, s.table[0, t // s.page], t % s.page, codes, scales)
        _check(E, s, scale)


def test_a_row_does_not_depend_on_the_others_in_a_batch_s_launches(E):
    """The same call twice, and on another stream: the same bits."""
    s = X.Step([5000, 40, 0], [1, 30, 200], (8, 2), 128, seed=51)
    first = _attend(E, s)
    assert np.array_equal(first, _attend(E, s))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    assert np.array_equal(first, _attend(E, s, stream=stream))


@pytest.mark.parametrize("new", [1, 3, 5, 40, 200])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_that_are_no_numbers(E, new, d):
    """Of a value: its columns are lost in the rows that see it, and no others.  Of a key: the rows that see it are lost."""
    for which in (1, 0):
        for where in ("hidden", "first", "middle", "all"):
            s = X.Step([150], [new], (4, 1), d, seed=61)
            keys = 150 + new
            at = {"hidden": [keys - 1], "first": [0], "middle": [75, 140, 150], "all": list(range(keys))}[where]
            for key in at:
                first = s.page * (d // 2) + key % s.page * (d // 32)
                s.caches[which][s.table[0, key // s.page], 0, first + 1] = 255
            got = bf16_to_f64(_attend(E, s))
            clean = X.Step([150], [new], (4, 1), d, seed=61)
            out, size, reach, n = M.attention(clean.cached, clean.new, clean.table, clean.page, clean.q, *clean.caches, d ** -0.5)
            sees = (150 + np.arange(new) >= min(at))[:, None, None]
            block = (np.arange(d) // 32 == 1)[None, None] if which else np.ones((1, 1, d), bool)
            lost = np.broadcast_to(sees & block, got.shape)
            assert np.array_equal(np.isnan(got), lost), (which, where)
            off = np.abs(got - out) / X.attention_bound(out, size, reach, n, d)
            assert lost.all() or off[~lost].max() <= 1.0


def test_queries_that_are_not_finite_keep_to_themselves(E):
    for new in (4, 60):
        s = X.Step([300], [new], (4, 1), 128, seed=71)
        clean = _attend(E, s)
        s.q[1, 2, 5], s.q[3, 0, 100] = 0x7F80, 0x7FC0
        got = _attend(E, s)
        hit = np.zeros(got.shape[:2], bool)
        hit[1, 2] = hit[3, 0] = True
        assert np.array_equal(got[~hit], clean[~hit])
        assert np.isnan(bf16_to_f64(got[3, 0])).all()


def test_caches_beyond_four_gigabytes(E):
    """Pages whose bytes lie behind 2^32 of the cache."""
    s = X.Step([600, 30], [3, 90], (16, 8), 128, 256, seed=81)
    pages = 33000
    assert E.efim_mx4_cache_bytes(pages, 8, 256, 128) > 2 ** 32
    high = s.table + (pages - s.pages)
    table = _dev(high)
    caches = []
    for c in s.caches:
        big = torch.empty((pages,) + s.shape[1:], dtype=torch.uint8, device="cuda")
        big[pages - s.pages:] = _dev(c)
        caches.append(big)
    desc = E.BatchDesc(s.cached, s.new, table, 16, 8, 128, 256, pages)
    size = E.efim_mx4_workspace_bytes(desc)
    out = torch.empty((s.total, 16, 128), dtype=torch.int16, device="cuda")
    E.efim_extend_attention_mx4(desc, U.dev_bits(s.q), *caches, out, 0.0, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
    assert np.array_equal(U.host_bits(out), _attend(E, s))
    E.efim_rope_append_mx4(desc, U.dev_bits(s.q), out, U.dev_bits(s.k), U.dev_bits(s.v), *caches, None, None, FREQ, 128)
    got = _append(E, s, FREQ, 128, 0)
    assert np.array_equal(caches[0][pages - s.pages:].cpu().numpy(), got[1])
    assert np.array_equal(caches[1][pages - s.pages:].cpu().numpy(), got[2])


def test_append_and_attention_captured_into_a_graph(E):
    """Captured once, replayed over other rows and other pages, with eager work between the replays."""
    s = X.Step([700, 40, 0], [1, 30, 200], (8, 2), 128, seed=91)
    table, caches = _dev(s.table), [_dev(c) for c in s.caches]
    q, k, v = (U.dev_bits(x) for x in (s.q, s.k, s.v))
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    desc = s.desc(E, table)
    size = E.efim_mx4_workspace_bytes(desc)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        E.efim_rope_append_mx4(desc, q, q_out, k, v, *caches, None, None, FREQ, 128, stream=stream)
        E.efim_extend_attention_mx4(desc, q_out, *caches, out, 0.0, ws, size, stream=stream)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for seed in range(3):
        other = X.Step([700, 40, 0], [1, 30, 200], (8, 2), 128, seed=100 + seed)
        table.copy_(_dev(other.table))
        for to, x in zip((q, k, v), (other.q, other.k, other.v)):
            to.copy_(U.dev_bits(x))
        for to, x in zip(caches, other.caches):
            to.copy_(_dev(x))
        graph.replay()
        torch.cuda.synchronize()
        replayed = (U.host_bits(out), *(c.cpu().numpy() for c in caches))
        for to, x in zip(caches, other.caches):
            to.copy_(_dev(x))
        step()
        torch.cuda.synchronize()
        for x, y in zip(replayed, (U.host_bits(out), *(c.cpu().numpy() for c in caches))):
            assert np.array_equal(x, y)


def test_two_streams_with_a_workspace_each(E):
    a, b = X.Step([3000], [1], (32, 8), 128, seed=95), X.Step([100, 900], [100, 7], (8, 2), 64, seed=96)
    want = [_attend(E, s) for s in (a, b)]
    runs = []
    for s in (a, b):
        desc = s.desc(E, _dev(s.table))
        size = E.efim_mx4_workspace_bytes(desc)
        runs.append((desc, U.dev_bits(s.q), _dev(s.caches[0]), _dev(s.caches[1]), torch.empty((s.total, s.hq, s.d), dtype=torch.int16, device="cuda"),
                     0.0, torch.empty(size, dtype=torch.uint8, device="cuda"), size))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for run, stream in zip(runs, streams):
            E.efim_extend_attention_mx4(*run, stream=stream)
    torch.cuda.synchronize()
    for run, x in zip(runs, want):
        assert np.array_equal(U.host_bits(run[4]), x)
