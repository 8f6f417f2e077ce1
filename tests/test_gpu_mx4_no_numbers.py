"""Blocks that are no numbers, anywhere in a 4-bit cache: which rows lose which columns, and what a step over them takes."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from oracle.efim_oracle import bf16_to_f64

import gpu_util as U
import mx4_util as X
from test_gpu_mx4 import E, _attend, _dev  # noqa: F401 (E is a fixture)
from test_gpu_mx4_launches import _step

pytestmark = pytest.mark.gpu


def _scale_at(s, r, key, head, block):
    """Index of a scale byte."""
    page = s.page
    return s.table[r, key // page], head, page * (s.d // 2) + key % page * (s.d // 32) + block


@pytest.mark.parametrize("new,heads,d", [(2, (4, 2), 64), (2, (28, 4), 128), (40, (4, 2), 64), (40, (64, 32), 64), (40, (8, 2), 128), (300, (4, 1), 128)])
def test_a_key_that_is_no_number_far_back(E, new, heads, d):  # noqa: F811
    """Seen by all rows, by the last one and by none: those that see it are no numbers, whichever part it lies in, the others as they were."""
    cached = [2900, 2800, 900]
    s = _step(cached, [new] * 3, heads, d, seed=3)
    clean = bf16_to_f64(_attend(E, s)).reshape(3, new, heads[1], -1, d)
    s.caches[0][_scale_at(s, 0, 1500, 0, 1)] = M.NAN_BYTE
    s.caches[0][_scale_at(s, 1, 2800 + new - 1, 1 % heads[1], 0)] = M.NAN_BYTE
    s.caches[0][_scale_at(s, 2, 900 + new, 0, 0)] = M.NAN_BYTE  # (a slot behind the last key)
    got = bf16_to_f64(_attend(E, s)).reshape(clean.shape)
    lost = np.zeros(clean.shape, bool)
    lost[0, :, 0] = lost[1, -1, 1 % heads[1]] = True
    assert np.array_equal(np.isnan(got), lost)
    assert np.array_equal(got[~lost], clean[~lost])


@pytest.mark.parametrize("seed", range(16))
def test_values_that_are_no_numbers_anywhere(E, seed):  # noqa: F811
    """A row loses the columns of a block exactly where it sees one that is no number."""
    rng = np.random.default_rng(seed)
    heads, d = [(4, 4), (28, 4), (8, 1), (64, 1), (6, 2)][rng.integers(5)], [64, 128][seed % 2]
    batch, long = int(rng.integers(1, 7)), int(rng.choice([40, 600, 5000]))
    new = 1 + rng.integers(0, [3, 9, 70, 300][seed % 4], batch)
    s = _step(rng.integers(0, long, batch), new, heads, d, int(rng.choice([8, 16, 64])), seed=seed)
    at, torn = 0, []  # (request, head, block, key)
    lost = np.zeros((s.total, heads[1], heads[0] // heads[1], d), bool)
    for r, (c, n) in enumerate(zip(s.cached, s.new)):
        for _ in range(int(rng.integers(0, 4))):
            # (mostly among the new tokens, where some rows see them and others do not)
            key = int(c + rng.integers(0, n) if rng.random() < 0.7 else rng.integers(0, c + n))
            head, block = int(rng.integers(heads[1])), int(rng.integers(d // 32))
            torn.append(_scale_at(s, r, key, head, block))
            lost[at + max(0, key - c):at + n, head, :, block * 32:block * 32 + 32] = True
        at += n
    out, size, reach, keys = M.attention(s.cached, s.new, s.table, s.page, s.q, *s.caches, d ** -0.5)
    for where in torn:
        s.caches[1][where] = M.NAN_BYTE
    lost = lost.reshape(s.total, heads[0], d)
    got = bf16_to_f64(_attend(E, s))
    assert np.array_equal(np.isnan(got), lost)
    off = np.abs(got - out) / X.attention_bound(out, size, reach, keys, d)
    assert off[~lost].max(initial=0.0) <= 1.0


@pytest.mark.parametrize("cached,new,heads,d", [(30000, 1, (8, 2), 128), (30000, 5, (8, 2), 64), (0, 8192, (8, 2), 128), (20000, 60, (8, 2), 64)])
def test_a_value_that_is_no_number_costs_little(E, cached, new, heads, d):  # noqa: F811
    """A block that is none stays in the cache: each step over it takes about as long as one over numbers."""
    s = _step([cached], [new], heads, d, seed=4)
    bad = s.caches[1].copy()
    for head in range(heads[1]):
        bad[_scale_at(s, 0, 0, head, 1)] = M.NAN_BYTE
    desc = s.desc(E, _dev(s.table))
    size = E.efim_mx4_workspace_bytes(desc)
    ws, q = torch.empty(size, dtype=torch.uint8, device="cuda"), U.dev_bits(s.q)
    out, k, values = torch.empty_like(q), _dev(s.caches[0]), (_dev(s.caches[1]), _dev(bad))
    times = ([], [])
    for turn in range(12):
        for v, of in zip(values, times):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for _ in range(5):
                E.efim_extend_attention_mx4(desc, q, k, v, out, 0.0, ws, size)
            end.record()
            end.synchronize()
            of.append(begin.elapsed_time(end) * 200.0)  # us a call
    plain, torn = (float(np.median(x[2:])) for x in times)
    print("%d + %d, %d/%d heads, head dim %d: %.1f us, with a block that is no number %.1f" % (cached, new, *heads, d, plain, torn), flush=True)
    assert torn <= 1.5 * plain + 10.0, (plain, torn)
