"""efim_block_tables with more requests than a wave has lanes: a scan and a launch that fills behind it, and what they refuse."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M

from test_gpu_block_tables import E, _check, _dev, _state  # noqa: F401 (E is a fixture)

pytestmark = pytest.mark.gpu

#: places of the slot map: few, more than there are tokens by far, and between them
ROOMS = (600, 2048, 2049, 5000)


def _spread(values, batch, at=None):
    """`values` among `batch` requests, zeros elsewhere; the places are the same for every call with as many."""
    rows = np.zeros(batch, np.int64)
    rows[np.random.default_rng(batch).permutation(batch)[:len(values)] if at is None else at] = values
    return rows


@pytest.mark.parametrize("batch", [65, 96, 128, 129, 256, 1024, 1025])
@pytest.mark.parametrize("same_count", [True, False])
def test_a_token_for_each_user(E, batch, same_count):  # noqa: F811
    rng = np.random.default_rng(batch)
    cached = rng.integers(1, 600, batch)
    cached[::5] = cached[::5] // 16 * 16 + 16  # whose next token begins a page
    held = cached + np.where(rng.random(batch) < 0.3, rng.integers(0, 60, batch), 0)
    new = np.ones(batch, np.int64)
    table, free, count = _state(held, 16, batch, batch, 48)
    for room in (batch, 2048, 2049, -1):
        assert _check(E, held, cached, new, 16, table, free, count, room, same_count=same_count)[5] == 0


@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("batch", [65, 70, 127, 128, 129, 200])
def test_short_steps_that_grow_and_shrink(E, batch, page):  # noqa: F811
    rng = np.random.default_rng(batch * page)
    for room in ROOMS:
        held = rng.integers(0, 300, batch)
        cached = np.where(rng.random(batch) < 0.3, 0, np.maximum(held - rng.integers(0, 100, batch), 0))
        new = np.where(rng.random(batch) < 0.3, 0, rng.integers(0, 6, batch))
        new[rng.integers(0, batch, 3)] = 30  # (fewer than 600 tokens in all, but for the largest batch)
        new[new.cumsum() > room] = 0
        wide = max([1] + [-(-max(int(a), int(b + c)) // page) for a, b, c in zip(held, cached, new)])
        table, free, count = _state(held, page, int(sum(-(-(cached + new) // page))) + 3, batch, wide)
        for same_count in (True, False):
            got = _check(E, held, cached, new, page, table, free, count, room, same_count=same_count)
            assert got[5] == 0
        rows = [got[0][r, :-(-int(c + n) // page)] for r, (c, n) in enumerate(zip(cached, new))]
        everywhere = np.concatenate(rows + [got[1][:got[2]]])
        assert len(np.unique(everywhere)) == len(everywhere) == len(free)


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("batch", [70, 300])
def test_pages_that_come_back_are_taken_in_the_same_step(E, batch, room):  # noqa: F811
    held, cached, new = (_spread(x, batch) for x in ([160, 0, 90, 16, 33], [0, 0, 20, 16, 0], [0, 100, 3, 40, 0]))
    table, free, count = _state(held, 16, 0, 3, 12)
    assert count == 0
    for same_count in (True, False):
        assert _check(E, held, cached, new, 16, table, free, count, room, same_count=same_count)[5] == 0


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("batch", [70, 300])
def test_pages_that_are_missing_leave_everything_as_it_was(E, batch, room):  # noqa: F811
    held, cached, new = (_spread(x, batch) for x in ([32, 5, 40], [32, 5, 10], [33, 60, 0]))  # seven asked for, two come back
    for spare, status in ((4, 1), (5, 0), (0, 5)):
        table, free, count = _state(held, 16, spare, 4, 8)
        for same_count in (True, False):
            assert _check(E, held, cached, new, 16, table, free, count, room, same_count=same_count)[5] == status


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("batch", [70, 300])
def test_lengths_and_counts_that_cannot_be(E, batch, room):  # noqa: F811
    where = [0, batch // 2, batch - 1]
    good = [_spread(x, batch, where) for x in ([32, 5, 9], [32, 5, 0], [3, 6, 0])]
    table, free, count = _state(good[0], 16, 6, 5, 8)
    assert _check(E, *good, 16, table, free, count, room)[5] == 0
    for which, value in ((0, -1), (1, -1), (2, -5), (0, 129), (1, 128), (2, 10 ** 6), (1, 2 ** 31 - 1), (2, 2 ** 31 - 1), (0, 2 ** 31 - 1), (0, -2 ** 31)):
        for r in where:
            rows = [x.copy() for x in good]
            rows[which][r] = value
            assert _check(E, *rows, 16, table, free, count, room, same_count=r == 0)[5] != 0
    for wrong in (-1, len(free), len(free) + 1, 2 ** 31 - 1, -2 ** 31):  # (a page comes back from the last request)
        assert _check(E, *good, 16, table, free, wrong, room)[5] == -1
    assert _check(E, *good, 16, table, free, count, 8)[5] == -1  # nine tokens
    assert _check(E, *good, 16, table, free, count, 9)[5] == 0


@pytest.mark.parametrize("room", [300, 5000])
@pytest.mark.parametrize("batch", [70, 300])
def test_tokens_whose_sum_passes_32_bits(E, batch, room):  # noqa: F811
    wide = 2 ** 31 // batch // 256 + 2
    table, free = np.zeros((batch, wide), np.int32), np.arange(9, dtype=np.int32)
    new = np.full(batch, (wide - 1) * 256)
    assert new.sum() > 2 ** 31
    got = _check(E, np.zeros(batch, int), np.zeros(batch, int), new, 256, table, free, 9, room)
    assert got[5] == -1 and not got[4].any()


@pytest.mark.parametrize("batch", [70, 130, 300])
def test_without_a_slot_map(E, batch):  # noqa: F811
    held, cached, new = (_spread(x, batch) for x in ([32, 5, 90], [32, 5, 0], [33, 60, 0]))
    table, free, count = _state(held, 16, 9, 6, 8)
    for same_count in (True, False):
        assert _check(E, held, cached, new, 16, table, free, count, -1, same_count=same_count)[5] == 0


@pytest.mark.parametrize("batch,room,most", [(70, 300, 6), (70, 5000, 70), (128, 2048, 24), (300, 700, 3)])
def test_a_captured_step_follows_the_lengths_on_the_device(E, batch, room, most):  # noqa: F811
    """Replayed over other lengths and its own tables, step after step, with eager work between: steps that fit and steps that do not."""
    page, wide, pages = 16, 12, 4 * batch
    rng = np.random.default_rng(batch)
    table, free, count = np.zeros((batch, wide), np.int32), np.arange(pages, dtype=np.int32)[::-1].copy(), pages
    t, f, cnt = _dev(table), _dev(free), _dev(np.array([count], np.int32))
    h, c, n = (torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(3))
    slots = torch.empty(room, dtype=torch.int64, device="cuda")
    start, status = torch.empty(batch + 1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    size = E.efim_block_tables_workspace_bytes(batch)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        E.efim_block_tables(batch, h, c, n, page, t, wide, f, pages, cnt, cnt, slots, room, start, status, ws, size, stream=stream)

    step()  # (nothing to do)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    held, seen = np.zeros(batch, np.int64), set()
    for k in range(12):
        cached = np.where(rng.random(batch) < 0.2, 0, np.maximum(held - rng.integers(0, 20, batch), 0))
        new = rng.integers(0, most + 1 if k % 4 < 3 else 3 * most, batch)
        new[cached + new > wide * page] = 0
        for to, x in ((h, held), (c, cached), (n, new)):
            to.copy_(_dev(x.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        want = M.block_tables(held, cached, new, page, table, free, count, room)
        got = (t.cpu().numpy(), f.cpu().numpy(), int(cnt), slots.cpu().numpy(), start.cpu().numpy(), int(status))
        for x, y in zip(got, want):
            assert np.array_equal(x, y), k
        table, free, count = want[:3]
        seen.add(np.sign(want[5]))
        if want[5] == 0:
            held = cached + new
    assert 0 in seen and len(seen) > 1
