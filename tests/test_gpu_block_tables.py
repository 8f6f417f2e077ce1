"""efim_block_tables against a loop over requests and columns: every entry of the tables, the stack and the slot map."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _state(held, page, spare, seed, wide=None, capacity=None):
    """A block table with the held pages, and the stack of the others."""
    rng = np.random.default_rng(seed)
    need = [-(-max(int(h), 0) // page) for h in held]
    order = rng.permutation(sum(need) + spare).astype(np.int32)
    table = np.full((len(held), max(need + [1]) if wide is None else wide), -9, np.int32)
    at = 0
    for r, k in enumerate(need):
        k = min(k, table.shape[1])
        table[r, :k] = order[at:at + k]
        at += k
    free = np.full(len(order) if capacity is None else capacity, -5, np.int32)
    free[:len(order) - at] = order[at:]
    return table, free, len(order) - at


def _run(E, held, cached, new, page, table, free, count, slot_capacity, same_count=True, stream=None):
    h, c, n = (_dev(np.asarray(x, np.int32)) for x in (held, cached, new))
    t, f, before = _dev(table), _dev(free), _dev(np.array([count], np.int32))
    after = before if same_count else torch.full_like(before, -77)
    slots = torch.full((max(slot_capacity, 0) + 3,), -33, dtype=torch.int64, device="cuda")
    start, status = torch.full((len(held) + 1,), -44, dtype=torch.int32, device="cuda"), torch.full((1,), 55, dtype=torch.int32, device="cuda")
    size = E.efim_block_tables_workspace_bytes(len(held))
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    E.efim_block_tables(len(held), h, c, n, page, t, table.shape[1], f, len(free), before, after, None if slot_capacity < 0 else slots,
                        max(slot_capacity, 0), start, status, ws, size, stream=stream)
    torch.cuda.synchronize()
    if not same_count:
        assert int(before) == count
    assert (slots[max(slot_capacity, 0):] == -33).all()
    return t.cpu().numpy(), f.cpu().numpy(), int(after), slots[:max(slot_capacity, 0)].cpu().numpy(), start.cpu().numpy(), int(status)


def _check(E, held, cached, new, page, table, free, count, slot_capacity, **how):
    got = _run(E, held, cached, new, page, table, free, count, slot_capacity, **how)
    want = M.block_tables(held, cached, new, page, table, free, count, slot_capacity)
    for x, y, what in zip(got, want, ("table", "stack", "count", "slots", "row_start", "status")):
        assert np.array_equal(x, y), what
    return got


@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("batch", [0, 1, 2, 17, 64, 65, 130])
def test_steps_that_grow_and_shrink(E, batch, page):
    rng = np.random.default_rng(batch * page)
    for room in (0, 40, 5000):  # of the slot map, more than there are tokens: both ways through the kernels
        held = rng.integers(0, 900, batch)
        cached = np.where(rng.random(batch) < 0.3, 0, np.maximum(held - rng.integers(0, 300, batch), 0))
        new = np.where(rng.random(batch) < 0.3, 0, rng.integers(0, 200, batch))
        wide = max([1] + [-(-max(int(a), int(b + c)) // page) for a, b, c in zip(held, cached, new)])
        spare = int(sum(-(-(cached + new) // page))) + 3
        table, free, count = _state(held, page, spare, batch, wide)
        got = _check(E, held, cached, new, page, table, free, count, int(new.sum()) + room, same_count=room != 40)
        assert got[5] == 0
        # pages are where they were or in one place
        rows = [got[0][r, :-(-int(c + n) // page)] for r, (c, n) in enumerate(zip(cached, new))]
        everywhere = np.concatenate(rows + [got[1][:got[2]]])
        assert len(np.unique(everywhere)) == len(everywhere) == len(free)


def test_pages_that_come_back_are_taken_in_the_same_step(E):
    held, cached, new = [160, 0, 90, 16], [0, 0, 20, 16], [0, 100, 3, 40]
    table, free, count = _state(held, 16, 0, 3, 12)
    got = _check(E, held, cached, new, 16, table, free, count, 143)
    assert got[5] == 0 and count == 0
    _check(E, held, cached, new, 16, table, free, count, 4000)


@pytest.mark.parametrize("room", [100, 5000])
def test_pages_that_are_missing_leave_everything_as_it_was(E, room):
    held, cached, new = [32, 5], [32, 5], [33, 60]
    table, free, count = _state(held, 16, 6, 4, 8)
    assert _check(E, held, cached, new, 16, table, free, count, room)[5] == 1
    table, free, count = _state(held, 16, 7, 4, 8)
    assert _check(E, held, cached, new, 16, table, free, count, room)[5] == 0


@pytest.mark.parametrize("room", [100, 5000])
def test_lengths_and_counts_that_cannot_be(E, room):
    good = ([32, 5, 9], [32, 5, 0], [3, 6, 0])
    table, free, count = _state(good[0], 16, 6, 5, 8)
    for which, value in ((0, -1), (1, -1), (2, -5), (0, 129), (1, 128), (2, 10 ** 6), (1, 2 ** 31 - 1), (2, 2 ** 31 - 1), (0, 2 ** 31 - 1), (0, -2 ** 31)):
        for r in range(3):
            rows = [list(x) for x in good]
            rows[which][r] = value
            assert _check(E, *rows, 16, table, free, count, room)[5] != 0
    for wrong in (-1, len(free), len(free) + 1, 2 ** 31 - 1, -2 ** 31):  # (a page comes back from the last request)
        assert _check(E, *good, 16, table, free, wrong, room)[5] == -1
    assert _check(E, *good, 16, table, free, count, 8)[5] == -1  # nine tokens
    assert _check(E, *good, 16, table, free, count, 9)[5] == 0


def test_without_a_slot_map(E):
    table, free, count = _state([32, 5], 16, 9, 6, 8)
    assert _check(E, [32, 5], [32, 5], [33, 60], 16, table, free, count, -1)[5] == 0


def test_thousands_of_requests_and_a_long_one(E):
    rng = np.random.default_rng(7)
    held = rng.integers(0, 60, 2500)
    cached, new = held // 2, rng.integers(0, 50, 2500)
    table, free, count = _state(held, 8, 20000, 8, 14)
    assert _check(E, held, cached, new, 8, table, free, count, int(new.sum()) + 9)[5] == 0
    table, free, count = _state([70000, 3], 16, 3000, 9, 5000)
    assert _check(E, [70000, 3], [10, 3], [9, 40000], 16, table, free, count, 40009)[5] == 0
    assert _check(E, [70000, 3], [70000, 3], [9, 40000], 16, table, free, count, 40009)[5] == 0


@pytest.mark.parametrize("room", [300, 5000])
def test_a_captured_step_follows_the_lengths_on_the_device(E, room):
    """Replayed over other lengths and its own tables, step after step, with eager work between."""
    batch, page, wide = 9, 16, 40
    rng = np.random.default_rng(10)
    table, free, count = np.zeros((batch, wide), np.int32), np.arange(300, dtype=np.int32)[::-1].copy(), 300
    t, f, cnt = _dev(table), _dev(free), _dev(np.array([count], np.int32))
    h, c, n = (torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(3))
    slots = torch.empty(room, dtype=torch.int64, device="cuda")
    start, status = torch.empty(batch + 1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    size = E.efim_block_tables_workspace_bytes(batch)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        E.efim_block_tables(batch, h, c, n, page, t, wide, f, 300, cnt, cnt, slots, room, start, status, ws, size, stream=stream)

    step()  # (nothing to do)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    held = np.zeros(batch, np.int64)
    for k in range(12):
        cached = np.where(rng.random(batch) < 0.2, 0, np.maximum(held - rng.integers(0, 20, batch), 0))
        new = rng.integers(0, 33, batch)
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
        if want[5] == 0:
            held = cached + new
