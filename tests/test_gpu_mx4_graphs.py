"""Two captured graphs of each operator of a step over a 4-bit cache, of different batches, in one workspace: replayed in turn, with eager
calls in the same workspace between, each gives what it gives alone."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M

import gpu_util as U
from test_gpu_block_tables import _state
from test_gpu_logit_probs import Rows
from test_gpu_mx4 import E, _attend, _dev  # noqa: F401 (E is a fixture)
from test_gpu_mx4_launches import _step

pytestmark = pytest.mark.gpu


def _captured(call):
    call(None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream())
    return graph


def _in_turn(calls, outputs, clear):
    """outputs: of each call, what it has to leave (numpy) and how to read it."""
    graphs = [_captured(call) for call in calls]
    for k in range(9):
        for i in ((0, 1), (1, 0), (1, 1))[k % 3]:
            clear(i)
            graphs[i].replay()
            torch.cuda.synchronize()
            want, read = outputs[i]
            assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(read(), want)), (k, i)
        clear(k % 2)
        calls[k % 2](None)
        torch.cuda.synchronize()
        want, read = outputs[k % 2]
        assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(read(), want)), k


def test_attention(E):  # noqa: F811
    steps = [_step([20000, 9], [1, 3], (8, 2), 128, seed=1), _step([3000, 0, 700], [150, 40, 2], (8, 2), 128, seed=2)]
    want = [_attend(E, s) for s in steps]
    descs = [s.desc(E, _dev(s.table)) for s in steps]
    size = max(E.efim_mx4_workspace_bytes(d) for d in descs)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    tensors = [(U.dev_bits(s.q), *map(_dev, s.caches), torch.empty((s.total, s.hq, s.d), dtype=torch.int16, device="cuda")) for s in steps]
    calls = [lambda stream, d=d, t=t: E.efim_extend_attention_mx4(d, *t, 0.0, ws, size, stream=stream) for d, t in zip(descs, tensors)]
    _in_turn(calls, [([w], lambda t=t: [U.host_bits(t[3])]) for w, t in zip(want, tensors)], lambda i: tensors[i][3].fill_(0x7FC1))


def test_probabilities(E):  # noqa: F811
    rows = [Rows([3, 0, 5], 70003, seed=1, history=300), Rows([1, 2], 5003, seed=2, bf16=False)]
    descs = [r.desc(E) for r in rows]
    size = max(E.efim_logit_workspace_bytes(d) for d in descs)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    outs = [torch.empty(len(r.logits), r.vocab, device="cuda") for r in rows]
    want = []
    for d, out, r in zip(descs, outs, rows):
        own = torch.empty(E.efim_logit_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        E.efim_logit_probs(d, out, r.vocab, own, len(own))
        want.append(out.cpu().numpy())
    calls = [lambda stream, d=d, o=o, r=r: E.efim_logit_probs(d, o, r.vocab, ws, size, stream=stream) for d, o, r in zip(descs, outs, rows)]
    _in_turn(calls, [([w], lambda o=o: [o.cpu().numpy()]) for w, o in zip(want, outs)], lambda i: outs[i].fill_(-7.0))


@pytest.mark.parametrize("batches", [(9, 30), (9, 90), (90, 300)])
def test_block_tables(E, batches):  # noqa: F811
    states, want = [], []
    for batch in batches:
        rng = np.random.default_rng(batch)
        held = rng.integers(0, 90, batch)
        cached, new = held // 2, rng.integers(0, 60, batch)
        table, free, count = _state(held, 16, 400 * batch // 50, batch, 12)
        host = (table, free, np.array([count], np.int32))
        want.append(M.block_tables(held, cached, new, 16, table, free, count, int(new.sum()) + 5))
        assert want[-1][5] == 0
        room = int(new.sum()) + 5
        states.append((batch, [_dev(x.astype(np.int32)) for x in (held, cached, new)], host, [_dev(x) for x in host], room,
                       torch.empty(room, dtype=torch.int64, device="cuda"), torch.empty(batch + 1, dtype=torch.int32, device="cuda"),
                       torch.empty(1, dtype=torch.int32, device="cuda")))
    size = max(E.efim_block_tables_workspace_bytes(b) for b in batches)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def call(stream, s):
        batch, lengths, host, (table, free, count), room, slots, start, status = s
        E.efim_block_tables(batch, *lengths, 16, table, 12, free, len(free), count, count, slots, room, start, status, ws, size, stream=stream)

    def clear(i):
        for x, y in zip(states[i][3], states[i][2]):
            x.copy_(_dev(y))

    def read(s):
        table, free, count = s[3]
        return [table.cpu().numpy(), free.cpu().numpy(), int(count), s[5].cpu().numpy(), s[6].cpu().numpy(), int(s[7])]

    _in_turn([lambda stream, s=s: call(stream, s) for s in states], [(w, lambda s=s: read(s)) for w, s in zip(want, states)], clear)
