"""efim_logit_probs against the definition: each adjustment in fp32, the softmax in fp64."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from oracle import step_oracle as S
from oracle.efim_oracle import bf16_to_f64
from paper_2505_21889_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding
    return binding


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


class Rows:
    """What a call takes, on the host."""

    def __init__(self, drafts, vocab, seed=0, history=40, biases=6, masks=3, spread=4.0, bf16=True, heats=(0.0, 0.7, 1.0, 2.5)):
        rng = np.random.default_rng(seed)
        self.drafts, self.vocab, self.bf16 = list(drafts), vocab, bf16
        batch, total = len(self.drafts), sum(self.drafts) + len(self.drafts)
        self.bits = W.gaussian_bf16(rng, (total, vocab), spread)
        self.logits = bf16_to_f64(self.bits).astype(np.float32) if bf16 else (rng.standard_normal((total, vocab)) * spread).astype(np.float32)
        few = max(1, vocab // 3)
        self.history = rng.integers(0, few, (batch, history)).astype(np.int32)
        self.tokens = rng.integers(0, few, sum(self.drafts)).astype(np.int32)
        self.bias_tokens = rng.integers(0, vocab, (batch, biases)).astype(np.int32)
        self.bias_values = rng.standard_normal((batch, biases)).astype(np.float32)
        self.masks = rng.integers(0, 2 ** 32, (masks, (vocab + 31) // 32), dtype=np.uint32)
        self.mask_rows = rng.integers(-1, masks, total).astype(np.int32)
        self.params = np.zeros(batch, _dtype())
        self.params["temperature"] = rng.choice(heats, batch)
        self.params["repetition"] = rng.choice([1.0, 1.2, 0.9], batch)
        self.params["presence"] = rng.choice([0.0, 0.4, -0.3], batch)
        self.params["frequency"] = rng.choice([0.0, 0.2, -0.1], batch)
        self.params["history_len"] = rng.integers(0, history + 1, batch)
        self.params["prompt_len"] = rng.integers(0, history + 1, batch)
        self.params["num_biases"] = rng.integers(0, biases + 1, batch)

    def desc(self, E, pad=0, shift=0):
        bits = self.bits.view(np.int16) if self.bf16 else self.logits
        rows, wide = len(bits), self.vocab + pad
        room = torch.zeros(rows * wide + shift + 16, dtype=torch.int16 if self.bf16 else torch.float32, device="cuda")
        view = room[shift:shift + rows * wide].view(rows, wide)
        view[:, :self.vocab] = _dev(bits)
        logits = view.view(torch.bfloat16) if self.bf16 and shift == 0 and wide % 2 == 0 else view
        return E.LogitsDesc(self.drafts, self.vocab, logits, wide, _dev(self.params.view(np.uint8)), _dev(self.history),
                            self.history.shape[1], _dev(self.tokens), _dev(self.bias_tokens), _dev(self.bias_values),
                            self.bias_tokens.shape[1], _dev(self.masks.view(np.int32)), self.masks.shape[1], len(self.masks),
                            _dev(self.mask_rows), bf16=int(self.bf16))


def _dtype():
    from paper_2505_21889_amd import binding
    return binding.SAMPLING_DTYPE


def _run(E, rows, pad=0, shift=0, stream=None):
    desc = rows.desc(E, pad, shift)
    wide = rows.vocab + pad
    out = torch.full((len(rows.logits), wide), -7.0, device="cuda")
    size = E.efim_logit_workspace_bytes(desc)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    E.efim_logit_probs(desc, out, wide, ws, size, stream=stream)
    torch.cuda.synchronize()
    out = out.cpu().numpy()
    assert (out[:, rows.vocab:] == -7.0).all(), "what is behind a row stays as it was"
    return out[:, :rows.vocab]


def _check(E, rows, **how):
    got = _run(E, rows, **how).astype(np.float64)
    want, far = M.probs(rows.drafts, rows.logits, rows.params, rows.history, rows.tokens, rows.bias_tokens, rows.bias_values,
                        rows.masks, rows.mask_rows)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    # z is the same in both.  Its distance from the largest and the factor to powers of two are three roundings of 2^-24, in the
    # element, in its chunk's rescaling and in the terms of the sum (where what is far weighs little: under 32 counts); powers of two
    # are within 2^-23; the sum goes over fewer than 64 additions and the division and product are two
    bound = want * 2.0 ** -24 * (6 * far + 3 * 32 + 64 + 16) + 2.0 ** -125
    fine = ~np.isnan(want)
    off = np.abs(got - want)[fine] - bound[fine]
    assert off.max(initial=0.0) <= 0.0, off.max()
    return got


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 31, 32, 33, 1000, 2048, 4095, 4096, 4097, 10007])
def test_vocabularies(E, vocab, bf16):
    _check(E, Rows([0, 3, 1], vocab, seed=vocab, bf16=bf16))


@pytest.mark.parametrize("drafts", [[0], [63], [5, 0, 15, 2], [0] * 40, [7] * 9])
def test_drafted_tokens_count_for_the_rows_behind_them(E, drafts):
    rows = Rows(drafts, 5003 if len(drafts) < 9 else 700, seed=len(drafts), masks=1)
    rows.tokens[:] = rows.tokens % 3  # the same few again and again
    rows.params["frequency"], rows.params["temperature"] = 0.3, 1.0
    _check(E, rows)


def test_many_rows_to_a_workgroup(E):
    """So many requests that a workgroup goes through all rows of one."""
    _check(E, Rows([2, 0, 5] * 180, 8200, seed=3, history=9, biases=2))


def test_more_requests_than_a_launch_takes(E):
    _check(E, Rows(([1, 0] * 300), 70, seed=4, history=9, biases=2))


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 2), (61, 5)])
@pytest.mark.parametrize("bf16", [True, False])
def test_strides_and_rows_that_begin_anywhere(E, pad, shift, bf16):
    _check(E, Rows([4, 0, 2], 4999, seed=pad, bf16=bf16), pad=pad, shift=shift)


def test_masks_that_leave_nothing_or_one(E):
    rows = Rows([3], 4100, seed=6, biases=0, heats=(1.0,))
    rows.masks[:] = 0
    rows.masks[1, 4099 // 32] = 1 << (4099 % 32)
    rows.mask_rows[:] = [0, 1, 3, 2 ** 31 - 1]  # none allowed, the last token, and masks that there are not
    for heat in (1.0, 0.0, float("nan"), -2.0):
        rows.params["temperature"] = heat
        got = _check(E, rows)
        assert got[0].sum() == got[2].sum() == got[3].sum() == 0 and got[1, 4099] == 1 and got[1].sum() == 1


def test_infinities_and_numbers_that_are_none(E):
    vocab = 4200
    for heat in (1.0, 0.0):
        rows = Rows([5], vocab, seed=7, bf16=False, biases=0, masks=1)
        rows.params["temperature"] = heat
        rows.mask_rows[:] = -1
        rows.masks[0] = 0xFFFFFFFF
        rows.masks[0, 3] = 0  # tokens 96 .. 127 are not allowed
        for i, bad in enumerate((np.nan, np.inf, -np.inf)):
            rows.logits[i, [5, 100, 4199]] = bad     # allowed
            rows.logits[3 + i, 96:128] = bad         # masked: does not matter
            rows.mask_rows[3 + i] = 0
        got = _check(E, rows)
        assert np.isfinite(got[2:]).all()
        assert heat == 0.0 or np.isnan(got[:2]).all()
    rows = Rows([1], vocab, seed=8, bf16=False, biases=0, history=0)
    rows.params["repetition"], rows.mask_rows[:] = 1.0, -1
    rows.logits[:] = -np.inf
    rows.logits[1] = np.nan
    for heat in (1.0, 0.0):
        rows.params["temperature"] = heat
        got = _check(E, rows)
        assert (got[0] == 0).all()


def test_the_first_of_equal_tokens_is_the_greedy_one(E):
    rows = Rows([2], 9000, seed=9, bf16=False, biases=0, masks=1, history=0)
    rows.params["temperature"], rows.mask_rows[:] = 0.0, -1
    rows.params["frequency"] = rows.params["presence"] = 0.0
    rows.params["repetition"] = 1.0
    rows.logits[0] = 1.5
    rows.logits[1, [8999, 4500, 4400]] = 99.0
    rows.logits[2, [0, 8192]] = 99.0
    got = _check(E, rows)
    assert [int(r.argmax()) for r in got] == [0, 4400, 0] and (got.sum(1) == 1).all()


@pytest.mark.parametrize("heat", [1e-3, 2.0 ** -100, 2.0 ** -120, 1e-45, 1e3, float("inf")])
def test_temperatures_far_from_one(E, heat):
    rows = Rows([2, 0], 5000, seed=10, masks=1)
    rows.params["temperature"] = heat
    _check(E, rows)


def test_counts_and_tokens_outside_their_ranges(E):
    rows = Rows([3, 2, 1, 0], 3000, seed=11)
    rows.history[:, ::3] = [-1, 3000, 2 ** 31 - 1, -2 ** 31][0]
    rows.history[1, 5], rows.history[2, 7], rows.history[3, 2] = 3000, 2 ** 31 - 1, -2 ** 31
    rows.tokens[[0, 4]] = [-5, 3000]
    rows.bias_tokens[:, 0] = [-1, 3000, 2 ** 31 - 1, 4]
    rows.params["history_len"] = [10 ** 6, -3, 40, 39]
    rows.params["prompt_len"] = [10 ** 6, 5, -7, 10]
    rows.params["num_biases"] = [100, -1, 6, 6]
    _check(E, rows)


def test_of_several_biases_of_a_token_the_last_counts(E):
    rows = Rows([1], 5000, seed=12, biases=300)
    rows.bias_tokens[:] = np.arange(300) % 7 + 4094
    rows.params["num_biases"], rows.params["temperature"] = 299, 1.0
    _check(E, rows)


def test_a_long_history(E):
    rows = Rows([2, 2], 4500, seed=13, history=20000)
    rows.params["history_len"], rows.params["prompt_len"] = 20000, [0, 15000]
    _check(E, rows)


def test_what_is_left_out(E):
    """No parameters, no history, no biases, no masks: the plain softmax; masks without rows of theirs: all is allowed."""
    rows = Rows([2, 0], 4500, seed=14)
    out = torch.empty(4, 4500, device="cuda")
    x = _dev(rows.logits)
    for masks in ({}, {"masks": _dev(rows.masks.view(np.int32)), "mask_stride": rows.masks.shape[1], "num_masks": len(rows.masks)}):
        desc = E.LogitsDesc(rows.drafts, 4500, x, 4500, draft_tokens=_dev(rows.tokens), **masks)
        size = E.efim_logit_workspace_bytes(desc)
        E.efim_logit_probs(desc, out, 4500, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
        want = torch.softmax(x.double(), -1)
        assert ((out.double() - want).abs() <= want * 2.0 ** -24 * 400).all()


def test_in_place(E):
    rows = Rows([4, 1], 6001, seed=15, bf16=False)
    want = _run(E, rows)
    desc = rows.desc(E)
    size = E.efim_logit_workspace_bytes(desc)
    logits = desc.tensors[0]
    E.efim_logit_probs(desc, logits, 6001, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
    assert np.array_equal(logits.cpu().numpy(), want)


def test_captured_into_a_graph_and_on_another_stream(E):
    """A replay reads logits, histories and parameters anew; its drafted tokens are verified behind it."""
    first, other = Rows([3, 0, 5], 5003, seed=16), Rows([3, 0, 5], 5003, seed=17)
    desc = first.desc(E)
    size = E.efim_logit_workspace_bytes(desc)
    ws, out = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(11, 5003, device="cuda")
    uniforms = np.random.default_rng(1).random(11, dtype=np.float32)
    u, tokens, accepted = _dev(uniforms), torch.empty(11, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    room = E.efim_verify_workspace_bytes(3, 5003)
    vws = torch.empty(room, dtype=torch.uint8, device="cuda")

    def step(stream=None):
        E.efim_logit_probs(desc, out, 5003, ws, size, stream=stream)
        E.efim_verify_drafts(first.drafts, 5003, out, 5003, None, 5003, desc.tensors[3], u, tokens, accepted, vws, room, stream=stream)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for rows in (first, other, first):
        for to, x in zip(desc.tensors, rows.desc(E).tensors):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        probs, drawn, kept = out.cpu().numpy(), tokens.cpu().numpy(), accepted.cpu().numpy()
        assert np.array_equal(probs, _run(E, rows))
        want = S.verify(rows.drafts, probs, None, rows.tokens, uniforms)
        assert np.array_equal(drawn, want[0]) and np.array_equal(kept, want[1])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert np.array_equal(_run(E, other, stream=stream), _run(E, other))
