"""efim_logit_probs beyond what one turn of its loops takes: vocabularies of several windows of marks (131072 tokens each), rows of more than
64 chunks (of 1024), and more listed tokens in a window than are counted in LDS (8192).

The bound of the small tests holds here as it stands.  A row of up to 256 chunks is summed by lanes that take up to four of them: per lane
16 additions in a chunk, 6 exchanges, 4 chunks, 6 exchanges, 32 of the 64 additions that it counts; up to 4 rescalings instead of
one are 4 powers of two more, 2 counts each, which the other 32 cover, and their distances add up to the one that it has."""
import numpy as np
import pytest

from test_gpu_logit_probs import E, Rows, _check, _run  # noqa: F401 (E is a fixture)

pytestmark = pytest.mark.gpu

WINDOW = 131072


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("vocab", [65536, 65537, 66561, 131071, 131072, 131073, 132100, 140003, 262144, 262147])
def test_vocabularies(E, vocab, bf16):  # noqa: F811
    rows = Rows([2, 0], vocab, seed=vocab, bf16=bf16, history=300, biases=40, masks=2)
    # tokens of every window, next to its borders too
    rng = np.random.default_rng(vocab)
    rows.history[:] = rng.integers(0, vocab, rows.history.shape)
    near = np.array([t for t in (0, 1023, 1024, 65535, 65536, WINDOW - 1, WINDOW, WINDOW + 31, vocab - 1) if t < vocab])
    rows.history[:, :len(near)] = near
    rows.bias_tokens[:, -len(near):] = near
    rows.tokens[:] = [vocab - 1, min(WINDOW, vocab - 1)]
    rows.params["history_len"], rows.params["prompt_len"], rows.params["num_biases"] = 300, [0, 150], 40
    rows.params["temperature"] = [0.8, 1.5]
    _check(E, rows)


@pytest.mark.parametrize("tokens", [(3 * 1024 + 5, 67 * 1024 + 5), (67 * 1024 + 5, 3 * 1024 + 6), (65535, 65536), (131071, 131072), (131072, 139999),
                                    (70000, 5, 134000), (0, 65536, 131072), (140002,), (64 * 1024, 128 * 1024)])
@pytest.mark.parametrize("bf16", [True, False])
def test_the_first_of_equal_tokens_is_the_greedy_one(E, tokens, bf16):  # noqa: F811
    """Equal largest ones in one chunk's lane and in different ones, in one window and in both; by bias, by the logit itself."""
    vocab = 140003
    rows = Rows([1, 0], vocab, seed=len(tokens), bf16=bf16, biases=4, masks=1, history=6, heats=(0.0,))
    rows.mask_rows[:] = -1
    rows.params["frequency"] = rows.params["presence"] = 0.0
    rows.params["repetition"] = 1.0
    for row in range(2):
        rows.logits[row, list(tokens)] = 96.0
        if bf16:
            rows.bits[row, list(tokens)] = 0x42C0
    rows.logits[2], rows.bits[2] = 1.5, 0x3FC0  # the third row's are raised by their biases
    rows.bias_tokens[1, :len(tokens)], rows.bias_values[1], rows.params["num_biases"] = tokens, 8.0, [0, len(tokens)]
    got = _check(E, rows)
    assert [int(r.argmax()) for r in got] == [min(tokens)] * 3 and (got.sum(1) == 1).all()


def _listed(rows, prompt, made):
    """History of these tokens, in an order that mixes them."""
    rng = np.random.default_rng(len(prompt))
    past = np.concatenate([rng.permutation(prompt), rng.permutation(made)])
    rows.history[:, :len(past)] = past
    rows.params["history_len"], rows.params["prompt_len"] = len(past), len(prompt)


@pytest.mark.parametrize("distinct", [8190, 8192, 8193, 12000])
@pytest.mark.parametrize("first", [0, WINDOW])
def test_more_listed_tokens_than_are_counted_in_lds(E, distinct, first):  # noqa: F811
    """On both sides of the border and in both windows; tokens of the prompt, made once and three times, drafted and biased ones among them."""
    vocab = 150001
    rows = Rows([3, 0], vocab, seed=distinct, history=20000, biases=50, masks=2)
    tokens = first + np.random.default_rng(distinct + first).permutation(15000)[:distinct]
    made = np.concatenate([tokens[distinct // 2:]] + [tokens[-1000:]] * 2)
    _listed(rows, tokens[:distinct * 2 // 3], made)
    # (no other token is listed)
    rows.tokens[:] = tokens[[5, -5, 5]]
    rows.bias_tokens[:] = np.random.default_rng(1).choice(tokens, 50)
    rows.params["num_biases"], rows.params["temperature"] = 50, [1.0, 0.9]
    rows.params["repetition"], rows.params["presence"], rows.params["frequency"] = 1.2, 0.3, 0.2
    assert len(np.unique(np.concatenate([rows.history[0, :rows.params["history_len"][0]], rows.tokens, rows.bias_tokens[0]]))) == distinct
    _check(E, rows)


def test_a_small_vocabulary_that_is_listed_throughout(E):  # noqa: F811
    rows = Rows([2], 9001, seed=2, history=10000, biases=3)
    rows.history[:] = np.random.default_rng(3).permutation(10000) % 9001
    rows.params["history_len"], rows.params["prompt_len"], rows.params["temperature"] = 10000, 4000, 1.0
    _check(E, rows)


def test_in_place_and_the_same_bits_again(E):  # noqa: F811
    """Counts in memory are whole numbers, so no order of theirs shows."""
    import torch
    rows = Rows([3, 1], 140003, seed=5, bf16=False, history=12000, biases=20)
    rows.history[:] = np.random.default_rng(6).permutation(12000)
    rows.params["history_len"], rows.params["prompt_len"] = 12000, 5000
    want = _run(E, rows)
    assert np.array_equal(_run(E, rows), want)
    desc = rows.desc(E)
    size = E.efim_logit_workspace_bytes(desc)
    logits = desc.tensors[0]
    E.efim_logit_probs(desc, logits, 140003, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
    assert np.array_equal(logits.cpu().numpy(), want)
