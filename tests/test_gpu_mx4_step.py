"""The operators of a step over a 4-bit cache together, as a service runs them: block tables, append, attention, probabilities and
the verification of the drafted tokens, step after step."""
import numpy as np
import pytest
import torch

from oracle import mx4_oracle as M
from oracle import step_oracle as S
from oracle.efim_oracle import bf16_to_f64
from paper_2505_21889_amd import workloads as W

import gpu_util as U
import mx4_util as X

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


@pytest.mark.parametrize("d,page,heads", [(128, 16, (8, 2)), (64, 8, (4, 4))])
def test_a_service_of_four_users(d, page, heads):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_21889_amd import binding as E
    rng = np.random.default_rng(d)
    users, pages, wide, vocab, (hq, hkv) = 4, 200, 40, 4500, heads
    freq = 1.0e4 ** (-2.0 * np.arange(d // 2) / d)
    shape = M.cache_shape(pages, hkv, page, d)
    caches, want_caches = [torch.full(shape, 255, dtype=torch.uint8, device="cuda") for _ in range(2)], [np.full(shape, 255, np.uint8) for _ in range(2)]
    table, want_table = torch.zeros(users, wide, dtype=torch.int32, device="cuda"), np.zeros((users, wide), np.int32)
    want_free, want_count = rng.permutation(pages).astype(np.int32), pages
    free, count = _dev(want_free), _dev(np.array([pages], np.int32))
    start, status = torch.empty(users + 1, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    room = E.efim_block_tables_workspace_bytes(users)
    table_ws = torch.empty(room, dtype=torch.uint8, device="cuda")
    history, made = [list(rng.integers(0, vocab, n)) for n in (70, 1, 33, 150)], np.zeros(users, int)
    prompt, held, cached = [len(h) for h in history], np.zeros(users, int), np.zeros(users, int)
    drafts = [np.zeros(0, np.int32) for _ in range(users)]
    unembed = rng.standard_normal((hq * d, vocab)) / (hq * d) ** 0.5 * 3
    for step in range(5):
        # first step: the prompts; then the drawn token and the drafted ones behind it
        new = np.array([len(h) for h in history]) - cached + np.array([len(x) for x in drafts])
        total = int(new.sum())
        slots = torch.empty(total, dtype=torch.int64, device="cuda")
        E.efim_block_tables(users, *(_dev(x.astype(np.int32)) for x in (held, cached, new)), page, table, wide, free, pages, count, count, slots,
                            total, start, status, table_ws, room)
        want_table, want_free, want_count, want_slots, _, code = M.block_tables(held, cached, new, page, want_table, want_free, want_count, total)
        assert code == 0 and int(status) == 0 and int(count) == want_count
        assert np.array_equal(table.cpu().numpy(), want_table) and np.array_equal(slots.cpu().numpy(), want_slots)
        req, pos = S.positions(cached, new)
        assert np.array_equal(want_slots, want_table[req, pos // page] * page + pos % page)

        q, k, v = (W.gaussian_bf16(rng, (total, h, d), 1.0) for h in (hq, hkv, hkv))
        desc = E.BatchDesc(cached, new, table, hq, hkv, d, page, pages)
        q_dev = U.dev_bits(q)
        E.efim_rope_append_mx4(desc, q_dev, q_dev, U.dev_bits(k), U.dev_bits(v), *caches, None, None, freq, d)
        q, _, _ = M.append(cached, new, want_table, page, q, k, v, *want_caches, freq, 0)
        assert np.array_equal(U.host_bits(q_dev), q)
        for got, want in zip(caches, want_caches):
            assert np.array_equal(got.cpu().numpy(), want)
        size = E.efim_mx4_workspace_bytes(desc)
        out = torch.empty_like(q_dev)
        E.efim_extend_attention_mx4(desc, q_dev, *caches, out, 0.0, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
        got = bf16_to_f64(U.host_bits(out))
        want, spread, reach, keys = M.attention(cached, new, want_table, page, q, *want_caches, d ** -0.5)
        assert (np.abs(got - want) <= X.attention_bound(want, spread, reach, keys, d)).all()

        # rows with a token to predict behind them: the last of the known tokens and the drafted ones
        ends = np.cumsum(new)
        rows = np.concatenate([np.arange(e - 1 - len(x), e) for e, x in zip(ends, drafts)])
        logits = (got[rows].reshape(len(rows), -1) @ unembed).astype(np.float32)
        params = np.zeros(users, E.SAMPLING_DTYPE)
        params["temperature"], params["repetition"], params["presence"], params["frequency"] = [0.8, 1.0, 0.0, 1.3], 1.2, 0.2, 0.1
        params["prompt_len"], params["history_len"] = prompt, [len(h) for h in history]
        past = np.zeros((users, max(len(h) for h in history)), np.int32)
        for u, h in enumerate(history):
            past[u, :len(h)] = h
        flat = np.concatenate(drafts).astype(np.int32)
        masks = rng.integers(0, 2 ** 32, (2, (vocab + 31) // 32), dtype=np.uint32)
        mask_rows = rng.integers(-1, 2, len(rows)).astype(np.int32)
        probs = torch.empty(len(rows), vocab, device="cuda")
        none = np.zeros((users, 0), np.int32)
        numbers = [len(x) for x in drafts]
        say = E.LogitsDesc(numbers, vocab, _dev(logits), vocab, _dev(params.view(np.uint8)), _dev(past), past.shape[1], _dev(flat),
                           masks=_dev(masks.view(np.int32)), mask_stride=masks.shape[1], num_masks=2, mask_rows=_dev(mask_rows))
        size = E.efim_logit_workspace_bytes(say)
        E.efim_logit_probs(say, probs, vocab, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
        want, far = M.probs(numbers, logits, params, past, flat, none, none, masks, mask_rows)
        drawn = probs.cpu().numpy()
        assert (np.abs(drawn - want) <= want * 2.0 ** -24 * (6 * far + 176) + 2.0 ** -125).all()
        uniforms = rng.random(len(rows), dtype=np.float32)
        tokens, accepted = torch.empty(len(rows), dtype=torch.int32, device="cuda"), torch.empty(users, dtype=torch.int32, device="cuda")
        size = E.efim_verify_workspace_bytes(users, vocab)
        E.efim_verify_drafts(numbers, vocab, probs, vocab, None, vocab, say.tensors[3], _dev(uniforms), tokens, accepted,
                             torch.empty(size, dtype=torch.uint8, device="cuda"), size)
        want = S.verify(numbers, drawn, None, flat, uniforms)
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])

        at = 0
        held = cached + new  # with the pages of refused tokens, which the next step gives back
        for u, n in enumerate(numbers):
            kept = int(want[1][u])
            cached[u] = len(history[u]) + kept
            history[u] += [int(t) for t in want[0][at:at + kept + 1]]
            at += n + 1
        if step == 2:  # a user leaves, another one comes
            history[3], prompt[3], cached[3] = list(rng.integers(0, vocab, 40)), 40, 0
        drafts = [rng.integers(0, vocab, rng.integers(0, 6)).astype(np.int32) if len(history[u]) - cached[u] == 1 else np.zeros(0, np.int32) for u in range(users)]
    assert (held <= wide * page).all()
