"""Plain CPU definitions of the operators of a step over a 4-bit cache: the format, the append, the attention, the block tables
and the probabilities of adjusted logits.

TEST INFRASTRUCTURE ONLY, as the other oracles: slow, untiled, shares no code with the HIP library.  Parity unpinned by the
paper, which models none of these.

bf16 tensors travel as ``numpy.uint16`` bit patterns, caches as ``numpy.uint8`` [pages, heads, page * (d / 2 + d / 32)].
"""
from __future__ import annotations

import numpy as np

from oracle.efim_oracle import bf16_to_f64, f64_to_bf16
from oracle.step_oracle import _softmax_mix, positions, rotate

BLOCK = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_BYTE = 255


def quantise(bits):
    """Codes [.., d] (one to a byte) and scale bytes [.., d / 32] of bf16 rows."""
    bits = np.ascontiguousarray(bits).reshape(bits.shape[:-1] + (bits.shape[-1] // BLOCK, BLOCK))
    with np.errstate(invalid="ignore"):
        x = bf16_to_f64(bits)
    fit = np.isfinite(x).all(axis=-1)
    x = np.where(fit[..., None], x, 0.0)
    most = np.abs(x).max(axis=-1)
    # the least whole s from -125 on with most <= 7 2^s
    s = np.full(most.shape, -125)
    for e in range(-125, 125):
        s = np.where((s == e) & (most > 7.0 * 2.0 ** e), e + 1, s)
    y = np.abs(x) / 2.0 ** s[..., None].astype(np.float64)
    away = np.abs(y[..., None] - LEVELS)
    # nearest level; of two as near the one with an even code
    near = away == away.min(axis=-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), near.argmax(axis=-1))
    code = np.where(fit[..., None], code + 8 * (bits >> 15), 0)
    return code.reshape(code.shape[:-2] + (code.shape[-2] * BLOCK,)).astype(np.uint8), np.where(fit, s + 127, NAN_BYTE).astype(np.uint8)


def values(codes, scales):
    """fp64 rows of codes [.., d] and scale bytes [.., d / 32]."""
    x = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    scale = np.where(scales == NAN_BYTE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(scale, BLOCK, axis=-1)


def cache_shape(pages, heads, page, d):
    return pages, heads, page * (d // 2 + d // BLOCK)


def put(cache, page, d, where, slot, codes, scales):
    """Writes rows [n, heads, ..] at pages `where` and slots `slot` [n]."""
    packed = codes[..., 0::2] | codes[..., 1::2] << 4
    for i, (at, s) in enumerate(zip(where, slot)):
        cache[at, :, s * (d // 2):(s + 1) * (d // 2)] = packed[i]
        first = page * (d // 2) + s * (d // BLOCK)
        cache[at, :, first:first + d // BLOCK] = scales[i]


def get(cache, page, d, where, slot):
    """Codes [n, heads, d] and scale bytes [n, heads, d / 32] at pages `where` and slots `slot`."""
    where, slot = np.asarray(where), np.asarray(slot)
    heads = np.arange(cache.shape[1])[None, :, None]
    packed = cache[where[:, None, None], heads, slot[:, None, None] * (d // 2) + np.arange(d // 2)]
    scales = cache[where[:, None, None], heads, page * (d // 2) + slot[:, None, None] * (d // BLOCK) + np.arange(d // BLOCK)]
    codes = np.stack([packed & 15, packed >> 4], axis=-1).reshape(packed.shape[:-1] + (d,))
    return codes, scales


def append(cached, new, table, page, q, k, v, k_cache, v_cache, inv_freq, interleaved):
    """Writes the caches in place; returns (q bits or None, what the new rows' codes stand for, of keys and of values)."""
    req, pos = positions(cached, new)
    turned = lambda x: f64_to_bf16(rotate(bf16_to_f64(x), pos, inv_freq, interleaved))
    where, slot, stored = table[req, pos // page], pos % page, []
    # (elements that are not rotated are copied: a NaN keeps its bits)
    for rows, cache in ((keep_tail(turned(k), k, 2 * len(inv_freq)), k_cache), (v, v_cache)):
        codes, scales = quantise(rows)
        put(cache, page, k.shape[-1], where, slot, codes, scales)
        stored.append(values(codes, scales))
    return (None if q is None else keep_tail(turned(q), q, 2 * len(inv_freq))), stored[0], stored[1]


def keep_tail(x, raw, rotary):
    x = x.copy()
    x[..., rotary:] = raw[..., rotary:]
    return x


def attention(cached, new, table, page, q, k_cache, v_cache, scale):
    """q bits [T, Hq, d] -> (out [T, Hq, d] fp64, mean magnitude of the values, largest sum of |q k| scale, keys) per element or row."""
    total, hq, d = q.shape
    hkv = k_cache.shape[1]
    g = hq // hkv
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    reach, keys = np.zeros((total, hq, 1)), np.zeros((total, hq, 1))
    at = 0
    with np.errstate(invalid="ignore"):
        qf = bf16_to_f64(q)
        for r, (c, n) in enumerate(zip(cached, new)):
            if n:
                t = np.arange(c + n)
                k = values(*get(k_cache, page, d, table[r, t // page], t % page))
                v = values(*get(v_cache, page, d, table[r, t // page], t % page))
                for h in range(hq):
                    x = qf[at:at + n, h]
                    out[at:at + n, h], size[at:at + n, h] = _softmax_mix(scale * (x @ k[:, h // g].T), v[:, h // g], c)
                    reach[at:at + n, h, 0] = scale * (np.abs(x) @ np.abs(k[:, h // g]).T).max(axis=1)
                    keys[at:at + n, h, 0] = c + n
            at += n
    return out, size, reach, keys


def block_tables(held, cached, new, page, table, free, count, slot_capacity):
    """(table, free, count, slots, row_start, status) behind efim_block_tables; the inputs are left alone."""
    table, free = table.copy(), free.copy()
    rows = [(int(h), int(c), int(n)) for h, c, n in zip(held, cached, new)]
    bad = any(min(row) < 0 for row in rows) or any(max(-(-h // page), -(-(c + n) // page)) > table.shape[1] for h, c, n in rows)
    slots = np.full(max(slot_capacity, 0), -1, np.int64)
    if bad or sum(n for _, _, n in rows) > 2 ** 31 - 1:
        return table, free, count, slots, np.zeros(len(rows) + 1, np.int32), -1
    start = np.concatenate([[0], np.cumsum([n for _, _, n in rows])]).astype(np.int32)
    span = [(-(-h // page), -(-(c + n) // page)) for h, c, n in rows]
    back, more = sum(max(0, h - w) for h, w in span), sum(max(0, w - h) for h, w in span)
    if count < 0 or count + back > len(free) or (slot_capacity >= 0 and start[-1] > slot_capacity):
        return table, free, count, slots, start, -1
    if more > count + back:
        return table, free, count, slots, start, more - count - back
    for r, (h, w) in enumerate(span):
        for col in range(w, h):
            free[count] = table[r, col]
            count += 1
    for r, (h, w) in enumerate(span):
        for col in range(h, w):
            count -= 1
            table[r, col] = free[count]
    at = 0
    for r, (_, c, n) in enumerate(rows):
        for pos in range(c, c + n):
            if slot_capacity >= 0:
                slots[at] = int(table[r, pos // page]) * page + pos % page
            at += 1
    return table, free, count, slots, start, 0


def probs(num_drafts, logits, params, history, drafts, bias_tokens, bias_values, masks, mask_rows):
    """logits float32 [rows, V]; params: a structured array -> (probabilities fp64, distance of z / temperature from the row's largest)."""
    vocab = logits.shape[1]
    out, far = np.zeros(logits.shape), np.zeros(logits.shape)
    row = d0 = 0
    f32 = np.float32
    with np.errstate(all="ignore"):
        for r, n in enumerate(num_drafts):
            p = params[r]
            past = history[r][:max(0, min(int(p["history_len"]), history.shape[1]))]
            prompt = max(0, min(int(p["prompt_len"]), len(past)))
            entries = max(0, min(int(p["num_biases"]), bias_tokens.shape[1]))
            for i in range(n + 1):
                seen, made = np.zeros(vocab, bool), np.zeros(vocab, np.int64)
                for t in past[:prompt]:
                    if 0 <= t < vocab:
                        seen[t] = True
                for t in list(past[prompt:]) + list(drafts[d0:d0 + i]):
                    if 0 <= t < vocab:
                        made[t] += 1
                seen |= made > 0
                z = logits[row].astype(f32).copy()
                z = np.where(seen, np.where(z > 0, z / p["repetition"], z * p["repetition"]), z).astype(f32)
                z = np.where(made > 0, (z - (p["frequency"] * made.astype(f32)).astype(f32)).astype(f32) - p["presence"], z).astype(f32)
                add = {int(t): v for t, v in zip(bias_tokens[r][:entries], bias_values[r][:entries])}
                for t, v in add.items():
                    if 0 <= t < vocab:
                        z[t] = f32(z[t] + v)
                ok = np.ones(vocab, bool)
                m = -1 if masks is None else int(mask_rows[row])
                if m >= 0:
                    ok = (masks[m][np.arange(vocab) // 32] >> (np.arange(vocab) % 32) & 1).astype(bool) if m < len(masks) else ~ok
                z = z.astype(np.float64)
                heat = float(p["temperature"])
                number = ok & ~np.isnan(z)
                top = z[number].max() if number.any() else -np.inf
                if not heat > 0:
                    if top > -np.inf:
                        out[row, int(np.flatnonzero(ok & (z == top))[0])] = 1.0
                elif ok.any():
                    heat = max(heat, 2.0 ** -100)
                    if np.isnan(z[ok]).any() or top == np.inf:
                        out[row, ok] = np.nan
                    elif top > -np.inf:
                        e = np.where(ok, np.exp((z - top) / heat), 0.0)
                        out[row] = e / e.sum()
                        far[row] = np.where(ok & np.isfinite(z), (top - z) / heat, 0.0)
                row += 1
            d0 += n
    return out, far
