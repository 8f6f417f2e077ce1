"""Plain fp64 CPU definitions of the operators around a drafted step: the append with norms, the latent cache and its
attention in both forms, and the verification of drafted tokens.

TEST INFRASTRUCTURE ONLY, as the other oracles: slow, untiled, shares no code with the HIP library.  Parity unpinned by the
paper, which models none of these; each function is the textbook definition, and the tests pin it further (closed forms,
the two forms of the attention against each other, the distribution of verified tokens).

bf16 tensors travel as ``numpy.uint16`` bit patterns where a function takes or returns a cache, as fp64 values elsewhere.
"""
from __future__ import annotations

import numpy as np

from oracle.efim_oracle import bf16_to_f64, f64_to_bf16

LATENT, ROPE, NOPE, VALUE = 512, 64, 128, 128


def rms_norm(x, weight, eps):
    """x * (mean(x^2) + eps)^(-1/2) * weight over the last axis; weight None: ones."""
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    return y if weight is None else y * weight


def rotate(x, pos, inv_freq, interleaved):
    """x [T, heads, d]: pair j of the leading 2 * len(inv_freq) elements turned by pos * inv_freq[j]."""
    half = len(inv_freq)
    angle = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y = x.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def positions(cached, new):
    """(request, position) of every packed new token."""
    req = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(cached, new)] + [np.zeros(0, np.int64)]).astype(np.int64)
    return req, pos


def latent_rows(cache, table_row, page, keys):
    """Rows 0 .. keys-1 of a request, as fp64 [keys, 576], from bit patterns [pages, page, 576]."""
    at = np.arange(keys)
    return bf16_to_f64(cache[table_row[at // page], at % page])


def _softmax_mix(scores, values, cached):
    """(softmax of scores [n, keys] over the keys 0 .. cached + i) @ values, and the same of |values|."""
    n, keys = scores.shape
    scores = np.where(np.arange(keys)[None] <= cached + np.arange(n)[:, None], scores, -np.inf)
    p = np.exp(scores - scores.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    return p @ values, p @ np.abs(values)


def latent_attention(cached, new, table, page, q, cache, scale):
    """q fp64 [T, H, 576] -> (out [T, H, 512], mean magnitude of the values under the same weights)."""
    out = np.zeros(q.shape[:2] + (LATENT,))
    size, at = np.zeros_like(out), 0
    for r, (c, n) in enumerate(zip(cached, new)):
        if n:
            rows = latent_rows(cache, table[r], page, c + n)
            for h in range(q.shape[1]):
                out[at:at + n, h], size[at:at + n, h] = _softmax_mix(scale * (q[at:at + n, h] @ rows.T), rows[:, :LATENT], c)
        at += n
    return out, size


def latent_attention_expanded(cached, new, table, page, q, cache, w_kv, scale, round_expanded=True):
    """q fp64 [T, H, 192], w_kv fp64 [H, 256, 512] -> (out [T, H, 128], mean magnitude of the values)."""
    keep = (lambda x: bf16_to_f64(f64_to_bf16(x))) if round_expanded else (lambda x: x)
    out = np.zeros(q.shape[:2] + (VALUE,))
    size, at = np.zeros_like(out), 0
    for r, (c, n) in enumerate(zip(cached, new)):
        if n:
            rows = latent_rows(cache, table[r], page, c + n)
            for h in range(q.shape[1]):
                keys = np.concatenate([keep(rows[:, :LATENT] @ w_kv[h, :NOPE].T), rows[:, LATENT:]], axis=1)
                values = keep(rows[:, :LATENT] @ w_kv[h, NOPE:].T)
                out[at:at + n, h], size[at:at + n, h] = _softmax_mix(scale * (q[at:at + n, h] @ keys.T), values, c)
        at += n
    return out, size


def fixed(p):
    """Probabilities as Python integers of 2^-40: rounded down, negative and NaN 0, above one 1."""
    return [0 if not x > 0 else int(min(float(x), 1.0) * 2 ** 40) for x in p]


def verify(num_drafts, target, draft, tokens, uniforms):
    """(tokens, accepted) as efim_verify_drafts returns them; target [sum(n + 1), V] and draft [sum n, V] are float32."""
    vocab = target.shape[1]
    out, accepted, d, t = [], [], 0, 0
    for n in num_drafts:
        a = 0
        while a < n:
            x = int(tokens[d + a])
            if not 0 <= x < vocab:
                break
            q = 1.0 if draft is None else float(draft[d + a, x])
            if not float(uniforms[t + a]) * q < float(target[t + a, x]):
                break
            a += 1
        p = fixed(target[t + a])
        w = list(p)
        if a < n:
            x = int(tokens[d + a])
            if draft is None:
                if 0 <= x < vocab:
                    w[x] = 0
            else:
                w = [max(0, i - j) for i, j in zip(p, fixed(draft[d + a]))]
        if sum(w) == 0:
            w = p
        token, total = -1, sum(w)
        if total:
            u = float(uniforms[t + n])
            part = min(int(u * 2 ** 24), 2 ** 24 - 1) if u > 0 else 0
            below, upto = part * total >> 24, 0
            for j, x in enumerate(w):
                upto += x
                if upto > below:
                    token = j
                    break
        out += [int(x) for x in tokens[d:d + a]] + [token] + [-1] * (n - a)
        accepted.append(a)
        d, t = d + n, t + n + 1
    return np.array(out, np.int32), np.array(accepted, np.int32)
