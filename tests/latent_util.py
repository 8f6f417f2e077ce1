"""What the tests of the latent attention's ways share: batches whose requests have one history in common, in shuffled pages,
and attention in 64 bits of chosen query rows."""
import numpy as np
import torch

import gpu_util as U
from oracle.efim_oracle import bf16_to_f64

SCALE, ROW, LATENT, PAGE = 192 ** -0.5, 576, 512, 64
NAN_BITS = 0x7FC1


class Shared:
    """Requests of given lengths over rows [longest, 576] (bit patterns): request r has the first cached[r] + new[r]."""

    def __init__(self, cached, new, rows, seed):
        self.cached, self.new = np.asarray(cached, np.int32), np.asarray(new, np.int32)
        self.keys = self.cached + self.new
        self.total = int(self.new.sum())
        pages = -(-int(self.keys.max()) // PAGE)
        order = np.random.default_rng(seed).permutation(pages + 1)[:pages]
        cache = np.full((pages + 1, PAGE, ROW), NAN_BITS, np.uint16)
        at = np.arange(self.keys.max())
        cache[order[at // PAGE], at % PAGE] = rows[at]
        self.pages = pages + 1
        self.cache = U.dev_bits(cache)
        self.table = torch.from_numpy(np.tile(order.astype(np.int32), (len(self.new), 1))).cuda()

    def visible(self):
        """Keys that each packed token sees."""
        return np.concatenate([np.arange(c + 1, c + n + 1) for c, n in zip(self.cached, self.new)])

    def desc(self, E, heads):
        return E.BatchDesc(self.cached, self.new, self.table, heads, 1, ROW, PAGE, self.pages)


def workspace(nbytes):
    return torch.full((max(nbytes, 256),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN patterns: nothing is taken from it


def absorbed(E, b, q):
    """q: bit patterns [T, H, 576] on the host; the outputs' bits."""
    desc, qd = b.desc(E, q.shape[1]), U.dev_bits(q)
    out = torch.full((b.total, q.shape[1], LATENT), NAN_BITS, dtype=torch.int16, device="cuda")
    nbytes = E.efim_latent_workspace_bytes(desc)
    E.efim_latent_attention(desc, qd, b.cache, out, SCALE, workspace(nbytes), nbytes)
    torch.cuda.synchronize()
    return U.host_bits(out)


def expanded(E, b, q, w):
    desc, qd, wd = b.desc(E, q.shape[1]), U.dev_bits(q), U.dev_bits(w)
    out = torch.full((b.total, q.shape[1], 128), NAN_BITS, dtype=torch.int16, device="cuda")
    nbytes = E.efim_latent_expanded_workspace_bytes(desc)
    E.efim_latent_attention_expanded(desc, qd, b.cache, wd, out, SCALE, workspace(nbytes), nbytes)
    torch.cuda.synchronize()
    return U.host_bits(out)


def attend(q, visible, keys, values, without=()):
    """(outputs, mean magnitude of the values) of query rows q [n, d], row i over the first visible[i] keys but for `without`."""
    scores = SCALE * (q @ keys.T)
    seen = np.arange(len(keys))[None] < np.asarray(visible)[:, None]
    seen[:, list(without)] = False
    scores = np.where(seen, scores, -np.inf)
    p = np.exp(scores - scores.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return p @ values, p @ np.abs(values)


def assert_close(got_bits, want, size, more=0.0):
    """size: the mean magnitude of the values under the softmax's weights.  A weight is rounded to bf16 (at most 2^-8 of it)
    in the sum and in the normaliser, the output once more; fp32 scores and the exponential: 1e-3 of size."""
    got = bf16_to_f64(got_bits)
    assert np.all(np.isfinite(got))
    worst = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 1e-3 + more) * size)
    assert np.all(worst <= 0), "bound passed by %.3e" % worst.max()


def relative_error(got_bits, want):
    return np.linalg.norm(bf16_to_f64(got_bits) - want) / np.linalg.norm(want)
