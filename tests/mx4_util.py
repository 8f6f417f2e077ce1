"""Batches over a 4-bit cache for the tests, on the host."""
import numpy as np

from oracle import mx4_oracle as M
from paper_2505_21889_amd import workloads as W


class Step:
    """Lengths, block table, raw rows of the new tokens and caches that hold random rows everywhere."""

    def __init__(self, cached, new, heads=(8, 2), d=128, page=16, seed=0, sigma=1.0, filled=True):
        rng = np.random.default_rng(seed)
        self.cached, self.new = np.asarray(cached, np.int32), np.asarray(new, np.int32)
        self.hq, self.hkv, self.d, self.page = heads[0], heads[1], d, page
        self.table, self.pages = W.make_block_table(self.cached, self.new, page, rng)
        self.total = int(self.new.sum())
        self.q, self.k, self.v = (W.gaussian_bf16(rng, (self.total, h, d), sigma) for h in (self.hq, self.hkv, self.hkv))
        self.shape = M.cache_shape(self.pages, self.hkv, page, d)
        self.caches = []
        for _ in range(2):
            cache = np.full(self.shape, M.NAN_BYTE, np.uint8)  # what no row holds is no number
            if filled:
                for r, keys in enumerate(self.cached + self.new):
                    t = np.arange(keys)
                    codes, scales = M.quantise(W.gaussian_bf16(rng, (keys, self.hkv, d), sigma))
                    M.put(cache, page, d, self.table[r, t // page], t % page, codes, scales)
            self.caches.append(cache)

    def desc(self, E, table):
        return E.BatchDesc(self.cached, self.new, table, self.hq, self.hkv, self.d, self.page, self.pages)


def attention_bound(out, size, reach, keys, d):
    """How far an output may be.  Probabilities are off by half a bf16 step, 2^-8 of each, in products and normaliser alike:
    2^-8 (size + |out|) / (1 - 2^-8).  A score is a sum of d products in fp32 and a factor: (d + 4) 2^-24 of the sum of magnitudes, in
    every key's weight and in the normaliser.  Sums over the keys in fp32: a step each at most, 2^-24, in both.  The output's own
    rounding: 2^-8 of it."""
    every = size + np.abs(out)
    off = every * (2.0 ** -8 / (1 - 2.0 ** -8) + (d + 4) * 2.0 ** -23 * reach + keys * 2.0 ** -23)
    return off + 2.0 ** -8 * (np.abs(out) + off) + 1e-37
