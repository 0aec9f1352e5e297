"""Inputs and tolerances of the tests of 8-bit caches with a scale per block, of windows with sinks and of page tables."""
import numpy as np

from cache_util import Case, attention_bound
from oracle import cache_blocks_ref


class BlockCase(Case):
    """A cache with its tables.  kind: "fp16", "e4m3" or "int8"; block: tokens of a scale (0: scales per key head, or none in fp16)."""

    def __init__(self, lengths, new, q_heads, kv_heads, dim, page, kind="int8", block=0, layout="heads", seed=0):
        import torch
        super().__init__(lengths, new, q_heads, kv_heads, dim, page, kind != "fp16", layout, seed)
        self.kind, self.block = kind, block
        rng = np.random.default_rng(seed + 1000)
        if kind == "int8":
            self.k_t, self.v_t = (torch.from_numpy(rng.integers(-127, 128, self.k_t.shape).astype(np.int8)) for _ in range(2))
        if block:
            shape = (self.pages, kv_heads, page // block)
            low, high = (0.004, 0.03) if kind == "int8" else (0.03, 0.09)
            self.k_scale, self.v_scale = (rng.uniform(low, high, shape).astype(np.float32) for _ in range(2))

    def place(self, x):
        import torch
        if self.layout == "wide" and x.dtype == torch.int8:
            return super().place(x.view(torch.float8_e4m3fn)).view(torch.int8)
        return super().place(x)

    def codes(self, x):
        import torch
        return x.numpy() if self.kind == "int8" else x.view(torch.uint8).numpy()

    def expand(self, x, scale):
        """the values of a cache, float64"""
        if self.kind == "fp16":
            return x.float().numpy().astype(np.float64)
        if self.block:
            return cache_blocks_ref.expanded(self.codes(x), scale)
        return cache_blocks_ref.values(self.codes(x)) * scale.astype(np.float64)[None, :, None, None]

    def sinks_ref(self, scale, window=0, sinks=0):
        return cache_blocks_ref.attention(self.q, self.expand(self.k_t, self.k_scale), self.expand(self.v_t, self.v_scale), self.table, self.lengths,
                                          self.starts, scale, window, sinks)

    def sinks_bound(self, ref):
        """attention_bound, and with scales by block: a weight times the scale of its value is held in units of a power of two that is
        below twice the largest scale s in sight, and is off by half a last place of fp16, 2^-25 of it where it is subnormal, while the
        largest weight of its row is at least 2^7 (they add up to more): 2^-25 * 2 s / 2^7 = 2^-31 s for every key, times its code, |c| <= 448."""
        bound = attention_bound(ref)
        if self.block and self.kind != "fp16":
            top = np.max(np.where(np.isfinite(self.v_scale), np.abs(self.v_scale), 0))
            bound = bound + 2.0 ** -31 * float(top) * 448 * ref[4]
        return bound
