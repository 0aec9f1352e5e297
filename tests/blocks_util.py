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

    def sinks_ref_on_gpu(self, scale, window=0, sinks=0):
        """sinks_ref in torch's 64 bits on the GPU, some tokens at a time: for many tokens."""
        import torch
        g = self.q_heads // self.kv_heads
        k_all, v_all = (torch.from_numpy(self.expand(t, s)).cuda() for t, s in ((self.k_t, self.k_scale), (self.v_t, self.v_scale)))
        out = [torch.zeros(self.T, self.q_heads, self.dim, dtype=torch.float64) for _ in range(3)]
        mass, keys = torch.zeros(self.T, self.q_heads, 1, dtype=torch.float64), torch.zeros(self.T, 1, 1, dtype=torch.float64)
        for b, (s, e) in enumerate(zip(self.starts[:-1], self.starts[1:])):
            n = int(self.lengths[b])
            at = torch.arange(max(n, 0), device="cuda")
            number = torch.from_numpy(self.table[b]).cuda().long()[at // self.page]
            there = (number >= 0) & (number < self.pages)
            k, v = (torch.where(there[None, :, None], x[number.clamp(0, self.pages - 1), :, at % self.page].transpose(0, 1), 0.0) for x in (k_all, v_all))
            for t in range(max(int(s), int(e) - n), int(e), 64):
                t1 = min(int(e), t + 64)
                p = torch.arange(n - int(e) + t, n - int(e) + t1, device="cuda")
                seen = at <= p[:, None]
                if window:
                    seen &= (at > p[:, None] - window) | (at < sinks)
                q = torch.from_numpy(self.q[t:t1]).cuda().double().view(-1, self.kv_heads, g, self.dim)
                x = torch.einsum("thgd,hjd->thgj", q, k) * scale
                w = torch.softmax(x.masked_fill(~seen[:, None, None], -torch.inf), -1)
                size = torch.einsum("thgd,hjd->thgj", q.abs(), k.abs()).masked_fill(~seen[:, None, None], 0).amax(-1) * abs(scale)
                for to, y in zip(out, (torch.einsum("thgj,hjd->thgd", w, v), torch.einsum("thgj,hjd->thgd", w, v.abs()),
                                       torch.einsum("tj,hjd->thd", seen.double(), v.abs()).repeat_interleave(g, 1))):
                    to[t:t1] = y.reshape(-1, self.q_heads, self.dim).cpu()
                mass[t:t1], keys[t:t1, 0, 0] = size.reshape(-1, self.q_heads, 1).cpu(), seen.sum(-1).double().cpu()
        return out[0].numpy(), out[1].numpy(), out[2].numpy(), mass.numpy(), keys.numpy()

    def sinks_bound(self, ref):
        """attention_bound, and with scales by block: a weight times the scale of its value is held in units of a power of two that is
        below twice the largest scale s in sight, and is off by half a last place of fp16, 2^-25 of it where it is subnormal, while the
        largest weight of its row is at least 2^7 (they add up to more): 2^-25 * 2 s / 2^7 = 2^-31 s for every key, times its code, |c| <= 448."""
        bound = attention_bound(ref)
        if self.block and self.kind != "fp16":
            top = np.max(np.where(np.isfinite(self.v_scale), np.abs(self.v_scale), 0))
            bound = bound + 2.0 ** -31 * float(top) * 448 * ref[4]
        return bound
