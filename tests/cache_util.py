"""Inputs and tolerances of the tests of the paged key-value cache."""
import numpy as np


class Case:
    """A cache with its tables, on the host (numpy) and, through dev(), on the GPU (torch)."""

    def __init__(self, lengths, new, q_heads, kv_heads, dim, page, eight_bit=False, layout="heads", seed=0, spare_pages=3):
        import torch
        rng = np.random.default_rng(seed)
        self.lengths = np.asarray(lengths, np.int32)
        self.B, self.q_heads, self.kv_heads, self.dim, self.page = len(lengths), q_heads, kv_heads, dim, page
        self.new = [new] * self.B if isinstance(new, int) else list(new)
        self.starts = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.single = isinstance(new, int) and new == 1
        self.T = int(self.starts[-1])
        used = [-(-int(n) // page) for n in lengths]
        self.pages = sum(used) + spare_pages
        free = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((self.B, max(max(used), 1) + 1), -7, np.int32)  # (entries behind the last page are not read)
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = free[at:at + n]
            at += n
        gen = torch.Generator().manual_seed(seed)

        def cache():
            x = torch.randn(self.pages, kv_heads, page, dim, generator=gen)
            return (x * 16).to(torch.float8_e4m3fn) if eight_bit else x.to(torch.float16)
        self.k_t, self.v_t = cache(), cache()
        self.eight_bit, self.layout = eight_bit, layout
        self.k_scale = rng.uniform(0.03, 0.09, kv_heads).astype(np.float32) if eight_bit else None
        self.v_scale = rng.uniform(0.03, 0.09, kv_heads).astype(np.float32) if eight_bit else None
        self.q = (rng.standard_normal((self.T, q_heads, dim)) * 1.5).astype(np.float16)
        self.qkv = rng.standard_normal((self.T, (q_heads + 2 * kv_heads) * dim)).astype(np.float16)

    @property
    def k(self):
        return self.k_t.float().numpy()

    @property
    def v(self):
        return self.v_t.float().numpy()

    def place(self, x):
        """A cache on the GPU in this case's layout, as [pages, heads, page_size, dim]."""
        import torch
        if self.layout == "heads":
            return x.cuda()
        if self.layout == "tokens":  # [pages, page_size, heads, dim]
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        assert self.layout == "wide"  # heads of a wider buffer: pages and tokens further apart than they would have to be
        big = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + 3, x.shape[3] + 16), float("nan"), device="cuda").to(x.dtype)
        view = big[:, 1:, 2:-1, 16:]
        (view.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else view).copy_(x.view(torch.uint8).cuda() if x.dtype == torch.float8_e4m3fn else x.cuda())
        return view

    def dev(self, marlin):
        import torch
        d = dict(k_cache=self.place(self.k_t), v_cache=self.place(self.v_t), pages=torch.from_numpy(self.table).cuda(),
                 lengths=torch.from_numpy(self.lengths).cuda(),
                 workspace=torch.zeros(marlin.attention_workspace_bytes(self.dim), dtype=torch.uint8, device="cuda"))
        if not self.single:
            d["starts"] = torch.from_numpy(self.starts).cuda()
        if self.eight_bit:
            d["k_scale"], d["v_scale"] = torch.from_numpy(self.k_scale).cuda(), torch.from_numpy(self.v_scale).cuda()
        return d

    def attention_ref(self, scale, window=0):
        from oracle import attention_ref
        return attention_ref.attention(self.q, self.k, self.v, self.table, self.lengths, self.starts, scale, window, self.k_scale,
                                       self.v_scale)


def attention_bound(ref):
    """How far an fp16 result may be from the one in 64 bits, per element.

    The result is rounded once: 2^-11 of it (2^-25 where it is subnormal).  A weight is rounded to fp16 before the product with v: 2^-11
    of it, or 2^-25 of the largest weight where it is subnormal, which is at most 2^-25 of their sum: (2^-11) sum w |v| + 2^-25 sum |v|.
    A logit is a sum of head_dim <= 256 products in fp32 and two multiplications: off by at most 258 * 2^-24 of sum |q k| scale, and
    as much again for the largest one, so a weight is off by twice that, and the sum of the weights too: 4 * 258 * 2^-24 * mass.
    Exponentials are off by 2^-21 (twice), the sums over the keys, and their joining (two factors at each of up to 320 parts), by
    2^-24 per addition: (keys + 1000) * 2^-23 of sum w |v|, for numerator and denominator."""
    out, spread, small, mass, keys = ref
    return 2.0 ** -11 * np.abs(out) + 2.0 ** -25 + 2.0 ** -25 * small + \
        (2.0 ** -11 + 4 * 258 * 2.0 ** -24 * mass + 2.0 ** -20 + (keys + 1000) * 2.0 ** -23) * 1.01 * spread
