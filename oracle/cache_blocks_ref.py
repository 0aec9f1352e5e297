"""numpy restatement of page tables from lengths, of 8-bit caches with a scale for each block of tokens and key head, and of attention
through a window with sinks, in 64 bits or in the fp32 operations that the definitions name; shares no code with the library."""
import numpy as np

E4M3 = np.array([(-1) ** (c >> 7) * (((c & 7) / 8 + 1) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) * 2.0 ** -9)
                 if c & 127 != 127 else np.nan for c in range(256)])  # the value of each code
E4M3_UP = E4M3[:127]  # those that are not negative, ascending


def to_e4m3(x):
    """fp32 -> codes (uint8): to nearest, ties to the even code, 448 at most, NaN kept."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.clip(np.searchsorted(E4M3_UP, a), 1, 126)
    lo = hi - 1
    down, up = a - E4M3_UP[lo], E4M3_UP[hi] - a
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), 127, code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def to_int8(x):
    x = np.asarray(x, np.float64)
    return np.clip(np.rint(np.where(np.isnan(x), 0, x)), -127, 127).astype(np.int8)


def values(codes):
    """codes (int8, or uint8 for e4m3) -> what they stand for without their scale, float64"""
    return codes.astype(np.float64) if codes.dtype == np.int8 else E4M3[codes]


def append(codes, scales, new, sequence_pages, first, block):
    """Puts new [tokens, heads, dim] (fp32) behind the `first` tokens of a sequence into codes [pages, heads, page, dim] and scales
    [pages, heads, blocks], in place, block by block."""
    page = codes.shape[2]
    eight = codes.dtype == np.int8
    largest, to = (np.float32(127), to_int8) if eight else (np.float32(448), to_e4m3)
    at, end = first, first + len(new)
    while at < end:
        stop = min(end, (at // block + 1) * block)
        number, part = sequence_pages[at // page], at % page // block
        if 0 <= number < codes.shape[0]:
            rows = new[at - first:stop - first].astype(np.float32)
            begin = at // block * block % page
            for h in range(codes.shape[1]):
                a = np.abs(rows[:, h])
                need = np.float32(np.max(np.where(np.isfinite(a), a, 0))) * (np.float32(1) / largest)
                old = scales[number, h, part]
                fill = at % block
                begun = fill > 0 and np.isfinite(old) and old > 0
                now, shrink = (old, np.float32(1)) if begun else (need, np.float32(0))
                while now < need:
                    now, shrink = now * np.float32(2), shrink * np.float32(0.5)
                scales[number, h, part] = now
                if fill and shrink != 1:
                    kept = codes[number, h, begin:begin + fill]
                    # (a scale that is not finite and above 0 stands for codes of 0, whatever they are)
                    codes[number, h, begin:begin + fill] = to((values(kept) * np.float64(shrink)).astype(np.float32)) if begun else 0
                with np.errstate(invalid="ignore", over="ignore"):
                    if now > 0:
                        y = rows[:, h] * min(np.float32(1) / now, np.finfo(np.float32).max)
                    else:  # nothing that is finite and not 0: codes of 0, but for NaN
                        y = np.where(np.isnan(rows[:, h]), rows[:, h], np.float32(0))
                    codes[number, h, at % page:at % page + stop - at] = to(y)
        at = stop


def expanded(codes, scales):
    """[pages, heads, page, dim] as the values that they stand for, float64"""
    with np.errstate(invalid="ignore"):
        return values(codes) * np.repeat(scales.astype(np.float64), codes.shape[2] // scales.shape[2], -1)[..., None]


def attention(q, k_cache, v_cache, table, lengths, starts, scale, window=0, sinks=0):
    """As attention_ref.attention, with sinks, over caches of float64 values."""
    T, Hq, D = q.shape
    Hkv, P = k_cache.shape[1], k_cache.shape[2]
    out = np.zeros((T, Hq, D))
    spread, small, mass, keys = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, 1)), np.zeros((T, 1, 1))
    g = Hq // Hkv
    for b, (s, e) in enumerate(zip(starts[:-1], starts[1:])):
        if e == s or lengths[b] <= 0:
            continue
        every = np.arange(lengths[b])
        pages = table[b][every // P]
        there = (pages >= 0) & (pages < k_cache.shape[0])
        k, v = (np.where(there[None, :, None], x[np.where(there, pages, 0), :, every % P].transpose(1, 0, 2).astype(np.float64), 0.0)
                for x in (k_cache, v_cache))
        for t in range(s, e):
            p = lengths[b] - (e - t)
            if p < 0:
                continue
            at = every[:p + 1]
            if window:
                at = at[(at > p - window) | (at < sinks)]
            keys[t] = len(at)
            rows = q[t].reshape(Hkv, g, D).astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                x = np.einsum("hgd,hjd->hgj", rows, k[:, at]) * scale
                w = np.exp(x - x.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[t] = np.einsum("hgj,hjd->hgd", w, v[:, at]).reshape(Hq, D)
                spread[t] = np.einsum("hgj,hjd->hgd", w, np.abs(v[:, at])).reshape(Hq, D)
                small[t] = np.repeat(np.abs(v[:, at]).sum(1), g, 0)
                mass[t] = (np.einsum("hgd,hjd->hgj", np.abs(rows), np.abs(k[:, at])).max(-1) * abs(scale)).reshape(Hq, 1)
    return out, spread, small, mass, keys


def reserve(lengths, table, free, count, page, tokens, counts, keep):
    """One step, a sequence after the other: (lengths, table, free, count, starts, slots, positions), all new."""
    lengths, table, free = lengths.copy(), table.copy(), free.copy()
    starts, slots, positions = [0], np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int32)
    needed, taken, back = 0, 0, []
    for b in range(len(lengths)):
        old = int(lengths[b] if lengths[b] >= 0 else ~lengths[b])
        base = old if keep is None else min(max(int(keep[b]), 0), old)
        n = 1 if counts is None else int(counts[b])
        begin = starts[-1]
        starts.append(begin + max(n, 0))
        held, after = -(-old // page), -(-(base + max(n, 0)) // page)
        if n < 0 or held > table.shape[1] or after > table.shape[1] or base + n > 1 << 30 or begin + n > tokens:
            lengths[b] = ~old
            continue
        needed += max(after - held, 0)
        if after > held:
            if needed > count:
                lengths[b] = ~old
                continue
            for e in range(held, after):
                table[b, e] = free[count - 1 - taken]
                taken += 1
        back += list(table[b, after:held])
        lengths[b] = base + n
        for i in range(n):
            p = base + i
            positions[begin + i] = p
            slots[begin + i] = int(table[b, p // page]) * page + p % page if table[b, p // page] >= 0 else -1
    now = count - taken + len(back)
    for j, number in enumerate(back):
        if now - 1 - j < len(free):
            free[now - 1 - j] = number
    return lengths, table, free, min(now, len(free)), np.minimum(starts, 2 ** 31 - 1), slots, positions
