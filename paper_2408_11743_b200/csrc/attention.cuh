// What the two attention kernels share: the ranges of the CTAs, what a row sees, results, and parts that are joined.  sm_100a only.
#pragma once
#include <limits.h>

#include <type_traits>

#include "kv_cache.cuh"

namespace marlin_b200 {

constexpr int kLeastTiles = 4;  // units that a CTA takes at least, where there are fewer than CTAs would like
constexpr uint32_t kMostUnits = 0xffffffffu;  // of a call, and more than it can have: sums that reach it stay there
constexpr int kMostCtas = kMaxWorkers;
constexpr int kItemCounters = 2 * kMostCtas;  // counters of items behind those of groups
static_assert(3 * kMostCtas * sizeof(int) <= kWsPartialOff - kWsCounterOff, "counters");
constexpr int kGroup = 8;  // parts that are joined at once; more of them are joined in groups first, each by its last CTA
constexpr float kNone = -INFINITY;
// A row's sums are kept relative to 2^base, base its largest logit (in units of log2) when the base was last moved, less kBelow.  It moves
// only when a logit exceeds it by more than kSlack, so that most tiles neither look for a maximum across lanes nor rescale.
// Weights are then at most 2^15 (fp16 ends at 2^16), and the largest of a row at least 2^7.  They are rounded to fp16 for the product
// with the values, the only operand type in which that product takes values as they lie in the cache: by 2^-11 of themselves at
// most, or by 2^-25 where they are below 2^-14.  So what a weight loses is at most 2^-11 of it or 2^-32 of the largest: a million
// keys far below one large one lose 2^-12 of the whole.  (Without kBelow, which costs nothing, they would lose 2^-5.)
constexpr float kBelow = 7.f;
constexpr float kSlack = 15.f;

// What a call may have beside a window and scales per key head, as an argument of the kernels' templates, so that calls without it stay as
// they are.  kExtra: first positions that stay visible in front of a window (sinks), blocks of rows that have tiles of their
// own, and, over 8 bits, a scale for each block of tokens and key head; kExtraInt8: the same with codes in two's complement.
enum Extra { kNoExtra, kExtra, kExtraInt8 };

constexpr int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// the same of four bytes, through the L1: neighbours in a table of scales are asked for one after the other
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  const int bytes = there ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  const int bytes = there ? 16 : 0;  // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// an arrival at `bar` when all copies that this thread has issued so far are complete
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// groups of copies of this thread, and a wait for all but its newest N
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// test builds: worker 0 leaves out an arrival that it owes (kTestWithholdMagic)
__device__ __forceinline__ bool withheld(const AttentionParams& p, bool owed) {
#ifdef MARLIN_TEST_HOOKS
  return owed && blockIdx.x == 0 && p.status[7] == kTestWithholdMagic;
#else
  return false;
#endif
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A row that does not see a key has weight 0 there, and 0 times an infinity or a NaN is NaN.  Keys that no row of a block sees are
// never loaded; values of keys that some of its rows see (those around the new tokens, and as many at the edge of a window)
// are looked through in shared memory, what is not finite is replaced by 0, and added to the rows that see it at the end.
template <bool F8>
__device__ __forceinline__ bool clean_vector(uint32_t saddr) {
  const uint4 v = lds128(saddr);
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool found = false;
  for (int i = 0; i < 4; ++i) {
    const uint32_t part = F8 ? 0xffu : 0xffffu, most = F8 ? 0x7fu : 0x7c00u;
    for (int j = 0; j < 32; j += F8 ? 8 : 16) {
      if (((w[i] >> j) & most) == most) {
        w[i] &= ~(part << j);
        found = true;
      }
    }
  }
  if (found)
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
  return found;
}

// bar.sync of some warps that also tells all of them whether `mine` is set for any of their threads
__device__ __forceinline__ bool any_of(int id, int threads, bool mine) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "barrier.cta.red.or.pred q, %2, %3, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"((uint32_t)mine), "r"(id), "r"(threads)
      : "memory");
  return r != 0;
}

// The page table is on its way to the L2 while the CTAs find their ranges: each asks for some lines of it.  (Its numbers are what the
// first copies wait for; they come in 0.3 us then instead of 0.8.)
__device__ __forceinline__ void prefetch_table(const AttentionParams& p, int threads) {
  const long long each = (long long)gridDim.x * threads;
  for (long long i = (long long)blockIdx.x * threads + threadIdx.x; i < p.table_lines; i += each)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(p.cache.table + (long long)i * 32));
}

// What a sequence asks for: new tokens [first, first + n) of the call, tiles [tile0, tile0 + tiles) of its len keys, blocks of
// rows per key head.  A sequence with new tokens has a tile at least: it writes the zeros.
// (Extra: every block of rows has as many tiles as the one that needs most of them, the tiles of the sinks, `sinks` of them, in
// front; where the others begin is its own, see Range::next.)
struct Sequence {
  int len, n, first, tile0, tiles, blocks, sinks;
};
template <int EXTRA = kNoExtra>
__device__ __forceinline__ Sequence sequence(const AttentionParams& p, int b, int rows, int tile, bool& bad) {
  Sequence s;
  s.len = cache_length(p.cache, b, bad);
  s.first = b;
  s.n = 1;
  if (p.starts) {
    const int from = min(max(load(p.starts + b), 0), p.tokens), to = min(max(load(p.starts + b + 1), from), p.tokens);
    s.first = from;
    s.n = to - from;
  }
  s.blocks = (s.n * p.group + rows - 1) / rows;
  if (EXTRA != kNoExtra) {
    const int total = max(1, (s.len + tile - 1) / tile);
    s.tile0 = s.sinks = 0;
    s.tiles = total;
    if (p.window) {
      s.sinks = min(total, (min(p.sinks, s.len) + tile - 1) / tile);
      if (s.blocks <= 1) {
        s.tiles = s.sinks + total - max(s.sinks, max(0, s.len - s.n - p.window + 1) / tile);
      } else {  // tokens that the rows of a block can belong to, keys that these see, tiles that so many keys can lie in
        const int tokens = rows % p.group ? (rows + p.group - 2) / p.group + 1 : rows / p.group, keys = p.window + tokens - 1;
        s.tiles = min(total, s.sinks + (keys + tile - 2) / tile + 1);
      }
    }
    return s;
  }
  s.tile0 = (p.window ? max(0, s.len - s.n - p.window + 1) : 0) / tile;
  s.tiles = max(1, (s.len + tile - 1) / tile - s.tile0);
  return s;
}

// The ranges of the CTAs.  What is numbered are the items (the tiles of one block of rows), each as `lead` units and one unit per tile: an
// item has a cost of its own beside its tiles (its Q, the sums of its warps that meet), and a CTA with many short ones would end
// late.  Worker w of W begins at unit w * (U / W) + min(w, U % W).  A range that would begin within the lead, or within `snap` tiles of
// the beginning or the end of an item, begins there instead: a part of an item costs a round trip through the workspace, which
// is worth a tile or two where a CTA has few.
struct Stripes {
  uint32_t total, workers, size, more, snap, lead;
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * size + min(w, more); }
  __device__ __forceinline__ uint32_t owner(uint32_t x) const {  // whose range, before any move, holds unit x
    const uint32_t wide = more * (size + 1);
    return x < wide ? x / (size + 1) : more + (x - wide) / size;
  }
  // boundary x of the ranges where it lies inside of item [i0, i1)
  __device__ __forceinline__ uint32_t moved(uint32_t x, uint32_t i0, uint32_t i1) const {
    if (x <= i0 || x >= i1) return x;
    if (x - i0 <= lead || (x - i0 <= lead + snap && x - i0 - lead <= i1 - x)) return i0;
    return i1 - x <= snap ? i1 : x;
  }
};

// One segment of a CTA's range: tiles [tile, tile + nt) of (sequence b, key head h, rows row0 .. row0 + rows - 1); row r is query
// head h * group + r % group of new token r / group.  Row r sees the positions [high - window, high) (all below high without a
// window), high = base_high + its token.  CTAs c0 .. c1 have tiles of the item.  nt = 0: there are no more segments.
struct Segment {
  int b, h, tile, nt, row0, rows, base_high, n, first, c0, c1;
};
// Extra: x.tile counts from the first tile of the item; of these the first `sinks` are the first of the sequence, the others lie `gap`
// further on.  (A row then sees the positions below `sinks` of the call, too.)
struct SegmentWithGap : Segment {
  int sinks, gap;
};
template <int EXTRA>
using SegmentOf = std::conditional_t<EXTRA == kNoExtra, Segment, SegmentWithGap>;
// tile i of the segment, in tiles of the sequence
template <int EXTRA>
__device__ __forceinline__ int tile_of(const SegmentOf<EXTRA>& x, int i) {
  int t = x.tile + i;
  if constexpr (EXTRA != kNoExtra) t += t >= x.sinks ? x.gap : 0;
  return t;
}
// positions that some row of a segment sees: [low_min, high_max), that all of them see: [low_max, high_min)
struct Visible {
  int low_min, low_max, high_min, high_max;
};
__device__ __forceinline__ Visible visible(const AttentionParams& p, const Segment& x) {
  Visible v;
  v.high_min = v.high_max = x.base_high;
  if (x.n > 1) {
    v.high_min += x.row0 / p.group;
    v.high_max += (x.row0 + x.rows - 1) / p.group;
  }
  v.low_min = p.window ? max(0, v.high_min - p.window) : 0;
  v.low_max = p.window ? max(0, v.high_max - p.window) : 0;
  return v;
}

// The segments of this CTA's range one after the other, as a whole warp follows them.  ROWS: of a block; TILE: keys of a tile;
// LEAD: what an item costs beside its tiles, in tiles.
template <int ROWS, int TILE, int LEAD, int EXTRA = kNoExtra>
struct Range {
  Stripes stripes;
  Sequence s;
  uint32_t at, end, skip;  // units; skip: those of the item in front of `at`
  int b, item;
  bool more;

  __device__ __forceinline__ void begin(const AttentionParams& p) {
    const KvCacheView& c = p.cache;
    const int lane = threadIdx.x & 31;
    // lane i counts the tiles of sequences [i * per, (i + 1) * per)
    const int per = (c.sequences + 31) / 32;
    uint32_t mine = 0;
    bool bad = false;
    for (int i = lane * per; i < min(c.sequences, (lane + 1) * per); ++i) {
      const Sequence s = sequence<EXTRA>(p, i, ROWS, TILE, bad);
      const unsigned long long units = (unsigned long long)c.kv_heads * s.blocks * (s.tiles + LEAD) + mine;
      mine = (uint32_t)min(units, (unsigned long long)kMostUnits);
    }
    if (bad) report_cache(p.status);
    uint32_t before = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t x = __shfl_up_sync(~0u, before, d);
      if (lane >= d) before = (uint32_t)min((unsigned long long)before + x, (unsigned long long)kMostUnits);
    }
    stripes.total = __shfl_sync(~0u, before, 31);
    before -= mine;
    more = stripes.total > 0;
    // More than are numbered (40 s of work with heads of 128 elements, several with the smallest) is refused.  (In 64 bits, counted from
    // the beginning of a CTA's own range, there need be no limit, but the code around this and the order that it leaves the tcgen05
    // kernel's in made prompts of 2048 tokens 10 % slower, with a window 25 %.)
    if (stripes.total == kMostUnits) {
      report_cache(p.status);
      more = false;
    }
    stripes.workers = min(gridDim.x, max(1u, stripes.total / kLeastTiles));
    more = more && blockIdx.x < stripes.workers;
    stripes.size = stripes.total / stripes.workers;
    stripes.more = stripes.total % stripes.workers;
    stripes.snap = stripes.size < 8 ? 2 : stripes.size < 48 ? 1 : 0;
    stripes.lead = LEAD;
    at = stripes.begin(blockIdx.x);
    end = stripes.begin(blockIdx.x + 1);
    skip = 0;
    b = item = 0;
    if (more) {  // where the range begins: (sequence, item of it, tile of that)
      const int owner = __ffs(__ballot_sync(~0u, mine > 0 && before <= at && at < before + mine)) - 1;
      b = owner * per;
      uint32_t off = at - __shfl_sync(~0u, before, owner);
      for (;; ++b) {
        s = sequence<EXTRA>(p, b, ROWS, TILE, bad);
        const uint32_t units = (uint32_t)c.kv_heads * s.blocks * (s.tiles + LEAD);
        if (off < units) break;
        off -= units;
      }
      const uint32_t units = s.tiles + LEAD;
      item = (int)(off / units);
      skip = off - item * units;
      const uint32_t to = stripes.moved(at, at - skip, at - skip + units);
      skip += to - at;
      at = to;
    }
  }

  // the next one; nt = 0: there is none
  __device__ __forceinline__ SegmentOf<EXTRA> next(const AttentionParams& p) {
    const KvCacheView& c = p.cache;
    if (more && skip == (uint32_t)s.tiles + LEAD) {
      more = at < end;
      if (more) {
        skip = 0;
        if (++item == c.kv_heads * s.blocks) {
          item = 0;
          bool bad = false;  // (reported by begin())
          do s = sequence<EXTRA>(p, ++b, ROWS, TILE, bad);
          while (s.blocks == 0);
        }
      }
    }
    SegmentOf<EXTRA> x = {};
    if (more) {
      const uint32_t i0 = at - skip, i1 = i0 + LEAD + s.tiles, to = min(stripes.moved(end, i0, i1), i1);
      if (at < to) {
        x.b = b;
        x.h = item / s.blocks;
        const int from = skip ? (int)skip - LEAD : 0;
        x.tile = s.tile0 + from;
        x.nt = (int)(to - i0) - LEAD - from;
        x.row0 = (item - x.h * s.blocks) * ROWS;
        x.rows = min(ROWS, s.n * p.group - x.row0);
        x.base_high = s.len - s.n + 1;
        x.n = s.n;
        x.first = s.first;
        if constexpr (EXTRA != kNoExtra) {  // (as many tiles as there are for every block: the last ones end with the sequence)
          const int low = p.window ? max(0, x.base_high + x.row0 / p.group - p.window) : 0;
          const int last = max(1, (s.len + TILE - 1) / TILE) - (s.tiles - s.sinks);
          x.sinks = s.sinks;
          x.gap = min(max(low / TILE, s.sinks), last) - s.sinks;
        }
        uint32_t c0 = blockIdx.x, c1 = blockIdx.x;
        if (x.nt != s.tiles) {
          c0 = stripes.owner(i0);
          while (c0 + 1 < stripes.workers && stripes.begin(c0 + 1) < i1 && stripes.moved(stripes.begin(c0 + 1), i0, i1) == i0) ++c0;
          c1 = stripes.owner(i1 - 1);
          while (stripes.begin(c1) > i0 && stripes.moved(stripes.begin(c1), i0, i1) == i1) --c1;
        }
        x.c0 = (int)c0;
        x.c1 = (int)c1;
      }
      skip += to - at;
      at = to;
    }
    return x;
  }
};

// new token of the segment's sequence that row r belongs to (a division only where there are several)
__device__ __forceinline__ int token_of(const AttentionParams& p, const Segment& x, int r) {
  return x.n > 1 ? (x.row0 + r) / p.group : 0;
}
// Row r, elements d .. d + 3 of a result: sums over the sum of the weights, zeros where the row sees nothing.
__device__ __forceinline__ void write_four(const AttentionParams& p, const Segment& x, int r, int d, float4 z, float li) {
  const int token = token_of(p, x, r), head = x.h * p.group + x.row0 + r - token * p.group;
  const bool nothing = x.base_high + token <= 0;
  const float f = nothing ? 0.f : (p.cache.v_scale ? load(p.cache.v_scale + x.h) : 1.f) / li;
  if (nothing) z = make_float4(0.f, 0.f, 0.f, 0.f);
  uint2 two;
  two.x = half2_bits(z.x * f, z.y * f);
  two.y = half2_bits(z.z * f, z.w * f);
  *reinterpret_cast<uint2*>(p.out + ((long long)(x.first + token) * p.q_heads + head) * p.cache.head_dim + d) = two;
}

// The value of element d at position pos of (sequence b, head h) if it is not finite, otherwise 0.
template <bool F8>
__device__ __forceinline__ float if_not_finite(const AttentionParams& p, int b, int h, int pos, int d) {
  const KvCacheView& c = p.cache;
  const long long off = cache_offset(c, load(c.table + b * c.table_stride + (pos >> c.page_shift)), h, pos, p.status);
  if (off < 0) return 0.f;
  float v;
  if (F8) {
    const uint32_t two = e4m3x2_to_f16x2(static_cast<const uint8_t*>(c.v)[off + d]);
    v = __low2float(*reinterpret_cast<const __half2*>(&two));
  } else {
    v = __half2float(static_cast<const __half*>(c.v)[off + d]);
  }
  return isfinite(v) ? 0.f : v;
}
// What was left out of the products of a segment, for element d of row r: the values that are not finite among the keys that some rows
// see and others do not.
template <bool F8>
__device__ __forceinline__ float not_finite_sum(const AttentionParams& p, const Segment& x, const Visible& sees, int tile_keys, int r, int d) {
  const KvCacheView& c = p.cache;
  const int high = x.base_high + token_of(p, x, r), low = p.window ? max(0, high - p.window) : 0;
  float sum = 0.f;
  if (d >= c.head_dim) return sum;
#pragma unroll 1
  for (int pos = max(low, x.tile * tile_keys); pos < min(high, (x.tile + x.nt) * tile_keys); ++pos) {
    if (pos >= sees.low_max && pos < sees.high_min) {  // (every row sees these: they were left where they are)
      pos = sees.high_min - 1;
      continue;
    }
    sum += if_not_finite<F8>(p, x.b, x.h, pos, d);
  }
  return sum;
}
// The same with sinks, which every row sees: from the edge of the window, as far as they are not sinks, and around the new tokens.
template <bool F8>
__device__ __forceinline__ float not_finite_sum(const AttentionParams& p, const SegmentWithGap& x, const Visible& sees, int tile_keys, int r, int d) {
  const int high = x.base_high + token_of(p, x, r), low = p.window ? max(0, high - p.window) : 0;
  float sum = 0.f;
  if (d >= p.cache.head_dim) return sum;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const int from = part ? sees.high_min : max(sees.low_min, p.sinks), to = part ? sees.high_max : min(sees.low_max, sees.high_min);
#pragma unroll 1
    for (int pos = max(from, 0); pos < to; ++pos) {
      const int tile = pos / tile_keys, at = tile < x.sinks ? tile : tile - x.gap;
      const bool here = (tile < x.sinks || tile >= x.sinks + x.gap) && at >= x.tile && at < x.tile + x.nt;
      if (here && pos < high && (pos >= low || pos < p.sinks)) sum += if_not_finite<F8>(p, x.b, x.h, pos, d);
    }
  }
  return sum;
}
// Whether some row of a segment sees a key: from its window on, or among the sinks.
template <int EXTRA>
__device__ __forceinline__ bool seen_by_some(const AttentionParams& p, int key, int low, int high) {
  return key < high && (key >= low || (EXTRA != kNoExtra && key < p.sinks));
}
// Whether all of `count` keys from key0 on are (all in the window or all sinks).
template <int EXTRA>
__device__ __forceinline__ bool all_seen_by_some(const AttentionParams& p, int key0, int count, int low, int high) {
  return key0 + count <= high && (key0 >= low || (EXTRA != kNoExtra && key0 + count <= p.sinks));
}
// where the scale of a token lies, from the number of its page (which is there)
__device__ __forceinline__ long long scale_offset(const AttentionParams& p, int page, int h, int pos) {
  const KvScalesView& s = p.scales;
  return page * s.s_page + h * s.s_head + ((pos & ((1 << p.cache.page_shift) - 1)) >> s.block_shift) * s.s_block;
}
static __device__ const float kScaleOfOne = 1.f;  // where a cache has no scales
// The least power of two that is not below x > 0, between 2^-126 and 2^127.
__device__ __forceinline__ float power_above(float x) {
  const uint32_t bits = __float_as_uint(x), up = (bits & 0x7f800000u) + (bits & 0x7fffffu ? 0x800000u : 0u);
  return __uint_as_float(min(max(up, 0x800000u), 254u << 23));
}

// ---- parts of an item in the workspace -----------------------------------------------------------
// Rows of DP sums, their base, the sum of their weights, and two floats that are not used.  A CTA has parts of at most two
// items that it shares: one that it begins (x.c0 is the CTA), one that it goes on with.
constexpr int part_line(int dp) { return dp + 4; }
__device__ __forceinline__ float* part_of(const AttentionParams& p, const Segment& x, uint32_t cta, int rows, int dp) {
  return p.partials + (size_t)(2 * cta + (cta == (uint32_t)x.c0)) * rows * part_line(dp);
}

// The last CTA of a group of parts joins the group, the last group the item, in the order of the keys.  For the THREADS threads
// (tid 0 .. THREADS - 1) that `meet` brings together; ml: room for ROWS pairs; kAtOnce, kBatch: vectors
// of a thread, and parts, whose loads are on their way together.  false: a wait ran out.
template <int ROWS, int DP, int THREADS, int kAtOnce, int kBatch, class Meet, class WriteOut>
__device__ __forceinline__ bool join_parts(const AttentionParams& p, const Segment& x, int tid, int* arrived, float2* ml, Meet meet,
                                           WriteOut write_out) {
  constexpr int kLine = part_line(DP);
  const uint32_t c0 = x.c0, c1 = x.c1;
  const int rows = x.rows;
  uint32_t first = c0 + (blockIdx.x - c0) / kGroup * kGroup, stride = 1;
  int count = (int)min((uint32_t)kGroup, c1 + 1 - first);
  const int groups = (int)(c1 - c0) / kGroup + 1;
  int* counter = p.counters + 2 * first + (first == c0);  // (a CTA may be the first of a group of each item that it shares)
#pragma unroll 1
  for (;;) {
    if (!meet()) return false;  // (all parts of the CTA are written; the release below carries them)
    if (tid == 0) *arrived = atom_add_acq_rel_gpu(counter, 1);
    if (!meet()) return false;
    if (*(volatile int*)arrived != count - 1) return true;
    if (tid == 0) *counter = 0;
    const bool last = groups == 1 || stride > 1;
#pragma unroll 1
    for (int i0 = tid; i0 < rows * (DP / 4); i0 += kAtOnce * THREADS) {
      float mi[kAtOnce], li[kAtOnce];
      float4 z[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        mi[e] = kNone;
        li[e] = 0.f;
        z[e] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll 1
      for (int w0 = 0; w0 < count; w0 += kBatch) {
        float2 sums[kAtOnce][kBatch];
        float4 u[kAtOnce][kBatch];
#pragma unroll
        for (int t = 0; t < kBatch; ++t) {
          if (w0 + t >= count) break;
          const float* part = part_of(p, x, first + (w0 + t) * stride, ROWS, DP);
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            const int i = min(i0 + e * THREADS, rows * (DP / 4) - 1), r = i / (DP / 4), d = (i % (DP / 4)) * 4;
            sums[e][t] = __ldcg(reinterpret_cast<const float2*>(part + r * kLine + DP));
            u[e][t] = ld_cg_f4(reinterpret_cast<const float4*>(part + r * kLine + d));
          }
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
          float top = mi[e];
#pragma unroll
          for (int t = 0; t < kBatch; ++t)
            if (w0 + t < count) top = fmaxf(top, sums[e][t].x);
          const float base = top == kNone ? 0.f : top, old = exp2_fast(mi[e] - base);
          mi[e] = top;
          li[e] *= old;
          z[e].x *= old; z[e].y *= old; z[e].z *= old; z[e].w *= old;
#pragma unroll
          for (int t = 0; t < kBatch; ++t) {
            if (w0 + t >= count) break;
            const float f = exp2_fast(sums[e][t].x - base);
            li[e] += sums[e][t].y * f;
            z[e].x += u[e][t].x * f; z[e].y += u[e][t].y * f; z[e].z += u[e][t].z * f; z[e].w += u[e][t].w * f;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        const int i = i0 + e * THREADS, r = i / (DP / 4), d = (i % (DP / 4)) * 4;
        if (i >= rows * (DP / 4) || d >= p.cache.head_dim) continue;
        if (last) {
          write_out(r, d, z[e], li[e]);
        } else {  // the sums of a group take the place of its first part; its base and weight when everybody has read them
          *reinterpret_cast<float4*>(part_of(p, x, first, ROWS, DP) + r * kLine + d) = z[e];
          if (d == 0) ml[r] = make_float2(mi[e], li[e]);
        }
      }
    }
    if (last) return true;
    if (!meet()) return false;
    for (int r = tid; r < rows; r += THREADS)
      *reinterpret_cast<float2*>(part_of(p, x, first, ROWS, DP) + r * kLine + DP) = ml[r];
    counter = p.counters + kItemCounters + c0;
    first = c0;
    stride = kGroup;
    count = groups;
  }
}

// ---- host ----------------------------------------------------------------------------------------
// Rows of a key head that most sequences of the call have at most; one with more takes several blocks of rows, and reads its keys again for
// each.  Where the tokens are not the same number for every sequence, some have more than the mean: up to twice as many are expected.
inline long long usual_rows(const AttentionParams& p) {
  const long long mean = (p.tokens + p.cache.sequences - 1) / p.cache.sequences;
  return (p.tokens % p.cache.sequences ? 2 * mean - 1 : mean) * p.group;
}

// One CTA per SM, but no more than there can be tiles: blocks of rows of all sequences, each with the most tiles that the table
// holds.  regs: registers a thread that the kernel must have been compiled to (0: any number).
template <void (*kernel)(const AttentionParams), int SMEM, int THREADS, int ROWS, int TILE>
cudaError_t launch_ranges(const AttentionParams& p, int sm_count, cudaStream_t stream, int regs = 0) {
  static bool attr_set[64] = {};
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
    if (err != cudaSuccess) return err;
    cudaFuncAttributes fa;
    err = cudaFuncGetAttributes(&fa, kernel);
    if (err != cudaSuccess) return err;
    if (regs && fa.numRegs != regs) return cudaErrorInvalidConfiguration;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  const long long most = sm_count < kMostCtas ? sm_count : kMostCtas;
  const long long blocks = ((long long)p.tokens * p.group + ROWS - 1) / ROWS + p.cache.sequences;
  const long long per_block = (((long long)p.cache.max_pages << p.cache.page_shift) + TILE - 1) / TILE + 1;
  const long long tiles = (blocks < most ? blocks : most) * (per_block < most ? per_block : most) * p.cache.kv_heads;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles < most ? tiles : most));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace marlin_b200
