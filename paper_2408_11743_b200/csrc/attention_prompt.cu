// Attention of prompts over the paged cache: many new tokens of a sequence at a time, through a window with sinks or without.
//
// For one key head a block has 256 rows (a new token's query heads side by side, token after token), in two halves of 128.  Per tile of 128 keys
// and half: S = Q K^T with the rows as the 128 rows of the product, so that a softmax thread has all of one row in its lane of tensor memory and
// looks for maxima and sums by itself; the weights go back to tensor memory over S, as fp16, and are the left operand of O += P V, with
// the values as they lie in shared memory (keys as rows, read across).  A block goes over the tiles that some of its rows see: from the edge of
// its first row's window (behind the tiles of the sinks) to its last row's position.
//
// What bounds it: the products, 4 x 128 x 128 x head_dim multiplications a tile, take 2040 cycles of the tensor cores with 128 elements; the
// exponentials, 256 x 128 of them at 16 a cycle, 2048 cycles.  The halves take turns: one is multiplied while the other one's weights are
// made.
//
// Warps: 0 - 3 the rows of the first half, 4 - 7 those of the second, 8 and 9 copy keys, 10 and 11 values (half of every tile each; all four Q),
// 12 issues S, 13 O.  Tensor memory: S (and the weights) of both halves, O of both.  Items (sequence, key head, block) are taken whole, every
// CTA the one after the next grid: a prompt has many of them, and nothing has to be joined.
#include "attention.cuh"
#include "tc_utils.cuh"

namespace marlin_b200 {
namespace {

constexpr int kTile = 128, kRows = 256, kHalf = 128;
constexpr int kBlock = kTile * 128;  // 64 elements of the keys of a tile (or of the rows of a half): rows of 128 bytes, as the swizzle has them
constexpr int kSoftmaxWarps = 8, kProducers = 4, kIssuers = 2, kThreads = 512;
constexpr int kNotes = 2;            // items that can be open at a time
// registers a thread: a softmax thread has a row of a tile, 128 logits
constexpr int kSoftmaxRegs = 200, kOtherRegs = 56;
static_assert(8 * kSoftmaxRegs + 8 * kOtherRegs <= 16 * 128, "registers");

template <int DP_>
struct PromptGeometry {
  static constexpr int DP = DP_;
  static constexpr int kSlot = DP / 64 * kBlock;   // the keys (or the values) of a tile, the rows of a half
  static constexpr int kSlots = DP == 64 ? 8 : 4;
  static constexpr int kKeySlots = kSlots / 2, kValueSlots = kSlots - kKeySlots;
  static constexpr int kSmem = (kSlots + 2) * kSlot + 1024;
  static constexpr int kOut = 2 * kTile;           // columns of tensor memory where O begins
  static constexpr int kColumns = 512;
  static_assert(kOut + 2 * DP <= kColumns, "tensor memory");
};

template <class G>
struct PromptShared {
  uint64_t full[G::kSlots], empty[G::kSlots];  // keys, then values
  uint64_t noted[kNotes], read[kNotes];        // an item is there; nobody needs its note any more
  uint64_t q_full[2], q_empty[2];              // of a half
  uint64_t s_full[2], p_full[2], done[2];      // logits are there; weights are; they are multiplied (S is free, O is complete so far)
  uint64_t drained[kIssuers];
  SegmentWithGap items[kNotes];
  int abort;
  int not_finite[4];  // values were left out of the products of item k: [k % 4]
  uint32_t tmem;
};

__device__ __forceinline__ uint64_t desc_columns(uint32_t addr, uint32_t block) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// D[tmem] (+)= A[smem] . B[smem]
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void fence_to_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <class G>
__device__ __forceinline__ bool arrived_at(PromptShared<G>& sh, uint64_t* bar, uint32_t parity, int* status) {
  mbar_wait(bar, parity, &sh.abort, status);
  return !__any_sync(~0u, *(volatile int*)&sh.abort);
}

// The items of this CTA, blockIdx.x, blockIdx.x + gridDim.x, .. of all, as a whole warp follows them.  Lane i knows how many items sequences
// [i * per, (i + 1) * per) have, and those in front.
struct Items {
  uint32_t total, mine, before, at;
  int per;
  __device__ __forceinline__ int blocks_of(const AttentionParams& p, int b, Sequence& s, bool& bad) const {
    s.len = cache_length(p.cache, b, bad);
    s.first = b;
    s.n = 1;
    if (p.starts) {
      const int from = min(max(load(p.starts + b), 0), p.tokens), to = min(max(load(p.starts + b + 1), from), p.tokens);
      s.first = from;
      s.n = to - from;
    }
    return (s.n * p.group + kRows - 1) / kRows;
  }
  __device__ __forceinline__ void begin(const AttentionParams& p) {
    const KvCacheView& c = p.cache;
    const int lane = threadIdx.x & 31;
    per = (c.sequences + 31) / 32;
    mine = 0;
    bool bad = false;
    for (int b = lane * per; b < min(c.sequences, (lane + 1) * per); ++b) {
      Sequence s;
      const unsigned long long items = (unsigned long long)c.kv_heads * blocks_of(p, b, s, bad) + mine;
      mine = (uint32_t)min(items, (unsigned long long)kMostUnits);
    }
    if (bad) report_cache(p.status);
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t x = __shfl_up_sync(~0u, sum, d);
      if (lane >= d) sum = (uint32_t)min((unsigned long long)sum + x, (unsigned long long)kMostUnits);
    }
    total = __shfl_sync(~0u, sum, 31);
    before = sum - mine;
    at = blockIdx.x;
    if (total == kMostUnits) {  // more than are numbered
      report_cache(p.status);
      total = 0;
    }
  }
  // the next one; nt = 0: there is none
  __device__ __forceinline__ SegmentWithGap next(const AttentionParams& p) {
    SegmentWithGap x = {};
    if (at >= total) return x;
    const int owner = __ffs(__ballot_sync(~0u, mine > 0 && before <= at && at - before < mine)) - 1;
    uint32_t off = at - __shfl_sync(~0u, before, owner);
    Sequence s;
    int blocks;
    bool bad = false;  // (reported by begin())
    for (x.b = owner * per;; ++x.b) {
      blocks = blocks_of(p, x.b, s, bad);
      const uint32_t items = (uint32_t)p.cache.kv_heads * blocks;
      if (off < items) break;
      off -= items;
    }
    x.h = (int)(off / blocks);
    x.row0 = (int)(off - x.h * blocks) * kRows;
    x.rows = min(kRows, s.n * p.group - x.row0);
    x.base_high = s.len - s.n + 1;
    x.n = s.n;
    x.first = s.first;
    const Visible v = visible(p, x);
    const int last = (max(v.high_max, 0) + kTile - 1) / kTile;
    x.sinks = p.window ? min(last, (min(p.sinks, max(v.high_max, 0)) + kTile - 1) / kTile) : 0;
    x.gap = max(v.low_min / kTile, x.sinks) - x.sinks;
    x.nt = max(1, last - x.gap);  // (an item without a key to see has a tile all the same: it writes the zeros)
    at = at + gridDim.x < at ? total : at + gridDim.x;
    return x;
  }
};

// ---- the warps that copy ---------------------------------------------------------------------------
template <class G>
__device__ __forceinline__ void produce(const AttentionParams& p, PromptShared<G>& sh, bool values, bool upper, uint32_t ring, uint32_t q_at) {
  const KvCacheView& c = p.cache;
  const int lane = threadIdx.x & 31, producer = 2 * values + upper;
  Items items;
  items.begin(p);
  constexpr int kVectors = G::DP / 8, kPer = 32 / kVectors;
  const int my_row = lane / kVectors, my_vec = lane % kVectors;
  const bool my_part = my_vec * 8 < c.head_dim;
  const bool big_pages = c.page_shift >= 4;  // sixteen keys lie in one page
  const uint8_t* const cache = static_cast<const uint8_t*>(values ? c.v : c.k);
  const long long pass = my_part ? kPer * c.s_token * 2 : 0, my_bytes = my_row * c.s_token * 2 + my_vec * 16;
  const int first_slot = values ? G::kKeySlots : 0, last_slot = values ? G::kSlots - 1 : G::kKeySlots - 1;
  int slot = first_slot, note = 0;
  uint32_t slot_phase = 1, note_phase = 1, q_phase = 1;
#pragma unroll 1
  for (;;) {
    const SegmentWithGap x = items.next(p);
    const Visible v = visible(p, x);
    const int* const table = c.table + x.b * c.table_stride;
    const int low = v.low_min, high = v.high_max;
    // where the four sixteens of this warp in eight tiles begin, a lane each, and in the next eight: the number of the page, and its place
    auto key_of = [&](int i) { return tile_of<kExtra>(x, i + lane / 4) * kTile + upper * 64 + lane % 4 * 16; };
    auto page_of = [&](int i) {
      const int key = key_of(i);
      return big_pages && i + lane / 4 < x.nt && key < high && (key + 16 > low || key < p.sinks) ? load(table + (key >> c.page_shift)) : -1;
    };
    auto place_of = [&](int i, int page) {
      return (unsigned)page < (unsigned)c.pages
                 ? (page * c.s_page + x.h * c.s_head + (key_of(i) & ((1 << c.page_shift) - 1)) * c.s_token) * 2 : -1ll;
    };
    const int page_first = page_of(0);
    int page_next = page_of(8);
    if (!arrived_at(sh, &sh.read[note], note_phase, p.status)) break;
    if (lane == 0 && producer == 0) {
      sh.items[note] = x;
      mbar_arrive(&sh.noted[note]);
    }
    if (++note == kNotes) {
      note = 0;
      note_phase ^= 1;
    }
    if (x.nt == 0) break;
    bool go_on = true;
#pragma unroll 1
    for (int half = 0; half < 2 && go_on; ++half) {  // Q; rows and elements that are not there are zeros
      go_on = arrived_at(sh, &sh.q_empty[half], q_phase, p.status);
      if (!go_on) break;
      const int r0 = half * kHalf + producer * 32;
      // a lane has a row: its token and head once
      const int r = r0 + lane, token = token_of(p, x, r), head = x.h * p.group + x.row0 + r - token * p.group;
      const long long mine = r < x.rows ? (long long)(x.first + token) * p.q_stride + head * c.head_dim : -1;
#pragma unroll 2
      for (int i = 0; i < 32; i += kPer) {
        const long long from = __shfl_sync(~0u, mine, i + my_row);
        const bool there = from >= 0 && my_part;
        const int row = producer * 32 + i + my_row;
        copy16(q_at + half * G::kSlot + my_vec / 8 * kBlock + row * 128 + ((my_vec ^ row) & 7) * 16, p.q + (there ? from + my_vec * 8 : 0), there);
      }
      copies_arrive(&sh.q_full[half]);
    }
    q_phase ^= 1;
    long long places = place_of(0, page_first);
    int in_batch = 0;
#pragma unroll 1
    for (int i = 0; i < x.nt && go_on; ++i, ++in_batch) {
      if (in_batch == 8) {
        in_batch = 0;
        places = place_of(i, page_next);
        page_next = page_of(i + 8);
      }
      const int key0 = tile_of<kExtra>(x, i) * kTile + upper * 64;
      const bool there4 = lane / 4 != in_batch || places >= 0;
      const bool whole = big_pages && all_seen_by_some<kExtra>(p, key0, 64, low, high) && __all_sync(~0u, there4);
      go_on = arrived_at(sh, &sh.empty[slot], slot_phase, p.status);
      if (!go_on) break;
      const uint32_t to = ring + slot * G::kSlot + my_vec / 8 * kBlock + (upper * 64 + my_row) * 128;
      if (whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const long long place = __shfl_sync(~0u, places, in_batch * 4 + j);
          const uint8_t* src = cache + (my_part ? place + my_bytes : 0);
#pragma unroll
          for (int r = 0; r < 16; r += kPer) {
            copy16(to + (j * 16 + r) * 128 + ((my_vec ^ (r + my_row)) & 7) * 16, src, my_part);
            src += pass;
          }
        }
      } else {  // pages smaller than that, the ends of a sequence, pages that are not there
#pragma unroll 2
        for (int r = 0; r < 64; r += kPer) {
          const int row = r + my_row, key = key0 + row;
          const bool asked = seen_by_some<kExtra>(p, key, low, high);
          const long long at = asked ? cache_offset(c, load(table + (key >> c.page_shift)), x.h, key, p.status) : -1;
          const bool there = at >= 0 && my_part;
          copy16(to + r * 128 + ((my_vec ^ row) & 7) * 16, cache + (there ? at * 2 + my_vec * 16 : 0), there);
        }
      }
      if (!withheld(p, slot == 0)) copies_arrive(&sh.full[slot]);
      if (slot == last_slot) {
        slot = first_slot;
        slot_phase ^= 1;
      } else {
        ++slot;
      }
    }
    if (!go_on) break;
  }
  copies_wait_all();
}

// ---- the threads that issue the products -----------------------------------------------------------
enum Product { kLogits, kResults };
template <class G, int WHICH>
__device__ __forceinline__ void multiply(const AttentionParams& p, PromptShared<G>& sh, uint32_t ring, uint32_t q_at, uint32_t tmem) {
  constexpr uint32_t kLogitsDesc = instr_desc_f16(kHalf, kTile);
  constexpr uint32_t kResultsDesc = instr_desc_f16(kHalf, G::DP) | 1u << 16;  // the values across their rows
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    mbar_wait(bar, parity, &sh.abort, p.status);
    return *(volatile int*)&sh.abort == 0;
  };
  constexpr int kFirst = WHICH == kLogits ? 0 : G::kKeySlots, kLast = WHICH == kLogits ? G::kKeySlots - 1 : G::kSlots - 1;
  int slot = kFirst, note = 0;
  uint32_t phase = 0, note_phase = 0, q_phase = 0, u = 0;
#pragma unroll 1
  for (;;) {
    if (!wait(&sh.noted[note], note_phase)) return;
    const int nt = *(volatile int*)&sh.items[note].nt;
    if (nt == 0) return;
    mbar_arrive(&sh.read[note]);  // (nothing else of the item is needed here)
#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      if (!wait(&sh.full[slot], phase)) return;
      const uint32_t there = ring + slot * G::kSlot;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        if (WHICH == kLogits) {
          if (i == 0 && !wait(&sh.q_full[half], q_phase)) return;
          if (!wait(&sh.done[half], (u & 1) ^ 1)) return;  // the weights of the tile before are multiplied: S is free
          fence_to_tensor_cores();
          tc_fence_after_sync();
          const uint32_t q = q_at + half * G::kSlot;
#pragma unroll
          for (int ks = 0; ks < G::DP / 16; ++ks)
            mma_ss(tmem + half * kTile, smem_desc_k_sw128(q + ks / 4 * kBlock + ks % 4 * 32),
                   smem_desc_k_sw128(there + ks / 4 * kBlock + ks % 4 * 32), kLogitsDesc, ks ? 1 : 0);
          tc_commit(&sh.s_full[half]);
          if (i + 1 == nt) tc_commit(&sh.q_empty[half]);
        } else {
          if (!wait(&sh.p_full[half], u & 1)) return;
          fence_to_tensor_cores();
          tc_fence_after_sync();
#pragma unroll
          for (int ks = 0; ks < kTile / 16; ++ks)
            tc_mma_ts(tmem + G::kOut + half * G::DP, tmem + half * kTile + ks * 8, desc_columns(there + ks * 2048, kBlock), kResultsDesc,
                      i || ks ? 1 : 0);
          tc_commit(&sh.done[half]);
        }
      }
      tc_commit(&sh.empty[slot]);
      if (slot == kLast) {
        slot = kFirst;
        phase ^= 1;
      } else {
        ++slot;
      }
    }
    q_phase ^= 1;
    if (++note == kNotes) {
      note = 0;
      note_phase ^= 1;
    }
  }
}

// All products that this thread has issued are complete before tensor memory is freed and the block's shared memory goes to another: also where
// a wait ran out and nobody else has waited for them.  With a limit of its own (1 ms).
__device__ __forceinline__ void drain_products(uint64_t* bar) {
  tc_commit(bar);
  for (int i = 0; i < 1000 && !mbar_try_wait(bar, 0); ++i) __nanosleep(1000);
}

// ---- softmax and results ---------------------------------------------------------------------------
// Whether a wait has run out is agreed upon where an item begins, so that the warps of a half always meet at the same barriers; the halves never
// wait for each other at one.
template <class G>
__device__ __forceinline__ void soften(const AttentionParams& p, PromptShared<G>& sh, uint32_t ring, uint32_t tmem, int half) {
  constexpr int DP = G::DP;
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x & 127, lane = tid & 31, warp = tid >> 5, row = half * kHalf + tid;
  const uint32_t lanes = tmem + ((uint32_t)warp << 21), s_at = lanes + half * kTile, o_at = lanes + G::kOut + half * DP;
  auto wait = [&](uint64_t* bar, uint32_t parity) { mbar_wait(bar, parity, &sh.abort, p.status); };
  // (a hidden logit is an infinity, and would not stay one under 0: products of finite numbers times 1e-30 have weights of 1 all the same)
  const float factor = p.scale_log2 == 0.f ? 1e-30f : p.scale_log2, hidden = factor < 0.f ? INFINITY : -INFINITY;

  uint32_t u = 0;  // tiles so far
  int note = 0, item = 0;
  uint32_t note_phase = 0;
#pragma unroll 1
  for (;; item = (item + 1) % 4) {
    wait(&sh.noted[note], note_phase);
    if (any_of(1 + half, 128, *(volatile int*)&sh.abort)) return;
    // (the item that used it last is three back, and two back are read by everybody before this one's note is written)
    if (half == 0 && tid == 0) sh.not_finite[(item + 1) % 4] = 0;
    const SegmentWithGap& x = sh.items[note];
    const int nt = x.nt, rows = x.rows;
    if (nt == 0) return;
    const Visible sees = visible(p, x);
    const int token = token_of(p, x, min(row, rows - 1)), high = x.base_high + token, low = p.window ? max(0, high - p.window) : 0;
    float base = kNone, sum = 0.f;  // of this row (attention.cuh)

#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const int pos0 = tile_of<kExtra>(x, i) * kTile;
      const bool all = all_seen_by_some<kExtra>(p, pos0, kTile, sees.low_max, sees.high_min);
      wait(&sh.s_full[half], u & 1);
      tc_fence_after_sync();
      float y[kTile];
#pragma unroll
      for (int j = 0; j < kTile; j += 64) tc_ld_x64(s_at + j, *reinterpret_cast<float(*)[64]>(y + j));
      tc_wait_ld();
      if (!all) {
        // bit j of a word: whether this row sees key j of 32
#pragma unroll
        for (int w = 0; w < kTile / 32; ++w) {
          const int at = pos0 + w * 32;
          auto below = [&](int end) { return end <= at ? 0u : end >= at + 32 ? ~0u : (1u << (end - at)) - 1; };
          const uint32_t seen = below(high) & (~below(low) | below(p.sinks));
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (!(seen >> j & 1)) y[w * 32 + j] = hidden;
        }
      }
      const float from = base == kNone ? 0.f : base;
      float top = kNone;
#pragma unroll
      for (int j = 0; j < kTile; j += 2) {
        y[j] = fmaf(y[j], factor, -from);
        y[j + 1] = fmaf(y[j + 1], factor, -from);
        top = fmaxf(top, fmaxf(y[j], y[j + 1]));
      }
      const bool move = top > kSlack || (base == kNone && top > kNone);
      if (__any_sync(~0u, move)) {
        float alpha = 1.f;
        if (move) {
          const float now = from + top - kBelow;
          alpha = exp2_fast(base - now);
          base = now;
          sum *= alpha;
          const float shift = from - now;
#pragma unroll
          for (int j = 0; j < kTile; ++j) y[j] += shift;
        }
        if (i > 0) {  // the sums so far, when the products that add to them are done
          wait(&sh.done[half], (u & 1) ^ 1);
          tc_fence_after_sync();
#pragma unroll 1
          for (int d = 0; d < DP; d += 16) {
            float z[16];
            tc_ld_x16(o_at + d, z);
            tc_wait_ld();
            uint32_t w[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(z[j] * alpha);
            tc_st_x8(o_at + d, *reinterpret_cast<const uint32_t(*)[8]>(w));
            tc_st_x8(o_at + d + 8, *reinterpret_cast<const uint32_t(*)[8]>(w + 8));
          }
        }
      }
      // weights, rounded to fp16 for the product (kBelow in attention.cuh), over the logits
#pragma unroll
      for (int w0 = 0; w0 < kTile; w0 += 64) {
        uint32_t w[32];
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 64; j += 2) {
          const float a = exp2_fast(y[w0 + j]), b = exp2_fast(y[w0 + j + 1]);
          part[0] += a;
          part[1] += b;
          w[j / 2] = half2_bits(a, b);
        }
        sum += part[0] + part[1];
        tc_st_x32(s_at + w0 / 2, w);
      }
      tc_wait_st();
      tc_fence_before_sync();
      if (x.n > 1 && !all && half == 0) {  // values of keys that not every row sees: what is not finite is left out
        const uint32_t v_slot = G::kKeySlots + u % G::kValueSlots;
        const int pos = pos0 + tid;
        wait(&sh.full[v_slot], u / G::kValueSlots & 1);
        if ((pos >= sees.high_min && pos < sees.high_max) || (pos >= sees.low_min && pos < sees.low_max && pos >= p.sinks)) {
          bool found = false;
#pragma unroll 1
          for (int vec = 0; vec < DP / 8; ++vec)
            found |= clean_vector<false>(ring + v_slot * G::kSlot + vec / 8 * kBlock + tid * 128 + ((vec ^ tid) & 7) * 16);
          if (found) sh.not_finite[item] = 1;
        }
        fence_to_tensor_cores();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[half]);
    }

    // ---- results
    wait(&sh.done[half], (u & 1) ^ 1);
    tc_fence_after_sync();
    // (set in front of the products of the tile that it is about, of which those of the second half are behind those of the first)
    const bool odd_values = x.n > 1 && *(volatile int*)&sh.not_finite[item];
    const int head = x.h * p.group + x.row0 + row - token * p.group;
    const bool there = row < rows, nothing = high <= 0;
    const float f = nothing ? 0.f : __fdividef(1.f, sum);
    uint16_t* const out = p.out + ((long long)(x.first + token) * p.q_heads + head) * c.head_dim;
#pragma unroll 1
    for (int d = 0; d < DP; d += 16) {
      float z[16];
      tc_ld_x16(o_at + d, z);
      tc_wait_ld();
      if (there && d < c.head_dim) {
        if (odd_values) {
#pragma unroll 1
          for (int j = 0; j < 16; ++j) {
            const float v = not_finite_sum<false>(p, x, sees, kTile, row, d + j);
#pragma unroll
            for (int k = 0; k < 16; ++k) z[k] += k == j ? v : 0.f;
          }
        }
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 16; j += 2) w[j / 2] = nothing ? 0u : half2_bits(z[j] * f, z[j + 1] * f);
        *reinterpret_cast<uint4*>(out + d) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(out + d + 8) = make_uint4(w[4], w[5], w[6], w[7]);
      }
      __syncwarp();
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.read[note]);
    if (++note == kNotes) {
      note = 0;
      note_phase ^= 1;
    }
  }
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1) attention_prompt_kernel(const AttentionParams p) {
  using G = PromptGeometry<DP>;
  extern __shared__ uint8_t smem[];
  __shared__ PromptShared<G> sh;
  const uint32_t ring = (smem_u32(smem) + 1023u) & ~1023u, q_at = ring + G::kSlots * G::kSlot;
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < G::kSlots; ++i) {
      mbar_init(&sh.full[i], 32 * kProducers / 2);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < kNotes; ++i) {
      mbar_init(&sh.noted[i], 1);
      mbar_init(&sh.read[i], kSoftmaxWarps + kIssuers);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 32 * kProducers);
      mbar_init(&sh.q_empty[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_full[i], kSoftmaxWarps / 2);
      mbar_init(&sh.done[i], 1);
    }
    for (int i = 0; i < kIssuers; ++i) mbar_init(&sh.drained[i], 1);
    sh.abort = 0;
    for (int i = 0; i < 4; ++i) sh.not_finite[i] = 0;
  }
  if (warp == kThreads / 32 - 1) {
    tmem_alloc(&sh.tmem, G::kColumns);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  prefetch_table(p, kThreads);
  if (warp < kSoftmaxWarps) {
    setmaxnreg_inc<kSoftmaxRegs>();
    soften<G>(p, sh, ring, tmem, warp / 4);
  } else {
    setmaxnreg_dec<kOtherRegs>();
    const int w = warp - kSoftmaxWarps;
    if (w >= kProducers && w < kProducers + kIssuers && threadIdx.x % 32 == 0) {
      if (w == kProducers)
        multiply<G, kLogits>(p, sh, ring, q_at, tmem);
      else
        multiply<G, kResults>(p, sh, ring, q_at, tmem);
      drain_products(&sh.drained[w - kProducers]);
    } else if (w < kProducers) {
      produce<G>(p, sh, w / 2, w % 2, ring, q_at);
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();  // (every role ends, by itself or when a wait ran out)
  if (warp == kThreads / 32 - 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, G::kColumns);
  }
}

template <int DP>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return launch_ranges<attention_prompt_kernel<DP>, PromptGeometry<DP>::kSmem, kThreads, kRows, kTile>(p, sm_count, stream, 128);
}

}  // namespace

cudaError_t launch_attention_prompt(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return padded_dim(p.cache.head_dim) == 64 ? launch<64>(p, sm_count, stream) : launch<128>(p, sm_count, stream);
}

}  // namespace marlin_b200
