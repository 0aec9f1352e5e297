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
// Measured, 64 heads over 8 of 128 elements, back to back in a graph: 1184 new tokens behind 8000 seen through a window of 6000, 231 us, 1008 TFLOP/s; a
// prompt of 2048, 136 us; 700 tokens each of three prompts through a window of 512 with sinks, 105 us (its products alone 19, on
// attention_tc.cuh 491): there an item has six or seven tiles of 4900 cycles, 2000 for the products and 2900 for the softmax of both halves, 1400
// more where some keys are hidden (a mask takes two instructions of half rate a logit), and 5500 at its end.
//
// Warps: 0 - 3 the rows of the first half, 4 - 7 those of the second, 8 and 9 copy keys, 10 and 11 values (half of every tile each),
// 12 and 13 issue the products of a half each, 14 and 15 bring Q and look through values that not every row sees.  Tensor memory: S (and the
// weights) of both halves, O of both.  Items (sequence, key head, block) are taken whole, a CTA's next one lies a grid further on: a prompt
// has many of them, and nothing has to be joined.
#include "attention.cuh"
#include "tc_utils.cuh"

namespace marlin_b200 {
namespace {

constexpr int kTile = 128, kRows = 256, kHalf = 128;
constexpr int kBlock = kTile * 128;  // 64 elements of the keys of a tile (or of the rows of a half): rows of 128 bytes, as the swizzle has them
constexpr int kSoftmaxWarps = 8, kProducers = 4, kIssuers = 2, kCleaners = 2, kThreads = 512;
constexpr int kStageRow = 80;        // bytes of a row of results on their way out: 32 of them, and room so that eight rows lie in different banks
// Tiles of an item from which on the halves take turns: without them both run in step after some tiles and wait for each other (1184 tokens behind
// 8000, a window of 6000: 267 us without, 231 with them), but items of few tiles end before that and wait for the turn instead (three prompts of 700
// tokens behind 1000, a window of 512: 111 without, 119 with them).
constexpr int kTurns = 12;
constexpr int kNotes = 2;            // items that can be open at a time
// registers a thread: a softmax thread has a row of a tile, 128 logits
constexpr int kSoftmaxRegs = 192, kOtherRegs = 64;
static_assert((kSoftmaxWarps + kProducers + kIssuers + kCleaners) * 32 == kThreads, "warps");
static_assert(8 * kSoftmaxRegs + 8 * kOtherRegs <= 16 * 128, "registers");

template <int DP_>
struct PromptGeometry {
  static constexpr int DP = DP_;
  static constexpr int kSlot = DP / 64 * kBlock;   // the keys (or the values) of a tile, the rows of a half
  static constexpr int kSlots = DP == 64 ? 8 : 4;
  static constexpr int kKeySlots = kSlots / 2, kValueSlots = kSlots - kKeySlots;
  static constexpr int kSmem = (kSlots + 2) * kSlot + kSoftmaxWarps * 32 * kStageRow + 1024;
  static constexpr int kOut = 2 * kTile;           // columns of tensor memory where O begins
  static constexpr int kColumns = 512;
  static_assert(kOut + 2 * DP <= kColumns, "tensor memory");
};

template <class G>
struct PromptShared {
  uint64_t full[G::kSlots], empty[G::kSlots];  // keys, then values
  uint64_t ready[G::kValueSlots];              // values have been looked through
  uint64_t noted[kNotes], read[kNotes];        // an item is there; nobody needs its note any more
  uint64_t q_full[2], q_empty[2];              // of a half
  uint64_t s_full[2], p_half[2], p_full[2];  // logits are there (and all products before them done); half of the weights, all are
  uint64_t done[2];                            // all products of an item
  uint64_t turn[2];                            // the thread that issues products of a half may go on (S is free, O is complete so far)
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two fp32 numbers, in one instruction
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(Pair x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// whether some of the eight fp16 elements of a vector is not finite: an exponent of ones, and one more, carries into the sign
__device__ __forceinline__ bool not_finite_in(uint4 v) {
  auto odd = [](uint32_t w) { return (w & 0x7c007c00u) + 0x04000400u; };
  return ((odd(v.x) | odd(v.y) | odd(v.z) | odd(v.w)) & 0x80008000u) != 0;
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
    x.c0 = min((v.low_max + kTile - 1) / kTile - x.gap, x.nt - 1);
    if (x.c0 < x.sinks) x.c0 = min(x.sinks, x.nt - 1);
    at = at + gridDim.x < at ? total : at + gridDim.x;
    return x;
  }
};

// Tile i of an item in the order in which it goes over them: from number c0 on and round again to the tiles in front, so that the first
// one is one that all rows see, if there is one.  (What a row sees of the sinks or at the edge of its window, a few keys, makes a poor base: with the tiles
// in the order of the keys most items moved the bases of some rows once more, at 1300 cycles each.)
__device__ __forceinline__ int tile_in_turn(const SegmentWithGap& x, int i) {
  const int n = i + x.c0;
  return tile_of<kExtra>(x, n >= x.nt ? n - x.nt : n);
}

// ---- the warps that copy ---------------------------------------------------------------------------
template <class G>
__device__ __forceinline__ void produce(const AttentionParams& p, PromptShared<G>& sh, bool values, bool upper, uint32_t ring) {
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
  uint32_t slot_phase = 1, note_phase = 1;
#pragma unroll 1
  for (;;) {
    const SegmentWithGap x = items.next(p);
    const Visible v = visible(p, x);
    const int* const table = c.table + x.b * c.table_stride;
    const int low = v.low_min, high = v.high_max;
    // where the four sixteens of this warp in eight tiles begin, a lane each, and in the next eight: the number of the page, and its place
    auto key_of = [&](int i) { return tile_in_turn(x, i + lane / 4) * kTile + upper * 64 + lane % 4 * 16; };
    auto page_of = [&](int i) {
      const int key = key_of(i);
      return big_pages && i + lane / 4 < x.nt && key < high && (key + 16 > low || key < p.sinks) ? load(table + (key >> c.page_shift)) : INT_MIN;
    };
    auto place_of = [&](int i, int page) {
      if (page != INT_MIN && (unsigned)page >= (unsigned)c.pages) report_cache(p.status);
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
    long long places = place_of(0, page_first);
    int in_batch = 0;
#pragma unroll 1
    for (int i = 0; i < x.nt && go_on; ++i, ++in_batch) {
      if (in_batch == 8) {
        in_batch = 0;
        places = place_of(i, page_next);
        page_next = page_of(i + 8);
      }
      const int key0 = tile_in_turn(x, i) * kTile + upper * 64;
      go_on = arrived_at(sh, &sh.empty[slot], slot_phase, p.status);
      if (!go_on) break;
      const uint32_t to = ring + slot * G::kSlot + my_vec / 8 * kBlock + (upper * 64 + my_row) * 128;
      if (big_pages) {
        const bool whole = all_seen_by_some<kExtra>(p, key0, 64, low, high);
#pragma unroll 1
        for (int j = 0; j < 64; j += 16) {
          const long long place = __shfl_sync(~0u, places, in_batch * 4 + j / 16);
          const bool there = place >= 0 && my_part;
          const uint8_t* src = cache + (there ? place + my_bytes : 0);
          const long long step = there ? pass : 0;
          if (whole) {
#pragma unroll
            for (int r = 0; r < 16; r += kPer) {
              copy16(to + (j + r) * 128 + ((my_vec ^ (r + my_row)) & 7) * 16, src, there);
              src += step;
            }
          } else {  // the ends of a window, of the sinks or of the sequence
            const int key = key0 + j + my_row;
#pragma unroll
            for (int r = 0; r < 16; r += kPer) {
              copy16(to + (j + r) * 128 + ((my_vec ^ (r + my_row)) & 7) * 16, src, there && seen_by_some<kExtra>(p, key + r, low, high));
              src += step;
            }
          }
        }
      } else {  // smaller pages: a number for every key
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

// ---- the threads that issue the products, one for each half ------------------------------------------
// The products with the values of one tile and right behind them those with the keys of the next one (of the next item, where there is none):
// products are executed in the order of their issue, so the new logits may take the place of the weights that are being multiplied, and
// nobody waits in between.  The halves take turns: products of both in a mixed order would be done at the same time, and from then on both would
// have their weights made at the same time and their products wait for each other, 5000 cycles a tile.  What else they need is waited for while
// the weights are made.  (A wait costs a thread some 190 cycles even where it is over, an issue 65: one thread for both halves took 2400 cycles
// for each, and everybody waited for it.)
template <class G>
__device__ __forceinline__ void multiply(const AttentionParams& p, PromptShared<G>& sh, uint32_t ring, uint32_t q_at, uint32_t tmem, int half) {
  const uint32_t logits_desc = instr_desc_f16(kHalf, kTile) | (p.scale_log2 < 0.f ? 1u << 13 : 0u);  // (bit 13: the left operand is negated)
  constexpr uint32_t kResultsDesc = instr_desc_f16(kHalf, G::DP) | 1u << 16;  // the values across their rows
  const uint32_t q = q_at + half * G::kSlot, s_at = tmem + half * kTile, o_at = tmem + G::kOut + half * G::DP;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    mbar_wait(bar, parity, &sh.abort, p.status);
    return *(volatile int*)&sh.abort == 0;
  };
  int key_slot = 0, value_slot = 0, note = 0;
  uint32_t key_phase = 0, value_phase = 0, note_phase = 0, q_phase = 1, u = 0, turn = 0;  // u: tiles whose values are multiplied; turn: those in turns
  // tiles of the next item; 0: there is none, -1: a wait ran out
  auto next_item = [&] {
    if (!wait(&sh.noted[note], note_phase)) return -1;
    const int nt = *(volatile int*)&sh.items[note].nt;
    if (nt == 0) return 0;
    mbar_arrive(&sh.read[note]);  // (nothing else of the item is needed here)
    if (++note == kNotes) {
      note = 0;
      note_phase ^= 1;
    }
    q_phase ^= 1;
    return nt;
  };
  auto keys_there = [&] { return wait(&sh.full[key_slot], key_phase); };
  auto logits = [&](bool last) {
    const uint32_t keys = ring + key_slot * G::kSlot;
#pragma unroll
    for (int ks = 0; ks < G::DP / 16; ++ks)
      mma_ss(s_at, smem_desc_k_sw128(q + ks / 4 * kBlock + ks % 4 * 32), smem_desc_k_sw128(keys + ks / 4 * kBlock + ks % 4 * 32), logits_desc,
             ks ? 1 : 0);
    tc_commit(&sh.s_full[half]);
    if (last) tc_commit(&sh.q_empty[half]);
    tc_commit(&sh.empty[key_slot]);
    if (++key_slot == G::kKeySlots) {
      key_slot = 0;
      key_phase ^= 1;
    }
  };
  int nt = next_item();
  if (nt <= 0 || !keys_there() || !wait(&sh.q_full[half], q_phase)) return;
  fence_to_tensor_cores();
  logits(nt == 1);
#pragma unroll 1
  for (;;) {
    int following = 0;
    const bool turns = nt >= kTurns;
#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const bool more = i + 1 < nt;
      if (!wait(&sh.ready[value_slot], value_phase) || (more && !keys_there())) return;
      fence_to_tensor_cores();
      const uint32_t values = ring + (G::kKeySlots + value_slot) * G::kSlot;
#pragma unroll
      for (int ks = 0; ks < kTile / 16; ++ks) {
        if (ks == 0 || ks == kTile / 32) {
          if ((ks && turns && !wait(&sh.turn[half], half ? turn & 1 : (turn & 1) ^ 1)) || !wait(ks ? &sh.p_full[half] : &sh.p_half[half], u & 1)) return;
          tc_fence_after_sync();
        }
        tc_mma_ts(o_at, s_at + ks * 8, desc_columns(values + ks * 2048, kBlock), kResultsDesc, i || ks ? 1 : 0);
      }
      if (more) {
        logits(i + 2 == nt);
        if (turns) mbar_arrive(&sh.turn[half ^ 1]);
      } else {
        if (turns) mbar_arrive(&sh.turn[half ^ 1]);
        tc_commit(&sh.done[half]);
        following = next_item();
        if (following < 0) return;
        if (following > 0) {
          if (!keys_there() || !wait(&sh.q_full[half], q_phase)) return;
          fence_to_tensor_cores();
          logits(following == 1);
        }
      }
      turn += turns;
      tc_commit(&sh.empty[G::kKeySlots + value_slot]);
      if (++value_slot == G::kValueSlots) {
        value_slot = 0;
        value_phase ^= 1;
      }
    }
    if (following == 0) return;
    nt = following;
  }
}

// All products that this thread has issued are complete before tensor memory is freed and the block's shared memory goes to another: also where
// a wait ran out and nobody else has waited for them.  With a limit of its own (1 ms).
__device__ __forceinline__ void drain_products(uint64_t* bar) {
  tc_commit(bar);
  for (int i = 0; i < 1000 && !mbar_try_wait(bar, 0); ++i) __nanosleep(1000);
}

// ---- the warps that bring Q and look through values --------------------------------------------------
// Values of keys that some rows of a block see and others do not: what is not finite is left out of the products (clean_vector in attention.cuh).
// The tiles go through their hands in any case; most have no such keys.
template <class G>
__device__ __forceinline__ void look_through(const AttentionParams& p, PromptShared<G>& sh, uint32_t ring, uint32_t q_at, int tid) {
  constexpr int kMine = 32 * kCleaners, kVectors = G::DP / 8, kPer = 32 / kVectors;
  const KvCacheView& c = p.cache;
  const int lane = tid % 32, my_row = lane / kVectors, my_vec = lane % kVectors;
  const bool my_part = my_vec * 8 < c.head_dim;
  int slot = G::kKeySlots, note = 0, item = 0;
  uint32_t phase = 0, note_phase = 0, q_phase = 1;
#pragma unroll 1
  for (;; item = (item + 1) % 4) {
    if (!arrived_at(sh, &sh.noted[note], note_phase, p.status)) return;
    const SegmentWithGap& x = sh.items[note];
    const int nt = x.nt;
    if (nt == 0) return;
    // (the item that used it last is three back, and two back are read by everybody before this one's note is written)
    if (tid == 0) sh.not_finite[(item + 1) % 4] = 0;
    // Q, 64 rows a warp of each half; rows and elements that are not there are zeros
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      if (!arrived_at(sh, &sh.q_empty[half], q_phase, p.status)) return;
#pragma unroll 1
      for (int r0 = tid / 32 * 64; r0 < tid / 32 * 64 + 64; r0 += 32) {
        // a lane has a row: its token and head once
        const int r = half * kHalf + r0 + lane, token = token_of(p, x, r), head = x.h * p.group + x.row0 + r - token * p.group;
        const long long mine = r < x.rows ? (long long)(x.first + token) * p.q_stride + head * c.head_dim : -1;
#pragma unroll 8
        for (int i = 0; i < 32; i += kPer) {
          const long long from = __shfl_sync(~0u, mine, i + my_row);
          const bool there = from >= 0 && my_part;
          const int row = r0 + i + my_row;
          copy16(q_at + half * G::kSlot + my_vec / 8 * kBlock + row * 128 + ((my_vec ^ row) & 7) * 16, p.q + (there ? from + my_vec * 8 : 0), there);
        }
      }
      copies_arrive(&sh.q_full[half]);
    }
    q_phase ^= 1;
    const Visible sees = visible(p, x);
#pragma unroll 1
    for (int i = 0; i < nt; ++i) {
      const int pos0 = tile_in_turn(x, i) * kTile;
      if (!arrived_at(sh, &sh.full[slot], phase, p.status)) return;
      if (x.n > 1 && !all_seen_by_some<kExtra>(p, pos0, kTile, sees.low_max, sees.high_min)) {
        // two ranges of keys, at the edge of the windows (but for sinks) and around the new tokens; vectors side by side to lanes side by side
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
          const int begin = max(part ? sees.high_min : max(sees.low_min, p.sinks), pos0) - pos0;
          const int end = min(part ? sees.high_max : min(sees.low_max, sees.high_min), pos0 + kTile) - pos0;
          const int all_of = (end - begin) * (G::DP / 8);
          bool found = false;
#pragma unroll 1
          for (int n0 = tid; n0 < all_of; n0 += 4 * kMine) {
            auto at = [&](int n) {
              const int key = begin + n / (G::DP / 8), vec = n % (G::DP / 8);
              return ring + slot * G::kSlot + vec / 8 * kBlock + key * 128 + ((vec ^ key) & 7) * 16;
            };
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = lds128(at(min(n0 + k * kMine, all_of - 1)));
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (n0 + k * kMine < all_of && not_finite_in(v[k])) found |= clean_vector<false>(at(n0 + k * kMine));
          }
          if (found) sh.not_finite[item] = 1;
        }
        fence_to_tensor_cores();
      }
      __syncwarp();
      if (tid % 32 == 0) mbar_arrive(&sh.ready[slot - G::kKeySlots]);
      if (++slot == G::kSlots) {
        slot = G::kKeySlots;
        phase ^= 1;
      }
    }
    __syncwarp();
    if (tid % 32 == 0) mbar_arrive(&sh.read[note]);
    if (++note == kNotes) {
      note = 0;
      note_phase ^= 1;
    }
  }
}

// ---- softmax and results ---------------------------------------------------------------------------
// Whether a wait has run out is agreed upon where an item begins, so that the warps of a half always meet at the same barriers; the halves never
// wait for each other at one.
template <class G>
__device__ __forceinline__ void soften(const AttentionParams& p, PromptShared<G>& sh, uint32_t ring, uint32_t stages, uint32_t tmem, int half) {
  constexpr int DP = G::DP;
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x & 127, lane = tid & 31, warp = tid >> 5, row = half * kHalf + tid;
  const uint32_t lanes = tmem + ((uint32_t)warp << 21), s_at = lanes + half * kTile, o_at = lanes + G::kOut + half * DP;
  const uint32_t stage = stages + (half * 4 + warp) * 32 * kStageRow;
  auto wait = [&](uint64_t* bar, uint32_t parity) { mbar_wait(bar, parity, &sh.abort, p.status); };
  // (a hidden logit is an infinity, and would not stay one under 0: products of finite numbers times 1e-30 have weights of 1 all the same; where the
  // scale is negative the products are with -Q)
  const float factor = p.scale_log2 == 0.f ? 1e-30f : fabsf(p.scale_log2);

  uint32_t u = 0;  // tiles so far
  int note = 0, item = 0;
  uint32_t note_phase = 0;
#pragma unroll 1
  for (;; item = (item + 1) % 4) {
    wait(&sh.noted[note], note_phase);
    if (any_of(1 + half, 128, *(volatile int*)&sh.abort)) return;
    const SegmentWithGap& x = sh.items[note];
    const int nt = x.nt, rows = x.rows;
    if (nt == 0) return;
    const Visible sees = visible(p, x);
    const int token = token_of(p, x, min(row, rows - 1)), high = x.base_high + token, low = p.window ? max(0, high - p.window) : 0;
    // below the first everything, from the second on everything in front of that, is seen by all rows of the warp
    const int warp_high_min = __shfl_sync(~0u, high, 0), warp_low_max = __shfl_sync(~0u, low, 31);
    float base = kNone, sum = 0.f;  // of this row (attention.cuh)

#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const int pos0 = tile_in_turn(x, i) * kTile;
      const bool whole = pos0 + kTile <= warp_high_min && (pos0 >= warp_low_max || pos0 + kTile <= p.sinks);
      wait(&sh.s_full[half], u & 1);
      tc_fence_after_sync();
      float y[kTile];
#pragma unroll
      for (int j = 0; j < kTile; j += 64) tc_ld_x64(s_at + j, *reinterpret_cast<float(*)[64]>(y + j));
      tc_wait_ld();
      if (!whole) {
#pragma unroll
        for (int w = 0; w < kTile; w += 32) {  // 32 keys
          const int at = pos0 + w;
          // bit j: whether this row sees key j of them
          auto below = [&](int end) { return end <= at ? 0u : end >= at + 32 ? ~0u : (1u << (end - at)) - 1; };
          const uint32_t seen = below(high) & (~below(low) | below(p.sinks));
#pragma unroll
          for (int j = 0; j < 32; ++j) y[w + j] = seen & (1u << j) ? y[w + j] : kNone;
        }
      }
      // the largest logit of the row, looked for along eight chains
      float tops[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) tops[j] = fmaxf(y[j], y[j + 8]);
#pragma unroll
      for (int j = 16; j < kTile; j += 16)
#pragma unroll
        for (int k = 0; k < 8; ++k) tops[k] = max3(tops[k], y[j + k], y[j + k + 8]);
      tops[0] = max3(max3(tops[0], tops[1], tops[2]), max3(tops[3], tops[4], tops[5]), fmaxf(tops[6], tops[7]));
      const float top = tops[0] * factor;
      const bool move = base == kNone ? top > kNone : top > base + kSlack;
      if (__any_sync(~0u, move)) {
        float alpha = 1.f;
        if (move) {
          const float now = top - kBelow;
          alpha = exp2_fast(base - now);
          base = now;
          sum *= alpha;
        }
        if (i > 0) {  // the sums so far (the products that add to them were issued in front of those of these logits, and are done)
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
      // weights, rounded to fp16 for the product (kBelow in attention.cuh), over the logits; the first half of them is multiplied while the second is made
      const float from = base == kNone ? 0.f : -base;
      const Pair from2 = pair_of(from, from), factor2 = pair_of(factor, factor);
      Pair parts[2] = {0, 0};
#pragma unroll
      for (int w0 = 0; w0 < kTile; w0 += 64) {
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 64; j += 2) {
          float a, b;
          unpair(fma2(pair_of(y[w0 + j], y[w0 + j + 1]), factor2, from2), a, b);
          a = exp2_fast(a);
          b = exp2_fast(b);
          parts[j / 2 % 2] = add2(parts[j / 2 % 2], pair_of(a, b));
          w[j / 2] = half2_bits(a, b);
        }
        tc_st_x32(s_at + w0 / 2, w);
        if (w0 == 0) {
          tc_wait_st();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.p_half[half]);
        }
      }
      float even, odd;
      unpair(add2(parts[0], parts[1]), even, odd);
      sum += even + odd;
      tc_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[half]);
    }

    // ---- results
    wait(&sh.done[half], item & 1);
    tc_fence_after_sync();
    // (set in front of the products of the tile that it is about, of which those of the second half are behind those of the first)
    const bool odd_values = x.n > 1 && *(volatile int*)&sh.not_finite[item];
    const int head = x.h * p.group + x.row0 + row - token * p.group;
    const bool there = row < rows, nothing = high <= 0;
    const float f = nothing ? 0.f : __fdividef(1.f, sum);
    // through shared memory, so that four lanes write 64 bytes of a row together (a row to a lane, 16 bytes at a time, took 6800 cycles an item);
    // this lane writes for rows lane / 4 + 8 k of the warp
    const long long out_at = there ? ((long long)(x.first + token) * p.q_heads + head) * c.head_dim : -1;
    const uint32_t mine_at = stage + (lane * kStageRow);
    long long row_at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) row_at[k] = __shfl_sync(~0u, out_at, lane / 4 + 8 * k);
#pragma unroll 1
    for (int d = 0; d < DP; d += 32) {
      float z[32];
      tc_ld_x32(o_at + d, z);
      tc_wait_ld();
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 32; j += 8) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 8; k += 2) w[k / 2] = nothing ? 0u : half2_bits(z[j + k] * f, z[j + k + 1] * f);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(mine_at + j * 2), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
      }
      __syncwarp();
      const int at = d + lane % 4 * 8;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 v = lds128(stage + (lane / 4 + 8 * k) * kStageRow + lane % 4 * 16);
        if (row_at[k] >= 0 && at < c.head_dim) *reinterpret_cast<uint4*>(p.out + row_at[k] + at) = v;
      }
    }
    if (odd_values) {  // values that were left out, where this row sees them: nothing that is added to them changes them
      __syncwarp();
#pragma unroll 1
      for (int d = 0; d < c.head_dim && there; ++d) {
        const __half v = __float2half_rn(not_finite_sum<false>(p, x, sees, kTile, row, d));
        if (!isfinite(__half2float(v))) p.out[out_at + d] = *reinterpret_cast<const uint16_t*>(&v);
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
      mbar_init(&sh.empty[i], kIssuers);
    }
    for (int i = 0; i < G::kValueSlots; ++i) mbar_init(&sh.ready[i], kCleaners);
    for (int i = 0; i < kNotes; ++i) {
      mbar_init(&sh.noted[i], 1);
      mbar_init(&sh.read[i], kSoftmaxWarps + kIssuers + kCleaners);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 32 * kCleaners);
      mbar_init(&sh.q_empty[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_half[i], kSoftmaxWarps / 2);
      mbar_init(&sh.p_full[i], kSoftmaxWarps / 2);
      mbar_init(&sh.done[i], 1);
      mbar_init(&sh.turn[i], 1);
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
    soften<G>(p, sh, ring, q_at + 2 * G::kSlot, tmem, warp / 4);
  } else {
    setmaxnreg_dec<kOtherRegs>();
    const int w = warp - kSoftmaxWarps;
    if (w >= kProducers && w < kProducers + kIssuers) {
      if (threadIdx.x % 32 == 0) {
        multiply<G>(p, sh, ring, q_at, tmem, w - kProducers);
        drain_products(&sh.drained[w - kProducers]);
      }
    } else if (w >= kProducers + kIssuers) {
      look_through<G>(p, sh, ring, q_at, (int)threadIdx.x - (kSoftmaxWarps + kProducers + kIssuers) * 32);
      copies_wait_all();
    } else if (w < kProducers) {
      produce<G>(p, sh, w / 2, w % 2, ring);
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
