// Attention of new tokens where a key head has more than eight rows (heads that share keys, several new tokens): the same ranges, segments and parts as
// attention_warp.cuh, with the products on the fifth-generation tensor cores.
//
// A tile has 128 keys.  S^T = K Q^T with the keys as the 128 rows of the product and the rows of Q as its columns, so that thread k of
// the softmax warps has key k and all N rows of it in its lane of tensor memory; the weights go to shared memory as P, and
// O^T += V^T P^T has the elements of the head as its 128 rows.  Both products are as narrow as there are rows: 128 x N x 16 a step.
// A thread sees one key of every row.  So the largest logits of rows, which would have to be looked for across threads, are looked for
// only when a logit exceeds the base of its row by kSlack (attention.cuh); the sums in tensor memory are rescaled then.  The
// weights of a row are summed by a block of ones beside the values where the head leaves room for it in the 128 rows of the second
// product (64 elements), and otherwise by the threads, over the keys that each of them sees.
//
// What bounds it: the products read every key and value from shared memory once, 128 bytes a cycle: 512 cycles for a tile of
// 64 KB, which takes 2800 to come from memory.  (A third product, of ones with the weights, cost as much as either of the two.)
// So the memory should bound it, and does not: 16 sequences of 1000 to 4099 keys with 48 rows for each of eight heads of 128 elements take
// 47.6 us (3.7 TB/s; the copies alone 40.6, mma.sync in its place 53), 24 of 900 to 16001 keys seen through a window of 2048, 29 rows of 64
// elements, 35 us (2.8 TB/s; copies alone 28, mma.sync 36).  So most of the distance to the time of their bytes, 26.6 and 14.9 us, lies in
// the copies and in what a call costs beside them (17 and 15 us).  The rest: the chain of one tile, from its logits through the
// weights to the second product, where an item has few tiles; the ends of the items; and instructions, since softmax, moves of
// the bases, read-out and joining do not fit into the nearest caches together (their order in the file moves these times by a tenth).
//
// Warps: 0 - 7 softmax and results (lane quarter w % 4 of tensor memory; 0 - 3 the first half of the rows, 4 - 7 the second, each
// half with bases of its own), 8 and 9 copy keys, 10 and 11 values (half of every tile each), 12 and 13 issue a product each: an issue
// costs its thread some 75 cycles and a commit 125, and with one thread for all of them everybody waited for it.
// An 8-bit cache (of 128 elements, for more than 32 rows) is converted to fp16 by the warps that copy: the products take operands of
// one type, and fp16 is what Q and the weights have.  The conversion bounds that: some 260 cycles for 16 keys of one warp.
// With scales by block a softmax thread has the scales of its key and its value: the logit is multiplied with one, the weight with the other one
// over a power of two that the sums are held in (`unit`).  16 sequences of 1000 to 4099 keys, up to six drafted tokens, 64 heads over 8,
// e4m3: 57.4 us (bytes alone 13.5).  A tile takes 3300 cycles: the warps that copy have 1000 of them for the conversion, 1500 for the
// copies, the softmax warps 1100 until the weights are to be made and 1500 until they are there; an item 8000 more for its end and its parts.
// Keys and values have rings of their own: values are held until the weights of their keys are there, and keys need not wait for that.
// Tensor memory: S twice, O, and what of O was put aside (kFold); N columns each.
#pragma once
#include "attention.cuh"
#include "tc_utils.cuh"

namespace marlin_b200 {
namespace {
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

constexpr int kTile = 128;
constexpr int kLead = 4;                 // what an item costs beside its tiles, in tiles
// Tiles whose results are summed in the products.  A product adds to its sums in fp32 but cuts off what lies below them, key by key, so that
// sums over 131 thousand keys come out too small by 2^-10.5 (7e-4, measured; over 524 thousand by 2.8e-3, where the weights are summed
// elsewhere), more than half a step of fp16.  After so many tiles they are therefore added to others, rounded, and
// begin again: 1e-4 whatever the length.  That is one pause in 16384 keys.
constexpr int kFold = 128;
constexpr int kBlock = kTile * 128;      // 64 elements of the keys of a tile: rows of 128 bytes, as the swizzle has them
constexpr int kSoftmaxWarps = 8;
constexpr int kSoftmaxThreads = kSoftmaxWarps * 32;
constexpr int kProducers = 4;
constexpr int kIssuers = 2;
constexpr int kThreads = 512;  // (two warps do nothing: registers are shared out by groups of four)
static_assert(kSoftmaxThreads + (kProducers + kIssuers) * 32 <= kThreads, "warps");

// DP: head_dim rounded up to 64 or 128; N: rows of a block, 16, 32 or 64; F8: e4m3 cache
template <int DP_, int N_, bool F8_, int EXTRA_>
struct TcGeometry {
  static constexpr int DP = DP_, N = N_, EXTRA = EXTRA_;
  static constexpr bool F8 = F8_;
  static constexpr bool kScaled = F8 && EXTRA != kNoExtra, kInt8 = F8 && EXTRA == kExtraInt8;
  static constexpr int kHalves = DP / 64;
  static constexpr int kSlot = kHalves * kBlock;   // the keys (or the values) of a tile
  static constexpr int kQBlock = N * 128;          // 64 elements of the rows
  static constexpr int kQBytes = kHalves * kQBlock;
  static constexpr int kOpen = 2;                  // segments that can be open at a time
  static constexpr int kPRow = 2 * N;              // weights: bytes of a key, swizzled over as many
  static constexpr int kPBytes = kTile * kPRow;
  static constexpr int kPBuffers = F8 ? 1 : 2;     // (room for the ring of the 8-bit keys)
  static constexpr bool kSumRows = DP == 64 && !kScaled;       // the weights are summed in the product
  static constexpr int kOnes = kSumRows ? 2048 : 0;  // 16 rows of 64 ones, beside the values of 16 keys
  static constexpr int kRest = kOpen * kQBytes + kPBuffers * kPBytes + kOnes;
  static constexpr int kFit = (222 * 1024 - kRest) / kSlot;
  static constexpr int kSlots = F8 ? 4 : kFit > 12 ? 12 : kFit;
  // 8-bit caches: sixteen keys (or values) as they come, and how many of them each warp that copies has on their way
  static constexpr int kRawBytes = 16 * DP;
  static constexpr int kRawFit = (222 * 1024 - kRest - kSlots * kSlot) / (kProducers * kRawBytes);
  static constexpr int kRaw = F8 ? (kRawFit > 16 ? 16 : kRawFit) : 0;
  static constexpr int kKeySlots = kSlots / 2, kValueSlots = kSlots - kKeySlots;
  // registers a thread where the launch's 128 are too few for the softmax warps (64 rows)
  static constexpr int kSoftmaxRegs = N == 64 ? 160 : 0, kOtherRegs = 96;
  static_assert(8 * kSoftmaxRegs + 8 * kOtherRegs <= 16 * 128, "registers");
  static constexpr int kSmem = kSlots * kSlot + kRest + kProducers * kRaw * kRawBytes + 1024;  // (the ring begins at a multiple of 1024)
  static constexpr int kColumns = 4 * N;           // of tensor memory: S, S, O, and O put aside
  static constexpr int kMine = N / 2;              // rows of a half of the softmax warps
  static_assert(kKeySlots >= 2 && kColumns <= 512, "ring");
};

template <class G>
struct TcShared {
  uint64_t full[G::kSlots], empty[G::kSlots];  // keys, then values
  uint64_t opened[G::kOpen], closed[G::kOpen];
  uint64_t s_full[2], s_free[2];                       // logits are there; have been read
  uint64_t p_full[G::kPBuffers], p_done[G::kPBuffers]; // weights are there; have been multiplied
  uint64_t drained[kIssuers];                          // all products of an issuing thread are complete
  SegmentOf<G::EXTRA> segments[G::kOpen];
  float2 ml[G::N];
  alignas(16) float base[G::N];  // of the rows, read four at a time; 0 where a row has seen nothing
  float largest[G::N];           // the same, -inf where a row has seen nothing (its largest logit less kBelow)
  float alpha[G::N];             // what the sums are multiplied with when the base moves
  float tops[4][G::N];           // of the warps: largest logits; sums of weights
  int high[G::N];                // positions below which the rows see
  int abort;
  int arrived;
  int not_finite[2];
  uint32_t tmem;
  float scale_tops[kSoftmaxWarps];  // kScaled: the largest scales of values of the warps
};

// shared-memory descriptors of 128-byte swizzled operands with eight rows of 128 bytes 1024 bytes apart.  Rows of the product along
// the rows of the tile: smem_desc_k_sw128 (`stride` 0: the same eight rows again and again).  Along its bytes: blocks of 64
// elements `block` bytes apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t addr, uint32_t stride) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(stride >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint64_t desc_columns(uint32_t addr, uint32_t block) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// the same along rows of 128, 64 or 32 bytes that are one block, swizzled over their length: modes 2, 4, 6; eight rows lie together
template <int ROW>
__device__ __forceinline__ uint64_t desc_weights(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(8 * ROW >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)(ROW == 128 ? 2 : ROW == 64 ? 4 : 6) << 61);
}
// what the 16-byte vectors of row `key` are permuted by
template <int ROW>
__device__ __forceinline__ int swizzle_of(int key) {
  return ROW == 128 ? key & 7 : ROW == 64 ? key >> 1 & 3 : key >> 2 & 1;
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
__device__ __forceinline__ void sts128(uint32_t saddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// what this thread (or another whose arrival it has seen) wrote to shared memory can be read by the tensor cores
__device__ __forceinline__ void fence_to_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
template <int C>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&x)[C]) {
  if constexpr (C == 32)
    tc_ld_x32(taddr, x);
  else if constexpr (C == 16)
    tc_ld_x16(taddr, x);
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void load_column(uint32_t taddr, float& x) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=f"(x) : "r"(taddr) : "memory");
}
template <int C>
__device__ __forceinline__ void store_columns(uint32_t taddr, const float (&x)[C]) {
#pragma unroll
  for (int i = 0; i < C; i += 8) {
    uint32_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(x[i + j]);
    tc_st_x8(taddr + i, r);
  }
}

// a wait of a whole warp (the same answer for all of it); false: it, or one of another warp, ran out
template <class G>
__device__ __forceinline__ bool arrived_at(TcShared<G>& sh, uint64_t* bar, uint32_t parity, int* status) {
  mbar_wait(bar, parity, &sh.abort, status);
  return !__any_sync(~0u, *(volatile int*)&sh.abort);
}

// ---- the warps that copy ---------------------------------------------------------------------------
// `values`: these, not keys; `upper`: the second half of every tile
template <class G>
__device__ __forceinline__ void produce(const AttentionParams& p, TcShared<G>& sh, bool values, bool upper, uint32_t ring, uint32_t q_slots,
                                        uint32_t raw) {
  constexpr int EXTRA = G::EXTRA;
  const KvCacheView& c = p.cache;
  const int lane = threadIdx.x & 31, producer = 2 * values + upper;
  Range<G::N, kTile, kLead, EXTRA> range;
  range.begin(p);

  constexpr int kVectors = G::DP / 8;
  constexpr int kPer = 32 / kVectors;
  const int my_row = lane / kVectors, my_vec = lane % kVectors;
  const bool my_part = my_vec * 8 < c.head_dim;
  constexpr int kElement = G::F8 ? 1 : 2;
  const bool big_pages = c.page_shift >= 4;  // sixteen keys lie in one page
  const uint8_t* const cache = static_cast<const uint8_t*>(values ? c.v : c.k);
  const long long pass = my_part ? kPer * c.s_token * 2 : 0;
  const int first_slot = values ? G::kKeySlots : 0, last_slot = values ? G::kSlots - 1 : G::kKeySlots - 1;
  int slot = first_slot, open = 0;
  uint32_t slot_phase = 1, open_phase = 1;
#pragma unroll 1
  for (;;) {
    const SegmentOf<EXTRA> x = range.next(p);
    // the page numbers of its first tiles are asked for before anything else: the first copies wait for them
    const Visible v = visible(p, x);
    const int* const table = c.table + x.b * c.table_stride;
    const int key_first = x.tile * kTile + upper * 64;
    const int low = EXTRA != kNoExtra ? v.low_min : max(v.low_min, x.tile * kTile);
    const int high = EXTRA != kNoExtra ? v.high_max : min(v.high_max, (x.tile + x.nt) * kTile);
    // where this warp's half of tile i begins
    auto begin_of = [&](int i) { return EXTRA != kNoExtra ? tile_of<EXTRA>(x, i) * kTile + upper * 64 : key_first + i * kTile; };
    // where the four sixteens of this warp in eight tiles begin in the cache, a lane each, and in the next eight: the page number
    // that was asked for, and what it comes to; -1 where it is not there (of 8 bits: or not all of them are seen)
    auto key_of = [&](int i) { return begin_of(i + lane / 4) + lane % 4 * 16; };
    auto page_of = [&](int i) {
      const int key = key_of(i);
      if (EXTRA != kNoExtra)
        return big_pages && i + lane / 4 < x.nt && key < high && (key + 16 > low || key < p.sinks) ? load(table + (key >> c.page_shift)) : -1;
      return big_pages && x.nt > 0 && key < high && key + 16 > low ? load(table + (key >> c.page_shift)) : -1;
    };
    auto place_of = [&](int i, int page) {
      return (unsigned)page < (unsigned)c.pages && (!G::F8 || all_seen_by_some<EXTRA>(p, key_of(i), 16, low, high))
                 ? (page * c.s_page + x.h * c.s_head + (key_of(i) & ((1 << c.page_shift) - 1)) * c.s_token) * kElement : -1ll;
    };
    const int page_first = page_of(0);
    int page_next = page_of(8);
    if (!arrived_at(sh, &sh.closed[open], open_phase, p.status)) break;
    if (lane == 0 && producer == 0) sh.segments[open] = x;
    if (x.nt > 0) {  // Q; rows and elements that are not there are zeros
#pragma unroll 1
      for (int i = producer * 32 + lane; i < G::N * kVectors; i += 32 * kProducers) {
        const int r = i / kVectors, vec = i % kVectors;
        const int token = token_of(p, x, r), head = x.h * p.group + x.row0 + r - token * p.group;
        const bool there = r < x.rows && vec * 8 < c.head_dim;
        const uint16_t* src = p.q + (there ? (long long)(x.first + token) * p.q_stride + head * c.head_dim + vec * 8 : 0);
        copy16(q_slots + open * G::kQBytes + vec / 8 * G::kQBlock + r * 128 + ((vec ^ r) & 7) * 16, src, there);
      }
    }
    copies_arrive(&sh.opened[open]);
    if (lane == 0 && producer == 0) mbar_arrive(&sh.opened[open]);
    if (++open == G::kOpen) {
      open = 0;
      open_phase ^= 1;
    }
    if (x.nt == 0) break;

    const long long my_bytes = my_row * c.s_token * 2 + my_vec * 16;
    long long places = place_of(0, page_first);
    int in_batch = 0;
    bool go_on = true;
    if constexpr (G::F8) {
      // eight bits: sixteen keys at a time go to a ring of this warp as they are, where every lane later finds what it copied itself
      constexpr int kVectors8 = G::DP / 16, kPer8 = 32 / kVectors8, kPasses = 16 / kPer8;
      const int row8 = lane / kVectors8, vec8 = lane % kVectors8;
      const bool part8 = vec8 * 16 < c.head_dim;
      const long long bytes8 = row8 * c.s_token + vec8 * 16, pass8 = part8 ? kPer8 * c.s_token : 0;
      const uint32_t mine = raw + producer * (G::kRaw * G::kRawBytes) + lane * 16;
      const int n = 4 * x.nt;
      auto ask = [&](int q, uint32_t to) {  // (in_batch: its tile; a group of copies even where nothing is left to ask for)
        if (q < n) {
          const long long place = __shfl_sync(~0u, places, in_batch * 4 + (q & 3));
          if (place >= 0) {
            const uint8_t* src = cache + (part8 ? place + bytes8 : 0);
#pragma unroll
            for (int j = 0; j < kPasses; ++j, src += pass8) copy16(to + j * 512, src, part8);
          } else {
            const int key0 = begin_of(q >> 2) + (q & 3) * 16;
#pragma unroll 1
            for (int j = 0; j < kPasses; ++j) {
              const int key = key0 + j * kPer8 + row8;
              const bool asked = seen_by_some<EXTRA>(p, key, low, high);
              const long long at = asked ? cache_offset(c, load(table + (key >> c.page_shift)), x.h, key, p.status) : -1;
              copy16(to + j * 512, cache + (at >= 0 && part8 ? at + vec8 * 16 : 0), at >= 0 && part8);
            }
          }
          if ((q & 3) == 3 && ++in_batch == 8) {
            in_batch = 0;
            places = place_of((q >> 2) + 1, page_next);
            page_next = page_of((q >> 2) + 9);
          }
        }
        copies_commit();
      };
#pragma unroll 1
      for (int q = 0; q < G::kRaw; ++q) ask(q, mine + q * G::kRawBytes);
      uint32_t from = mine;
#pragma unroll 1
      for (int q = 0; q < n; ++q) {
        if ((q & 3) == 0) {
          go_on = arrived_at(sh, &sh.empty[slot], slot_phase, p.status);
          if (!go_on) break;
        }
        copies_wait<G::kRaw - 1>();
        const int row0 = upper * 64 + (q & 3) * 16 + row8;
        const uint32_t to = ring + slot * G::kSlot + vec8 / 4 * kBlock + row0 * 128;
        uint4 w[kPasses];
#pragma unroll
        for (int j = 0; j < kPasses; ++j) w[j] = lds128(from + j * 512);
#pragma unroll
        for (int j = 0; j < kPasses; ++j) {
          const uint32_t row = to + j * kPer8 * 128, at = vec8 * 2 ^ (row0 + j * kPer8);
          if constexpr (G::kInt8) {
            const uint32_t x8 = int8_biased(w[j].x), y8 = int8_biased(w[j].y), z8 = int8_biased(w[j].z), w8 = int8_biased(w[j].w);
            sts128(row + (at & 7) * 16, int8x2_to_f16x2(x8, 0x4140), int8x2_to_f16x2(x8, 0x4342), int8x2_to_f16x2(y8, 0x4140), int8x2_to_f16x2(y8, 0x4342));
            sts128(row + ((at ^ 1) & 7) * 16, int8x2_to_f16x2(z8, 0x4140), int8x2_to_f16x2(z8, 0x4342), int8x2_to_f16x2(w8, 0x4140), int8x2_to_f16x2(w8, 0x4342));
          } else {
            sts128(row + (at & 7) * 16, e4m3x2_to_f16x2(w[j].x), e4m3x2_to_f16x2(w[j].x >> 16), e4m3x2_to_f16x2(w[j].y), e4m3x2_to_f16x2(w[j].y >> 16));
            sts128(row + ((at ^ 1) & 7) * 16, e4m3x2_to_f16x2(w[j].z), e4m3x2_to_f16x2(w[j].z >> 16), e4m3x2_to_f16x2(w[j].w), e4m3x2_to_f16x2(w[j].w >> 16));
          }
        }
        ask(q + G::kRaw, from);
        from = from == mine + (G::kRaw - 1) * G::kRawBytes ? mine : from + G::kRawBytes;
        if ((q & 3) == 3) {
          fence_to_tensor_cores();
          if (!withheld(p, slot == 0)) mbar_arrive(&sh.full[slot]);
          if (slot == last_slot) {
            slot = first_slot;
            slot_phase ^= 1;
          } else {
            ++slot;
          }
        }
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < x.nt; ++i, ++in_batch) {
        if (in_batch == 8) {
          in_batch = 0;
          places = place_of(i, page_next);
          page_next = page_of(i + 8);
        }
        const int key0 = begin_of(i);
        const bool there4 = lane / 4 != in_batch || places >= 0;
        const bool whole = big_pages && all_seen_by_some<EXTRA>(p, key0, 64, low, high) && __all_sync(~0u, there4);
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
#pragma unroll 4
          for (int r = 0; r < 64; r += kPer) {
            const int row = r + my_row, key = key0 + row;
            const bool asked = seen_by_some<EXTRA>(p, key, low, high);
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
    }
    if (!go_on) break;
  }
  copies_wait_all();
}

// ---- the threads that issue the products -----------------------------------------------------------
enum Product { kLogits, kResults };
template <class G, int WHICH>
__device__ __forceinline__ void multiply(const AttentionParams& p, TcShared<G>& sh, uint32_t ring, uint32_t q_slots, uint32_t weights,
                                         uint32_t ones, uint32_t tmem) {
  constexpr int N = G::N;
  constexpr uint32_t kRowsDesc = instr_desc_f16(128, N);
  constexpr uint32_t kColumnsDesc = kRowsDesc | 1u << 15 | 1u << 16;  // A and B along their bytes
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    mbar_wait(bar, parity, &sh.abort, p.status);
    return *(volatile int*)&sh.abort == 0;
  };
  constexpr int kFirst = WHICH == kLogits ? 0 : G::kKeySlots, kLast = WHICH == kLogits ? G::kKeySlots - 1 : G::kSlots - 1;
  int slot = kFirst, open = 0;
  uint32_t phase = 0, open_phase = 0, u = 0;
#pragma unroll 1
  for (;;) {
    if (!wait(&sh.opened[open], open_phase)) return;
    const int nt = *(volatile int*)&sh.segments[open].nt;
    if (nt == 0) return;
    if (WHICH != kLogits) mbar_arrive(&sh.closed[open]);  // (nothing else of the segment is needed here)
#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const uint32_t buf = u & 1, pb = u % G::kPBuffers;
      if (WHICH == kLogits) {
        if (!wait(&sh.full[slot], phase) || !wait(&sh.s_free[buf], (u >> 1 & 1) ^ 1)) return;
      } else {
        if (!wait(&sh.full[slot], phase) || !wait(&sh.p_full[pb], u / G::kPBuffers & 1)) return;
      }
      fence_to_tensor_cores();
      tc_fence_after_sync();
      if (WHICH == kLogits) {
        const uint32_t keys = ring + slot * G::kSlot, q = q_slots + open * G::kQBytes;
#pragma unroll
        for (int ks = 0; ks < G::DP / 16; ++ks)
          mma_ss(tmem + buf * N, desc_rows(keys + ks / 4 * kBlock + ks % 4 * 32, 1024),
                 desc_rows(q + ks / 4 * G::kQBlock + ks % 4 * 32, 1024), kRowsDesc, ks ? 1 : 0);
        tc_commit(&sh.s_full[buf]);
        tc_commit(&sh.empty[slot]);
        if (i + 1 == nt) tc_commit(&sh.closed[open]);
      } else {
        const uint32_t w = weights + pb * G::kPBytes, values = ring + slot * G::kSlot;
#pragma unroll
        for (int ks = 0; ks < kTile / 16; ++ks) {
          const uint32_t v = values + ks * 2048;
          mma_ss(tmem + 2 * N, desc_columns(v, G::kSumRows ? ones - v : kBlock), desc_weights<G::kPRow>(w + ks * 16 * G::kPRow),
                 kColumnsDesc, i % kFold || ks ? 1 : 0);
        }
        tc_commit(&sh.p_done[pb]);
        tc_commit(&sh.empty[slot]);
      }
      if (slot == kLast) {
        slot = kFirst;
        phase ^= 1;
      } else {
        ++slot;
      }
    }
    if (++open == G::kOpen) {
      open = 0;
      open_phase ^= 1;
    }
  }
}

// All products that this thread has issued are complete, and what they signal has arrived, before tensor memory is freed and the block's shared
// memory goes to another: also where a wait ran out and nobody else has waited for them.  With a limit of its own (1 ms; a product takes
// well below one microsecond), since the others do not wait any more then.
__device__ __forceinline__ void drain_products(uint64_t* bar) {
  tc_commit(bar);
  for (int i = 0; i < 1000 && !mbar_try_wait(bar, 0); ++i) __nanosleep(1000);
}

// ---- softmax and results ---------------------------------------------------------------------------
// Whether a wait has run out is agreed upon where a segment begins, so that these warps always meet at the same barriers; what
// they compute of a segment whose copies did not come is thrown away with the call.
template <class G>
__device__ __forceinline__ void soften(const AttentionParams& p, TcShared<G>& sh, uint32_t ring, uint32_t weights, uint32_t tmem) {
  constexpr int N = G::N, DP = G::DP, kMine = G::kMine, EXTRA = G::EXTRA;
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int key = tid & 127, half = tid >> 7, mine = half * kMine;  // this thread's key, and the first of its rows
  const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);       // (lane 32 * (warp % 4) of tensor memory)
  auto wait = [&](uint64_t* bar, uint32_t parity) { mbar_wait(bar, parity, &sh.abort, p.status); };
  auto meet_half = [&] { named_bar_sync(1 + half, 128); };
  auto meet = [&] {
    named_bar_sync(3, kSoftmaxThreads);
    return true;
  };

  uint32_t u = 0;  // tiles so far
  int open = 0, odd = 0;
  uint32_t open_phase = 0;
#pragma unroll 1
  for (;; odd ^= 1) {
    wait(&sh.opened[open], open_phase);
    if (any_of(3, kSoftmaxThreads, *(volatile int*)&sh.abort)) return;
    const SegmentOf<EXTRA>& x = sh.segments[open];
    const int nt = x.nt, rows = x.rows;
    if (nt == 0) return;
    const Visible sees = visible(p, x);
    const bool several = x.n > 1;
    const int one_high = x.base_high;
    if (several) {
      for (int r = mine + key; r < mine + kMine; r += 128) sh.high[r] = x.base_high + (x.row0 + min(r, rows - 1)) / p.group;
      meet_half();
    }
    bool fresh = true;  // some row has not seen a key yet
    const float scale = p.scale_log2 * (G::F8 && c.k_scale ? load(c.k_scale + x.h) : 1.f);
    // (a hidden logit is an infinity, and would not stay one under 0: products of finite numbers times 1e-30 have weights of 1 all the same;
    // with a scale for each key they are multiplied with it and with `scale` first)
    const float factor = G::kScaled ? 1.f : scale == 0.f ? 1e-30f : scale, hidden = factor < 0.f ? INFINITY : -INFINITY;
    // kScaled: the sums are in units of `unit`, a power of two and not below any scale of a value so far.  This thread's scales are asked for
    // a tile ahead, the number of the page that they lie in two tiles ahead
    float unit = 0.f, inverse = 0.f;
    auto scale_page = [&](int i) {
      const int at = tile_of<EXTRA>(x, i) * kTile + key;
      return i < nt && seen_by_some<EXTRA>(p, at, sees.low_min, sees.high_max) ? load(c.table + x.b * c.table_stride + (at >> c.page_shift)) : -1;
    };
    auto scale_at = [&](const float* scales, int i, int page) {
      if ((unsigned)page >= (unsigned)c.pages) return 0.f;
      return scales ? load(scales + scale_offset(p, page, x.h, tile_of<EXTRA>(x, i) * kTile + key)) : 1.f;
    };
    float key_next = 0.f, value_next = 0.f;
    int page_next = -1;
    if constexpr (G::kScaled) {
      const int page = scale_page(0);
      page_next = scale_page(1);
      key_next = scale_at(p.scales.k, 0, page);
      value_next = scale_at(p.scales.v, 0, page);
    }
    float l[kMine];     // (kSumRows: not used)
#pragma unroll
    for (int r = 0; r < kMine; ++r) l[r] = 0.f;

#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const uint32_t buf = u & 1, pb = u % G::kPBuffers;
      const int pos0 = tile_of<EXTRA>(x, i) * kTile, pos = pos0 + key;
      const bool all = all_seen_by_some<EXTRA>(p, pos0, kTile, sees.low_max, sees.high_min);
      float key_factor = 1.f, value_scale = 1.f;
      if constexpr (G::kScaled) {
        key_factor = scale * key_next;
        value_scale = value_next;
        key_next = scale_at(p.scales.k, i + 1, page_next);
        value_next = scale_at(p.scales.v, i + 1, page_next);
        page_next = scale_page(i + 2);
      }
      wait(&sh.s_full[buf], u >> 1 & 1);
      tc_fence_after_sync();
      float y[kMine];
      load_columns(lanes + buf * N + mine, y);
      tc_wait_ld();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.s_free[buf]);
      const bool plain = G::kScaled && all && i > 0;  // (nothing to hide, no bases to look for: multiplied where the bases are subtracted)
      if (G::kScaled && !plain) {
#pragma unroll
        for (int r = 0; r < kMine; ++r) y[r] *= key_factor;
      }
      auto hides = [&](int r) {
        const int high = several ? sh.high[mine + r] : one_high;
        return pos >= high || (p.window && pos < high - p.window && (EXTRA == kNoExtra || pos >= p.sinks));
      };
      if (!all) {  // (a logit that becomes -inf whatever it is multiplied with)
#pragma unroll
        for (int r = 0; r < kMine; ++r) {
          // (without sinks as an expression of its own: through `hides` the compiler took another order, and prompts of 2048 tokens 3 % longer)
          const int high = several ? sh.high[mine + r] : one_high;
          if (EXTRA == kNoExtra ? pos >= high || (p.window && pos < high - p.window) : hides(r)) y[r] = hidden;
        }
      }
      if (i == 0) {  // bases to begin with: the largest logit of a row over the 32 keys of one warp, a quarter of the rows each
        bool none = false;
#pragma unroll
        for (int r = 0; r < kMine; r += 4) {
          // (row r + warp % 4, without an index that is not known to the compiler)
          const float z = (warp & 2) ? ((warp & 1) ? y[r + 3] : y[r + 2]) : ((warp & 1) ? y[r + 1] : y[r]);
          const float top = warp_max(z == hidden ? kNone : z * factor) - kBelow;
          none |= top == kNone;
          if (lane == 0) {
            sh.largest[mine + r + (warp & 3)] = top;
            sh.base[mine + r + (warp & 3)] = top == kNone ? 0.f : top;
          }
        }
        if constexpr (G::kScaled) {  // and the unit, which would move with the bases otherwise (3000 cycles)
          const float top = warp_max(finite_or_zero(value_scale));
          if (lane == 0) sh.scale_tops[warp] = top;
        }
        fresh = any_of(1 + half, 128, none);
        if constexpr (G::kScaled) {
          const float* const tops = sh.scale_tops + half * 4;
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
          if (top > 0.f) {
            unit = power_above(top);
            inverse = 1.f / unit;
          }
        }
      }
      // logits in units of log2, relative to the bases; `over`: some are too far above, or there is no base yet
      float top = kNone;
      const float times = plain ? key_factor : factor;
#pragma unroll
      for (int r = 0; r < kMine; r += 4) {
        const float4 base = *reinterpret_cast<const float4*>(&sh.base[mine + r]);
        if constexpr (G::kScaled) {
          const f32x2 t2 = pack2(times, times);
          unpack2(fma2(pack2(y[r], y[r + 1]), t2, pack2(-base.x, -base.y)), y[r], y[r + 1]);
          unpack2(fma2(pack2(y[r + 2], y[r + 3]), t2, pack2(-base.z, -base.w)), y[r + 2], y[r + 3]);
        } else {
          y[r] = fmaf(y[r], times, -base.x);
          y[r + 1] = fmaf(y[r + 1], times, -base.y);
          y[r + 2] = fmaf(y[r + 2], times, -base.z);
          y[r + 3] = fmaf(y[r + 3], times, -base.w);
        }
        top = fmaxf(fmaxf(fmaxf(top, y[r]), fmaxf(y[r + 1], y[r + 2])), y[r + 3]);
      }
      // by any row: weights of 0, whatever the bases are
      const bool unseen = (pos0 + kTile <= sees.low_min && (EXTRA == kNoExtra || pos0 >= p.sinks)) || pos0 >= sees.high_max;
      const bool fold = i % kFold == 0 && i > 0;
      const bool over = (fresh && !unseen) || fold || top > kSlack || (G::kScaled && finite_or_zero(value_scale) > unit);
      if (any_of(1 + half, 128, over)) {  // move the bases: the largest logit of every row over the 128 keys
#pragma unroll
        for (int r = 0; r < kMine; ++r) {
          const float top = warp_max(y[r]);
          if (lane == 0) sh.tops[warp & 3][mine + r] = top;
        }
        float ratio = 1.f;
        if constexpr (G::kScaled) {
          const float top = warp_max(finite_or_zero(value_scale));
          if (lane == 0) sh.scale_tops[warp] = top;
        }
        meet_half();
        if constexpr (G::kScaled) {
          const float* const tops = sh.scale_tops + half * 4;
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
          if (top > unit) {
            const float now = power_above(top);
            ratio = unit / now;
            unit = now;
            inverse = 1.f / now;
          }
        }
        for (int r = mine + key; r < mine + kMine; r += 128) {
          const float old = sh.largest[r], from = sh.base[r];
          const float top = fmaxf(fmaxf(sh.tops[0][r], sh.tops[1][r]), fmaxf(sh.tops[2][r], sh.tops[3][r])) + from - kBelow;
          const float now = fmaxf(old, top), to = now == kNone ? 0.f : now;
          sh.alpha[r] = exp2_fast(old - to);
          sh.tops[0][r] = from - to;
          sh.largest[r] = now;
          sh.base[r] = to;
        }
        meet_half();
        bool none = false;
#pragma unroll
        for (int r = 0; r < kMine; ++r) {
          y[r] += sh.tops[0][mine + r];
          if (!G::kSumRows) l[r] *= i ? sh.alpha[mine + r] : 1.f;
          none |= sh.largest[mine + r] == kNone;
        }
        fresh = none;  // (the same for all of them)
        if (i > 0) {  // the sums so far, when the products that add to them are done
          const uint32_t before = u - 1;
          wait(&sh.p_done[before % G::kPBuffers], before / G::kPBuffers & 1);
          tc_fence_after_sync();
          float z[8];
#pragma unroll 1
          for (int r0 = 0; r0 < kMine; r0 += 8) {
            load_columns(lanes + 2 * N + mine + r0, z);
            tc_wait_ld();
#pragma unroll
            for (int r = 0; r < 8; ++r) z[r] *= G::kScaled ? sh.alpha[mine + r0 + r] * ratio : sh.alpha[mine + r0 + r];
            store_columns(lanes + 2 * N + mine + r0, z);
            if (i >= kFold) {  // those that were put aside, and these to them
              float aside[8];
              load_columns(lanes + 3 * N + mine + r0, aside);
              tc_wait_ld();
#pragma unroll
              for (int r = 0; r < 8; ++r) 
                aside[r] = (i > kFold ? aside[r] * (G::kScaled ? sh.alpha[mine + r0 + r] * ratio : sh.alpha[mine + r0 + r]) : 0.f) + (fold ? z[r] : 0.f);
              store_columns(lanes + 3 * N + mine + r0, aside);
            }
          }
          tc_wait_st();
        }
        meet_half();  // (alpha and tops are free again)
      }
      // weights, rounded to fp16 for the product (kBelow in attention.cuh)
      wait(&sh.p_done[pb], (u / G::kPBuffers & 1) ^ 1);  // (those that were there are multiplied)
      const uint32_t w_to = weights + pb * G::kPBytes + key * G::kPRow;
      const float value_factor = value_scale * inverse;
#pragma unroll
      for (int r = 0; r < kMine; r += 8) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          y[r + e] = exp2_fast(y[r + e]);
          y[r + e + 1] = exp2_fast(y[r + e + 1]);
          if constexpr (G::kScaled) {  // (0 where a row does not see the key, also where its scale is not finite)
            float lo, hi;
            unpack2(mul2(pack2(y[r + e], y[r + e + 1]), pack2(value_factor, value_factor)), lo, hi);
            w[e / 2] = half2_bits(lo, hi);
          } else {
            w[e / 2] = half2_bits(y[r + e], y[r + e + 1]);
          }
          if (!G::kSumRows) {
            if constexpr (G::kScaled) {
              unpack2(add2(pack2(l[r + e], l[r + e + 1]), pack2(y[r + e], y[r + e + 1])), l[r + e], l[r + e + 1]);
            } else {
              l[r + e] += y[r + e];
              l[r + e + 1] += y[r + e + 1];
            }
          }
        }
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(w_to + (((mine + r) / 8) ^ swizzle_of<G::kPRow>(key)) * 16),
                     "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
      }
      if (G::kScaled && !all && !(fabsf(value_factor) < INFINITY)) {  // (0 where a row does not see the key, also where its scale is not finite)
#pragma unroll 1
        for (int r = 0; r < kMine; ++r)
          if (hides(r)) asm volatile("st.shared.u16 [%0], %1;" ::"r"(w_to + (((mine + r) / 8) ^ swizzle_of<G::kPRow>(key)) * 16 + (r & 7) * 2), "h"((uint16_t)0) : "memory");
      }
      tc_fence_before_sync();
      if (!G::kInt8 && several && !all && half == 0) {  // values of keys that not every row sees: what is not finite is left out
        const uint32_t v_slot = G::kKeySlots + u % G::kValueSlots;
        wait(&sh.full[v_slot], u / G::kValueSlots & 1);
        if ((pos >= sees.high_min && pos < sees.high_max) || (pos >= sees.low_min && pos < sees.low_max && (EXTRA == kNoExtra || pos >= p.sinks))) {
          bool found = false;
#pragma unroll 1
          for (int vec = 0; vec < DP / 8; ++vec)
            found |= clean_vector<false>(ring + v_slot * G::kSlot + vec / 8 * kBlock + key * 128 + ((vec ^ key) & 7) * 16);
          if (found) sh.not_finite[odd] = 1;
        }
      }
      fence_to_tensor_cores();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[pb]);
    }

    // ---- results: lane d has element d of all rows; the sums of the weights go to `alpha`
    if (!G::kSumRows) {
      // lanes exchange halves of their sums until each has all of one row (of `same` lanes that end with the same one)
      constexpr int kSame = 32 / kMine;
#pragma unroll
      for (int n = kMine / 2, bit = 16; n >= 1; n /= 2, bit /= 2) {
#pragma unroll
        for (int r = 0; r < n; ++r) {
          const float mine_of = (lane & bit) ? l[r + n] : l[r], other = (lane & bit) ? l[r] : l[r + n];
          l[r] = mine_of + __shfl_xor_sync(~0u, other, bit);
        }
      }
#pragma unroll
      for (int bit = kSame / 2; bit >= 1; bit /= 2) l[0] += __shfl_xor_sync(~0u, l[0], bit);
      if (lane % kSame == 0) sh.tops[warp & 3][mine + lane / kSame] = l[0];
    }
    const uint32_t last = u - 1;
    wait(&sh.p_done[last % G::kPBuffers], last / G::kPBuffers & 1);
    tc_fence_after_sync();
    if (nt > kFold) {  // what was put aside joins the rest
#pragma unroll 1
      for (int r0 = 0; r0 < kMine; r0 += 8) {
        float z[8], aside[8];
        load_columns(lanes + 2 * N + mine + r0, z);
        load_columns(lanes + 3 * N + mine + r0, aside);
        tc_wait_ld();
#pragma unroll
        for (int r = 0; r < 8; ++r) z[r] += aside[r];
        store_columns(lanes + 2 * N + mine + r0, z);
      }
      tc_wait_st();
    }
    if (G::kSumRows && (warp & 3) == 2) {  // (lanes 64 - 127 all have them)
      float z[kMine];
      load_columns(lanes + 2 * N + mine, z);
      tc_wait_ld();
#pragma unroll
      for (int r = 0; r < kMine; ++r)
        if (lane == 0) sh.alpha[mine + r] = z[r];
    }
    meet();
    if (!G::kSumRows) {
      if (tid < N) sh.alpha[tid] = (sh.tops[0][tid] + sh.tops[1][tid]) + (sh.tops[2][tid] + sh.tops[3][tid]);
      meet();
    }
    if (tid == 0) sh.not_finite[odd ^ 1] = 0;
    const bool whole = x.c0 == x.c1;
    constexpr int kLine = part_line(DP);
    // row after row: its token and its head of the group, and where it goes
    int token = (x.row0 + mine) / p.group, head = x.row0 + mine - token * p.group;
    uint16_t* to_out = p.out + ((long long)(x.first + token) * p.q_heads + x.h * p.group + head) * c.head_dim + key;
    float* to_part = part_of(p, x, blockIdx.x, N, DP) + mine * kLine;
    const int next_token = (p.q_heads - p.group) * c.head_dim;
    const float values_of = G::kScaled ? unit : G::F8 && c.v_scale ? load(c.v_scale + x.h) : 1.f;
    auto give = [&](int r, float z) {
      const float sum = sh.alpha[r];
      if (whole) {
        const __half y = __float2half_rn(x.base_high + token <= 0 ? 0.f : __fdividef(z * values_of, sum));
        if (key < c.head_dim) *to_out = *reinterpret_cast<const uint16_t*>(&y);
        to_out += c.head_dim;
        if (++head == p.group) {
          head = 0;
          ++token;
          to_out += next_token;
        }
      } else {
        if (key < DP) to_part[key] = G::kScaled ? z * unit : z;
        if (key == 0) *reinterpret_cast<float2*>(to_part + DP) = make_float2(sh.largest[r], sum);
        to_part += kLine;
      }
    };
    // (lanes with and without an element of the head part in `give`, and meet again before the warp reads tensor memory as one)
    if (several && *(volatile int*)&sh.not_finite[odd]) {  // (one column at a time, with what was left out)
#pragma unroll 1
      for (int r = mine; r < min(rows, mine + kMine); ++r) {
        float z;
        load_column(lanes + 2 * N + r, z);
        tc_wait_ld();
        give(r, z + not_finite_sum<G::F8>(p, x, sees, kTile, r, key));
        __syncwarp();
      }
    } else {
#pragma unroll 1
      for (int r0 = mine; r0 < min(rows, mine + kMine); r0 += 8) {
        float z[8];
        load_columns(lanes + 2 * N + r0, z);
        tc_wait_ld();
        if (G::kScaled && !whole) {  // (rows that are not there have room, too)
          if (key < DP) {
#pragma unroll
            for (int r = 0; r < 8; ++r) to_part[r * kLine + key] = z[r] * unit;
          }
          if (key < 8) *reinterpret_cast<float2*>(to_part + key * kLine + DP) = make_float2(sh.largest[r0 + key], sh.alpha[r0 + key]);
          to_part += 8 * kLine;
          __syncwarp();
          continue;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r0 + r < rows) give(r0 + r, z[r]);
        __syncwarp();
      }
    }
    tc_fence_before_sync();
    auto write_out = [&](int r, int d, float4 z, float li) { write_four(p, x, r, d, z, li); };
    if (!whole) join_parts<N, DP, kSoftmaxThreads, 4, 2>(p, x, tid, &sh.arrived, sh.ml, meet, write_out);
    meet();  // (bases and notes are free again)
    if (lane == 0) mbar_arrive(&sh.closed[open]);
    if (++open == G::kOpen) {
      open = 0;
      open_phase ^= 1;
    }
  }
}

template <int DP, int N, bool F8, int EXTRA>
__global__ void __launch_bounds__(kThreads, 1) attention_tc_kernel(const AttentionParams p) {
  using G = TcGeometry<DP, N, F8, EXTRA>;
  extern __shared__ uint8_t smem[];
  __shared__ TcShared<G> sh;
  const uint32_t ring = (smem_u32(smem) + 1023u) & ~1023u;
  const uint32_t q_slots = ring + G::kSlots * G::kSlot, weights = q_slots + G::kOpen * G::kQBytes, ones = weights + G::kPBuffers * G::kPBytes;
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < G::kSlots; ++i) {
      mbar_init(&sh.full[i], 32 * kProducers / 2);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < G::kOpen; ++i) {
      mbar_init(&sh.opened[i], 32 * kProducers + 1);  // the copies of all lanes, and the note itself
      mbar_init(&sh.closed[i], kSoftmaxWarps + kIssuers);  // the softmax warps, the issuers, and for one of them its last product that reads Q
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], kSoftmaxWarps);
    }
    for (int i = 0; i < G::kPBuffers; ++i) {
      mbar_init(&sh.p_full[i], kSoftmaxWarps);
      mbar_init(&sh.p_done[i], 1);
    }
    for (int i = 0; i < kIssuers; ++i) mbar_init(&sh.drained[i], 1);
    sh.abort = 0;
    sh.not_finite[0] = sh.not_finite[1] = 0;
  }
  for (int i = threadIdx.x; i < G::kOnes / 16; i += kThreads)
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ones + i * 16), "r"(0x3c003c00u) : "memory");
  if (G::kSumRows) fence_to_tensor_cores();
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
  // (the order of the roles in the file decides how their loops share the nearest instruction caches, and is the best of three: with the
  // copies in front of the products prompts of 2048 tokens take 3 % longer, with the softmax last drafts 1 % and windows 3 %)
  if (warp < kSoftmaxWarps) {
    if constexpr (G::kSoftmaxRegs > 0) setmaxnreg_inc<G::kSoftmaxRegs>();
    soften<G>(p, sh, ring, weights, tmem);
  } else {
    if constexpr (G::kSoftmaxRegs > 0) setmaxnreg_dec<G::kOtherRegs>();
    const int w = warp - kSoftmaxWarps;
    if (w >= kProducers && w < kProducers + kIssuers && threadIdx.x % 32 == 0) {
      if (w == kProducers)
        multiply<G, kLogits>(p, sh, ring, q_slots, weights, ones, tmem);
      else
        multiply<G, kResults>(p, sh, ring, q_slots, weights, ones, tmem);
      drain_products(&sh.drained[w - kProducers]);
    } else if (w < kProducers) {
      produce<G>(p, sh, w / 2, w % 2, ring, q_slots, ones + G::kOnes);
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

template <int DP, int N, bool F8, int EXTRA>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  using G = TcGeometry<DP, N, F8, EXTRA>;
  return launch_ranges<attention_tc_kernel<DP, N, F8, EXTRA>, G::kSmem, kThreads, N, kTile>(p, sm_count, stream, G::kSoftmaxRegs ? 128 : 0);
}
template <int DP, int EXTRA>
cudaError_t launch_rows(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  const long long rows = usual_rows(p);
  if (rows <= 16) return launch<DP, 16, false, EXTRA>(p, sm_count, stream);
  if (rows <= 32) return launch<DP, 32, false, EXTRA>(p, sm_count, stream);
  return launch<DP, 64, false, EXTRA>(p, sm_count, stream);
}

}  // namespace
}  // namespace marlin_b200
