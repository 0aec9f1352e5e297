// Attention of new tokens over an fp16 cache where a key head has more than eight rows (heads that share keys, several new
// tokens): the same ranges, segments and parts as attention.cu, with the products on the fifth-generation tensor cores.
//
// A tile has 128 keys.  S^T = K Q^T with the keys as the 128 rows of the product and the rows of Q as its columns, so that thread k of
// the softmax warps has key k and all N rows of it in its lane of tensor memory; the weights go to shared memory as P, and
// O^T += V^T P^T has the elements of the head as its 128 rows.  Both products are as narrow as there are rows: 128 x N x 16 a step.
// What a thread sees of a row is one key, so nothing is summed over keys by threads at all: the sums of the weights are a third product,
// of a matrix of ones with P, and the largest logits are looked for only when one exceeds the base of its row by kSlack
// (attention.cuh), which needs the sums in tensor memory to be rescaled.
//
// Warps: 0 - 7 softmax and results (lane quarter w % 4 of tensor memory; 0 - 3 the first half of the rows, 4 - 7 the second, each
// half with bases of its own), 8 - 11 copies (32 keys of every tile each), 12 - 14 issue one of the three products each: an issue
// costs its thread some 75 cycles and a commit 125, and with one thread for all of them (24 products and four commits a tile of
// 128 x 128) everybody waited for it.  Keys and values take slots of the ring in turn.  Tensor memory: S twice, O, the sums of the weights; N columns each.
#include "attention.cuh"
#include "tc_utils.cuh"

namespace marlin_b200 {
namespace {

constexpr int kTile = 128;
constexpr int kLead = 1;                 // what an item costs beside its tiles, in tiles
constexpr int kBlock = kTile * 128;      // 64 elements of the keys of a tile: rows of 128 bytes, as the swizzle has them
constexpr int kSoftmaxWarps = 8;
constexpr int kSoftmaxThreads = kSoftmaxWarps * 32;
constexpr int kProducers = 4;
constexpr int kIssuers = 3;
constexpr int kThreads = kSoftmaxThreads + (kProducers + kIssuers) * 32;

// DP: head_dim rounded up to 64 or 128; N: rows of a block
template <int DP_, int N_>
struct TcGeometry {
  static constexpr int DP = DP_, N = N_;
  static constexpr int kHalves = DP / 64;
  static constexpr int kSlot = kHalves * kBlock;   // the keys (or the values) of a tile
  static constexpr int kQBlock = N * 128;          // 64 elements of the rows
  static constexpr int kQBytes = kHalves * kQBlock;
  static constexpr int kOpen = N == 128 ? 1 : 2;   // segments that can be open at a time
  static constexpr int kPBytes = 2 * kQBlock;      // weights: 64 keys of the rows, twice
  static constexpr int kPBuffers = N == 128 ? 1 : 2;
  static constexpr int kOnes = 1024;               // eight rows of 64 ones
  static constexpr int kRest = kOpen * kQBytes + kPBuffers * kPBytes + kOnes;
  static constexpr int kSlots = (222 * 1024 - kRest) / kSlot > 12 ? 12 : (222 * 1024 - kRest) / kSlot;
  static constexpr int kSmem = kSlots * kSlot + kRest + 1024;  // (the ring begins at a multiple of 1024)
  static constexpr int kColumns = 4 * N < 32 ? 32 : 4 * N;     // of tensor memory: S, S, O, sums of weights
  static constexpr int kMine = N / 2;                          // rows of a half of the softmax warps
  static constexpr int kChunk = kMine < 16 ? kMine : 16;       // columns that a thread holds at a time
  static_assert(kSlots >= 3 && kColumns <= 512, "ring");
};

template <class G>
struct TcShared {
  uint64_t full[G::kSlots], empty[G::kSlots];
  uint64_t opened[G::kOpen], closed[G::kOpen];
  uint64_t s_full[2], s_free[2];                       // logits are there; have been read
  uint64_t p_full[G::kPBuffers], p_done[G::kPBuffers]; // weights are there; have been multiplied
  Segment segments[G::kOpen];
  float2 ml[G::N];
  alignas(16) float base[G::N];  // of the rows, read four at a time; 0 where a row has seen nothing
  float largest[G::N];    // the same, -inf where a row has seen nothing
  float alpha[G::N];      // what the sums are multiplied with when the base moves
  float tops[4][G::N];
  int high[G::N];         // positions below which the rows see
  int abort;
  int arrived;
  int not_finite[2];
  uint32_t tmem;
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
// what this thread (or another whose arrival it has seen) wrote to shared memory can be read by the tensor cores
__device__ __forceinline__ void fence_to_tensor_cores() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void store_half(uint32_t addr, float x) {
  const __half h = __float2half_rn(x);
  asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"(*reinterpret_cast<const uint16_t*>(&h)) : "memory");
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
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
template <int C>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&x)[C]) {
  if constexpr (C == 16)
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
template <class G>
__device__ __forceinline__ void produce(const AttentionParams& p, TcShared<G>& sh, int producer, uint32_t ring, uint32_t q_slots) {
  const KvCacheView& c = p.cache;
  const int lane = threadIdx.x & 31;
  Range<G::N, kTile, kLead> range;
  range.begin(p);

  constexpr int kVectors = G::DP / 8;
  constexpr int kPer = 32 / kVectors;
  const int my_row = lane / kVectors, my_vec = lane % kVectors;
  const bool my_part = my_vec * 8 < c.head_dim;
  const bool big_pages = c.page_shift >= 4;  // sixteen keys lie in one page
  int slot = 0, open = 0;
  uint32_t slot_phase = 1, open_phase = 1;
#pragma unroll 1
  for (;;) {
    const Segment x = range.next(p);
    if (!arrived_at(sh, &sh.closed[open], open_phase, p.status)) break;
    if (lane == 0 && producer == 0) sh.segments[open] = x;
    if (x.nt > 0) {  // Q; rows and elements that are not there are zeros
#pragma unroll 1
      for (int i = producer * 32 + lane; i < G::N * kVectors; i += 32 * kProducers) {
        const int r = i / kVectors, vec = i % kVectors;
        const int token = (x.row0 + r) / p.group, head = x.h * p.group + (x.row0 + r) - token * p.group;
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

    const Visible v = visible(p, x);
    const int* const table = c.table + x.b * c.table_stride;
    const int key_first = x.tile * kTile + producer * 32;
    const int low = max(v.low_min, x.tile * kTile), high = min(v.high_max, (x.tile + x.nt) * kTile);
    // pages: of the two sixteens of this warp in sixteen tiles, a lane each, and in the next sixteen; or, where pages are smaller,
    // of the 32 keys of one tile and of the next one.  INT_MIN where no key is asked for
    auto page_of = [&](int i) {
      const int key = key_first + (big_pages ? (i + lane / 2) * kTile + lane % 2 * 16 : i * kTile + lane);
      return key < high && key + (big_pages ? 16 : 1) > low ? __ldg(table + (key >> c.page_shift)) : INT_MIN;
    };
    const int batch = big_pages ? 16 : 1;
    const long long head_bytes = (x.h * c.s_head + my_row * c.s_token) * 2 + my_vec * 16;
    const long long pass = my_part ? kPer * c.s_token * 2 : 0;
    int pages = page_of(0), pages_next = page_of(batch), in_batch = 0;
    bool go_on = true;
#pragma unroll 1
    for (int i = 0; i < x.nt && go_on; ++i, ++in_batch) {
      if (in_batch == batch) {
        in_batch = 0;
        pages = pages_next;
        pages_next = page_of(i + batch);
      }
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {  // keys, values
        if (!arrived_at(sh, &sh.empty[slot], slot_phase, p.status)) {
          go_on = false;
          break;
        }
        const uint8_t* const cache = static_cast<const uint8_t*>(which ? c.v : c.k);
#pragma unroll 1
        for (int j = 0; j < 2; ++j) {
          const int key0 = key_first + i * kTile + j * 16, row0 = producer * 32 + j * 16;
          const uint32_t to = ring + slot * G::kSlot + my_vec / 8 * kBlock + (row0 + my_row) * 128;
          const int page = __shfl_sync(~0u, pages, big_pages ? in_batch * 2 + j : 0);
          if (big_pages && key0 >= low && key0 + 16 <= high && (unsigned)page < (unsigned)c.pages) {
            const uint8_t* src = cache + (my_part ? (page * c.s_page + (key0 & ((1 << c.page_shift) - 1)) * c.s_token) * 2 + head_bytes : 0);
#pragma unroll
            for (int r = 0; r < 16; r += kPer) {
              copy16(to + r * 128 + ((my_vec ^ (r + my_row)) & 7) * 16, src, my_part);
              src += pass;
            }
          } else {
#pragma unroll 1
            for (int r = 0; r < 16; r += kPer) {
              const int key = key0 + r + my_row;
              const int mine = __shfl_sync(~0u, pages, big_pages ? in_batch * 2 + j : j * 16 + r + my_row);
              const long long from = key >= low && key < high ? cache_offset(c, mine, x.h, key, p.status) : -1;
              const bool there = from >= 0 && my_part;
              copy16(to + r * 128 + ((my_vec ^ (r + my_row)) & 7) * 16, cache + (there ? from * 2 + my_vec * 16 : 0), there);
            }
          }
        }
        copies_arrive(&sh.full[slot]);
        if (++slot == G::kSlots) {
          slot = 0;
          slot_phase ^= 1;
        }
      }
    }
    if (!go_on) break;
  }
  copies_wait_all();
}

// ---- the threads that issue the products -----------------------------------------------------------
enum Product { kLogits, kResults, kSums };
template <class G, int WHICH>
__device__ __forceinline__ void multiply(const AttentionParams& p, TcShared<G>& sh, uint32_t ring, uint32_t q_slots, uint32_t weights,
                                         uint32_t ones, uint32_t tmem) {
  constexpr int N = G::N;
  constexpr uint32_t kRowsDesc = instr_desc_f16(128, N);
  constexpr uint32_t kColumnsDesc = kRowsDesc | 1u << 15;  // A along its bytes
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    mbar_wait(bar, parity, &sh.abort, p.status);
    return *(volatile int*)&sh.abort == 0;
  };
  int slot = WHICH == kLogits ? 0 : 1, open = 0;  // slots go round: keys of tile u, values of tile u
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
        if (WHICH == kResults && !wait(&sh.full[slot], phase)) return;
        if (!wait(&sh.p_full[pb], u / G::kPBuffers & 1)) return;
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
          const uint64_t b = desc_rows(w + ks / 4 * G::kQBlock + ks % 4 * 32, 1024);
          if (WHICH == kResults)
            mma_ss(tmem + 2 * N, desc_columns(values + ks * 2048, G::kHalves == 2 ? kBlock : 0), b, kColumnsDesc, i || ks ? 1 : 0);
          else
            mma_ss(tmem + 3 * N, desc_rows(ones, 0), b, kRowsDesc, i || ks ? 1 : 0);
        }
        tc_commit(&sh.p_done[pb]);
        if (WHICH == kResults) tc_commit(&sh.empty[slot]);
      }
      slot += 2;
      if (slot >= G::kSlots) {
        slot -= G::kSlots;
        phase ^= 1;
      }
    }
    if (++open == G::kOpen) {
      open = 0;
      open_phase ^= 1;
    }
  }
}

// ---- softmax and results ---------------------------------------------------------------------------
// Whether a wait has run out is agreed upon where a segment begins, so that these warps always meet at the same barriers; what
// they compute of a segment whose copies did not come is thrown away with the call.
template <class G>
__device__ __forceinline__ void soften(const AttentionParams& p, TcShared<G>& sh, uint32_t ring, uint32_t weights, uint32_t tmem) {
  constexpr int N = G::N, DP = G::DP, kMine = G::kMine, kChunk = G::kChunk;
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
  // where this thread's key lies in the weights: byte of row r = w_key + r * 128, with the 16-byte vectors of a row permuted by r
  const uint32_t w_key = key / 64 * G::kQBlock + key % 8 * 2 + mine * 128, w_vec = key % 64 / 8;
#pragma unroll 1
  for (;; odd ^= 1) {
    wait(&sh.opened[open], open_phase);
    if (any_of(3, kSoftmaxThreads, *(volatile int*)&sh.abort)) return;
    const Segment& x = sh.segments[open];
    const int nt = x.nt, rows = x.rows;
    if (nt == 0) return;
    const Visible sees = visible(p, x);
    const bool several = x.n > 1;
    for (int r = mine + key; r < mine + kMine; r += 128) {
      sh.largest[r] = kNone;
      sh.base[r] = 0.f;
      sh.high[r] = several ? x.base_high + (x.row0 + min(r, rows - 1)) / p.group : x.base_high;
    }
    meet_half();
    bool fresh = true;  // some row has not seen a key yet

#pragma unroll 1
    for (int i = 0; i < nt; ++i, ++u) {
      const uint32_t buf = u & 1, pb = u % G::kPBuffers;
      const int pos0 = (x.tile + i) * kTile, pos = pos0 + key;
      const bool all = pos0 >= sees.low_max && pos0 + kTile <= sees.high_min;
      const uint32_t logits = lanes + buf * N + mine, w_to = weights + pb * G::kPBytes + w_key;
      wait(&sh.s_full[buf], u >> 1 & 1);
      tc_fence_after_sync();
      auto seen = [&](int r) {
        const int high = sh.high[mine + r];
        return all || (pos < high && !(p.window && pos < high - p.window));
      };
      if (i == 0) {  // bases to begin with: the largest logit of a row over the 32 keys of one warp, a quarter of the rows each
#pragma unroll 1
        for (int c0 = 0; c0 < kMine; c0 += kChunk) {
          float y[kChunk];
          load_columns(logits + c0, y);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < kChunk; r += 4) {
            // (row r + warp % 4, without an index that is not known to the compiler)
            const float z = (warp & 2) ? ((warp & 1) ? y[r + 3] : y[r + 2]) : ((warp & 1) ? y[r + 1] : y[r]);
            const int row = c0 + r + (warp & 3);
            const float top = warp_max(seen(row) ? z * p.scale_log2 : kNone);
            if (lane == 0) {
              sh.largest[mine + row] = top;
              sh.base[mine + row] = top == kNone ? 0.f : top;
            }
          }
        }
        meet_half();
        bool none = false;
        for (int r = lane; r < kMine; r += 32) none |= *(volatile float*)&sh.largest[mine + r] == kNone;
        fresh = __any_sync(~0u, none);
      }
      wait(&sh.p_done[pb], (u / G::kPBuffers & 1) ^ 1);  // (the weights that were there are multiplied)

      // weights relative to the bases as they are; `over`: some logit is too far above its base (or there is none yet), and
      // all of it is done again
      bool over = fresh;
      auto weigh = [&](bool look) {
#pragma unroll 1
        for (int c0 = 0; c0 < kMine; c0 += kChunk) {
          float y[kChunk];
          load_columns(logits + c0, y);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < kChunk; r += 4) {
            const float4 base = *reinterpret_cast<const float4*>(&sh.base[mine + c0 + r]);
            y[r] = fmaf(y[r], p.scale_log2, -base.x);
            y[r + 1] = fmaf(y[r + 1], p.scale_log2, -base.y);
            y[r + 2] = fmaf(y[r + 2], p.scale_log2, -base.z);
            y[r + 3] = fmaf(y[r + 3], p.scale_log2, -base.w);
          }
          if (!all) {
#pragma unroll
            for (int r = 0; r < kChunk; ++r)
              if (!seen(c0 + r)) y[r] = kNone;
          }
          if (look) {
#pragma unroll
            for (int r = 0; r < kChunk; ++r) over |= y[r] > kSlack;
          }
#pragma unroll
          for (int r = 0; r < kChunk; ++r) store_half(w_to + (c0 + r) * 128 + (w_vec ^ (r & 7)) * 16, exp2_fast(y[r]));
        }
      };
      weigh(true);
      over = any_of(1 + half, 128, over);
      if (over) {  // move the bases: the largest logit of every row over the 128 keys
#pragma unroll 1
        for (int c0 = 0; c0 < kMine; c0 += kChunk) {
          float y[kChunk];
          load_columns(logits + c0, y);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < kChunk; ++r) {
            const float top = warp_max(seen(c0 + r) ? y[r] * p.scale_log2 : kNone);
            if (lane == 0) sh.tops[warp & 3][mine + c0 + r] = top;
          }
        }
        meet_half();
        for (int r = mine + key; r < mine + kMine; r += 128) {
          const float old = sh.largest[r];
          const float now = fmaxf(fmaxf(fmaxf(old, sh.tops[0][r]), fmaxf(sh.tops[1][r], sh.tops[2][r])), sh.tops[3][r]);
          const float base = now == kNone ? 0.f : now;
          sh.alpha[r] = exp2_fast(old - base);
          sh.largest[r] = now;
          sh.base[r] = base;
        }
        meet_half();
        bool none = false;
        for (int r = lane; r < kMine; r += 32) none |= *(volatile float*)&sh.largest[mine + r] == kNone;
        fresh = __any_sync(~0u, none);
        if (i > 0) {  // the sums so far, when the products that add to them are done
          const uint32_t before = u - 1;
          wait(&sh.p_done[before % G::kPBuffers], before / G::kPBuffers & 1);
          tc_fence_after_sync();
#pragma unroll 1
          for (int c0 = 0; c0 < 2 * kMine; c0 += kChunk) {
            const uint32_t sums = lanes + (c0 < kMine ? 2 * N : 3 * N - kMine) + mine + c0;
            float y[kChunk];
            load_columns(sums, y);
            tc_wait_ld();
#pragma unroll
            for (int r = 0; r < kChunk; ++r) y[r] *= sh.alpha[mine + c0 % kMine + r];
            store_columns(sums, y);
          }
          tc_wait_st();
        }
        weigh(false);
      }
      tc_fence_before_sync();
      if (several && !all && half == 0) {  // values of keys that not every row sees: what is not finite is left out
        const uint32_t v_slot = (2 * u + 1) % G::kSlots;
        wait(&sh.full[v_slot], (2 * u + 1) / G::kSlots & 1);
        if ((pos >= sees.high_min && pos < sees.high_max) || (pos >= sees.low_min && pos < sees.low_max)) {
          bool found = false;
#pragma unroll 1
          for (int vec = 0; vec < DP / 8; ++vec)
            found |= clean_vector<false>(ring + v_slot * G::kSlot + vec / 8 * kBlock + key * 128 + ((vec ^ key) & 7) * 16);
          if (found) sh.not_finite[odd] = 1;
        }
      }
      fence_to_tensor_cores();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.s_free[buf]);
        mbar_arrive(&sh.p_full[pb]);
      }
    }

    // ---- results: lane d has element d of all rows
    const uint32_t last = u - 1;
    wait(&sh.p_done[last % G::kPBuffers], last / G::kPBuffers & 1);
    tc_fence_after_sync();
    if (several) meet();
    if (tid == 0) sh.not_finite[odd ^ 1] = 0;
    const bool whole = x.c0 == x.c1;
    constexpr int kLine = part_line(DP);
    auto give = [&](int r, int token, int head, float z, float l) {
      if (whole) {
        uint16_t* to = p.out + ((long long)(x.first + token) * p.q_heads + x.h * p.group + head) * c.head_dim;
        const __half h = __float2half_rn(x.base_high + token <= 0 ? 0.f : __fdividef(z, l));
        if (key < c.head_dim) to[key] = *reinterpret_cast<const uint16_t*>(&h);
      } else {
        float* to = part_of(p, x, blockIdx.x, N, DP) + r * kLine;
        if (key < DP) to[key] = z;
        if (key == 0) *reinterpret_cast<float2*>(to + DP) = make_float2(sh.largest[r], l);
      }
    };
    int token = (x.row0 + mine) / p.group, head = x.row0 + mine - token * p.group;
    if (several && *(volatile int*)&sh.not_finite[odd]) {  // (one column at a time, with what was left out)
#pragma unroll 1
      for (int r = mine; r < min(rows, mine + kMine); ++r) {
        float z, l;
        load_column(lanes + 2 * N + r, z);
        load_column(lanes + 3 * N + r, l);
        tc_wait_ld();
        give(r, token, head, z + not_finite_sum<false>(p, x, sees, kTile, r, key), l);
        if (++head == p.group) {
          head = 0;
          ++token;
        }
      }
    } else {
#pragma unroll 1
      for (int c0 = mine; c0 < min(rows, mine + kMine); c0 += kChunk) {
        float y[kChunk], l[kChunk];
        load_columns(lanes + 2 * N + c0, y);
        load_columns(lanes + 3 * N + c0, l);
        tc_wait_ld();
#pragma unroll
        for (int r = 0; r < kChunk; ++r) {
          if (c0 + r < rows) give(c0 + r, token, head, y[r], l[r]);
          if (++head == p.group) {
            head = 0;
            ++token;
          }
        }
      }
    }
    tc_fence_before_sync();
    auto write_out = [&](int r, int d, float4 z, float li) { write_four(p, x, r, d, z, li); };
    if (!whole) join_parts<N, DP, kSoftmaxThreads, 2>(p, x, tid, &sh.arrived, sh.ml, meet, write_out);
    meet();  // (bases and notes are free again)
    if (lane == 0) mbar_arrive(&sh.closed[open]);
    if (++open == G::kOpen) {
      open = 0;
      open_phase ^= 1;
    }
  }
}

template <int DP, int N>
__global__ void __launch_bounds__(kThreads, 1) attention_tc_kernel(const AttentionParams p) {
  using G = TcGeometry<DP, N>;
  extern __shared__ uint8_t smem[];
  __shared__ TcShared<G> sh;
  const uint32_t ring = (smem_u32(smem) + 1023u) & ~1023u;
  const uint32_t q_slots = ring + G::kSlots * G::kSlot, weights = q_slots + G::kOpen * G::kQBytes, ones = weights + G::kPBuffers * G::kPBytes;
  const int warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < G::kSlots; ++i) {
      mbar_init(&sh.full[i], 32 * kProducers);
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
      mbar_init(&sh.p_done[i], 2);
    }
    sh.abort = 0;
    sh.not_finite[0] = sh.not_finite[1] = 0;
  }
  if (threadIdx.x < G::kOnes / 16) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ones + threadIdx.x * 16), "r"(0x3c003c00u) : "memory");
    fence_to_tensor_cores();
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
  if (warp < kSoftmaxWarps) {
    soften<G>(p, sh, ring, weights, tmem);
  } else if (warp < kSoftmaxWarps + kProducers) {
    produce<G>(p, sh, warp - kSoftmaxWarps, ring, q_slots);
  } else if (threadIdx.x % 32 == 0) {
    if (warp == kSoftmaxWarps + kProducers)
      multiply<G, kLogits>(p, sh, ring, q_slots, weights, ones, tmem);
    else if (warp == kSoftmaxWarps + kProducers + 1)
      multiply<G, kResults>(p, sh, ring, q_slots, weights, ones, tmem);
    else
      multiply<G, kSums>(p, sh, ring, q_slots, weights, ones, tmem);
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();  // (every role ends, by itself or when a wait ran out)
  if (warp == kThreads / 32 - 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, G::kColumns);
  }
}

template <int DP, int N>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  using G = TcGeometry<DP, N>;
  return launch_ranges<attention_tc_kernel<DP, N>, G::kSmem, kThreads, N, kTile>(p, sm_count, stream);
}
template <int DP>
cudaError_t launch_rows(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  const long long rows = usual_rows(p);
  if (rows <= 16) return launch<DP, 16>(p, sm_count, stream);
  if (rows <= 32) return launch<DP, 32>(p, sm_count, stream);
  if (rows <= 64) return launch<DP, 64>(p, sm_count, stream);
  return launch<DP, 128>(p, sm_count, stream);
}

}  // namespace

cudaError_t launch_attention_tc(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return padded_dim(p.cache.head_dim) == 64 ? launch_rows<64>(p, sm_count, stream) : launch_rows<128>(p, sm_count, stream);
}

}  // namespace marlin_b200
