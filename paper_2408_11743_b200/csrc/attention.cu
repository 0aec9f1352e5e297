// Attention of new tokens over the paged cache, split over the keys and joined in the same launch.
//
// For one key head and the R = (tokens) * (query heads per key head) rows that read it:  s_j = scale q . k_j,
// o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), m the largest s_j.  Sums over different ranges of keys join exactly:
// (m, l, o) of two ranges give m = max(m1, m2), l = l1 e^(m1 - m) + l2 e^(m2 - m), o alike.  So the work is numbered in
// tiles of some keys of (sequence, key head, block of rows), and every CTA takes an equal range of that numbering, whatever
// the lengths are: the lengths are read on the device, so a captured launch stays balanced as sequences grow.
//
// What bounds it: the cache is read once (2 * 2 * head_dim bytes per key and key head), at 8 rows for 4 * 8 * head_dim
// operations of the tensor cores: 8 operations a byte, so the copies have to be kept in flight and little else counts.  One CTA
// per SM: four warps that do nothing but follow the range and issue copies (16 bytes each, addresses by key, so that a page may
// end anywhere) into a ring of stages of all the shared memory there is, and eight warps that multiply what has arrived, one
// 16-key part of a stage each.  (An issue of a copy takes a warp 33 cycles: with one warp that copied, it was what bounded the kernel.)
// The copies run ahead over the ends of segments, so the next sequence's keys are on their way while this one's sums are joined.
// The products are mma.sync.m16n8k16 with the keys (of S^T = K Q^T) and the values (of O^T = V^T P^T) on the 16-wide side and
// the rows on the 8-wide one: a decode step has few rows, and eight of them fill an operand.
//
// Measured, back to back in a graph: 64 sequences of 2000 to 4096 keys, 32 heads of 128 elements, 458 us, 7.0 TB/s; 64 of up to 8191 keys that
// eight query heads share, 160 us, 6.7 TB/s; one of 131009 keys, 88 us, 6.1 TB/s; 16 of 500 to 1531 keys, 47 us, 5.8 TB/s: a call costs some
// 8.4 us beside the time of its bytes, of which 4 pass before the first products (launch, ranges, page numbers, first keys) and 4 in
// CTAs that end before others and in the joining of parts; one of 129 keys takes 5.8.  8-bit caches, 32 of 2000 to 4099 keys, 64 heads
// over 8: 43 us, 4.7 TB/s, where the copies alone take 38.  No unit is full there (issue 36 %, ALU 32 %, tensor 13 %, DRAM 54 %): two warps
// that multiply on each scheduler wait for what they convert and for what that is multiplied with.
#include "attention.cuh"

namespace marlin_b200 {
namespace {

// DP: head_dim rounded up to 64, 128 or 256.  NT: tiles of 8 rows per warp.  TW: warps side by side over the rows.
// F8: e4m3 cache.  A stage of kTile keys is multiplied by kParts * TW warps (a group): stage s by group s % kGroups, always.  (A wait for
// a parity only tells the phase before the current one: two groups must not wait for consecutive fillings of one stage, which
// may be there before an earlier stage is.)
template <int DP_, int NT, int TW, bool F8>
struct Geometry {
  static constexpr int DP = DP_;
  static constexpr int kRows = 8 * NT * TW;
  static constexpr int kTile = DP == 256 ? 32 : 64;
  static constexpr int kParts = kTile / 16;
  static constexpr int kConsumers = 8;               // warps that multiply (DP * NT / 4 sums a thread; twelve for 8 bits gained nothing)
  static constexpr int kGroups = kConsumers / (kParts * TW);
  static constexpr int kTeams = kConsumers / TW;     // warps that have the same rows
  static constexpr int kProducers = 4;
  static constexpr int kThreads = (kConsumers + kProducers) * 32;
  // The warps that copy hand registers to those that multiply, where these need more than the launch gives.
  static constexpr int kLaunchRegs = 168, kProducerRegs = 88, kConsumerRegs = 208;
  static_assert(kConsumers * kConsumerRegs + 4 * kProducerRegs <= (kConsumers + 4) * kLaunchRegs, "registers");
  static constexpr int kRowBytes = DP * (F8 ? 1 : 2);
  static constexpr int kVectors = kRowBytes / 16;    // 16-byte vectors of a key
  static constexpr int kHalf = kTile * kRowBytes;    // the keys (or the values) of a tile
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kLead = NT == 1 ? (F8 ? 3 : 2) : 4;  // what an item costs beside its tiles, in tiles
  static constexpr int kQVectors = DP / 8;
  static constexpr int kQBytes = kRows * DP * 2;
  static constexpr int kOpen = kQBytes <= 4096 ? 4 : 2;  // segments that can be open at a time
  static constexpr bool kQInRegisters = NT * DP <= 256;
  // the warps' sums meet in shared memory, a range of elements at a time: kRounds of them
  static constexpr int kSums = kTeams * kRows * DP * 4;
  static constexpr int kRounds = kSums <= 65536 ? 1 : kSums <= 131072 ? 2 : 4;
  static constexpr int kColumns = DP / kRounds;
  static constexpr int kJoin = kTeams * kRows * kColumns * 4;
  static constexpr int kRoom = 223 * 1024 - kOpen * kQBytes - kJoin;
  static constexpr int kStages = kRoom / kStage > 16 ? 16 : kRoom / kStage;
  static constexpr int kSmem = kOpen * kQBytes + kJoin + kStages * kStage;
  static_assert(kConsumers % (kParts * TW) == 0 && kStages >= 2 && kStages >= kGroups && DP % (16 * kRounds) == 0, "ring");
};

__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t saddr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(saddr));
}
// the transpose of an 8 x 8 matrix of 16-bit elements held as the operands hold it
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// byte of a 16-byte vector of a row in half a stage: vectors are permuted within 128-byte lines, so that eight rows of one
// vector lie in eight different groups of banks
template <int VECTORS>
__device__ __forceinline__ uint32_t place(int row, int vec) {
  const int v = VECTORS >= 8 ? vec ^ (row & 7) : vec ^ ((row >> 1) & 3);
  return (uint32_t)(row * VECTORS + v) * 16;
}
// the same `vec` vectors further on, `vec` even, from an address in a line-aligned stage: one instruction and an offset
template <int VECTORS>
__device__ __forceinline__ uint32_t further(uint32_t address, int vec) {
  constexpr int kLine = VECTORS >= 8 ? 8 : 4;
  return (address ^ (uint32_t)(vec % kLine * 16)) + vec / kLine * (kLine * 16);
}

// Barriers and notes in shared memory.  Every wait for one is bounded (mbar_wait): when one runs out, `abort` is set, all others return at
// once, and the host finds MARLIN_ERR_DEVICE_TIMEOUT.  The warps that multiply agree on that where a segment begins, so that
// they always meet at the same hardware barriers; what they compute of a segment whose copies did not come is thrown away with
// the call.
template <class G>
struct Shared {
  uint64_t full[G::kStages], empty[G::kStages];  // a stage has arrived; has been multiplied
  uint64_t opened[G::kOpen], closed[G::kOpen];   // a segment and its Q are there; nobody needs them any more
  Segment segments[G::kOpen];
  float2 ml[G::kTeams * G::kRows];               // base and sum of weights of the warps' rows
  int abort;
  int arrived;
  int not_finite[2];  // values were left out of the products of this segment (of an even, an odd number)
};

// false: this wait, or one of another warp, ran out (the same answer for the whole warp)
template <class G>
__device__ __forceinline__ bool arrived_at(Shared<G>& sh, uint64_t* bar, uint32_t parity, int* status) {
  mbar_wait(bar, parity, &sh.abort, status);
  return !__any_sync(~0u, *(volatile int*)&sh.abort);
}

// ---- the warps that copy: each follows the range, and brings one part of every tile ------------------------------------------------------------
template <class G, bool F8>
__device__ __forceinline__ void produce(const AttentionParams& p, Shared<G>& sh, int producer, uint32_t q_slots, uint32_t ring) {
  constexpr int kTile = G::kTile;
  const KvCacheView& c = p.cache;
  const int lane = threadIdx.x & 31;

  Range<G::kRows, kTile, G::kLead> range;
  range.begin(p);

  constexpr int kPer = G::kVectors < 32 ? 32 / G::kVectors : 1;  // keys per pass of the warp
  constexpr int kElement = F8 ? 1 : 2;
  const int my_row = lane / G::kVectors, my_vec = lane % G::kVectors;
  const bool my_part = my_vec * (16 / kElement) < c.head_dim;
  const bool big_pages = c.page_shift >= 4;  // the sixteen keys of a part lie in one page
  // the part of this warp; where there are fewer parts than warps, keys and values apart
  const int part = producer % G::kParts;
  const bool with_keys = G::kParts == G::kProducers || producer < G::kParts, with_values = G::kParts == G::kProducers || !with_keys;
  int stage = 0;
  uint32_t stage_phase = 1, segment = 0, slot_phase = 1;
  int slot = 0;
#pragma unroll 1
  for (;; ++segment) {
    const Segment x = range.next(p);
    // the page numbers of its first tiles are asked for before anything else: the first copies wait for them
    const Visible v = visible(p, x);
    const int* const table = c.table + x.b * c.table_stride;
    const int key_first = x.tile * kTile + part * 16, key_end = (x.tile + x.nt) * kTile;
    const int low = max(v.low_min, x.tile * kTile), high = min(v.high_max, key_end);
    // pages of this part in 32 tiles, a lane each, and in the next 32; or, where pages are smaller than a part, of the keys of
    // one tile and of the next one.  INT_MIN where no key is asked for
    auto page_of = [&](int i) {
      const int key = key_first + (big_pages ? i + lane : i) * kTile + (big_pages ? 0 : lane & 15);
      return x.nt > 0 && key < high && key + (big_pages ? 16 : 1) > low ? load(table + (key >> c.page_shift)) : INT_MIN;
    };
    const int batch = big_pages ? 32 : 1;
    const long long head_bytes = (x.h * c.s_head + my_row * c.s_token) * kElement + my_vec * 16;
    int pages = page_of(0), pages_next = page_of(batch), in_batch = 0;
    if (!arrived_at(sh, &sh.closed[slot], slot_phase, p.status)) break;
    if (lane == 0 && producer == 0) sh.segments[slot] = x;
    if (x.nt > 0) {  // Q; rows and elements that are not there are zeros
      const uint32_t q_to = q_slots + slot * G::kQBytes;
#pragma unroll 1
      for (int i = producer * 32 + lane; i < G::kRows * G::kQVectors; i += 32 * G::kProducers) {
        const int r = i / G::kQVectors, vec = i % G::kQVectors;
        const int token = token_of(p, x, r), head = x.h * p.group + x.row0 + r - token * p.group;
        const bool there = r < x.rows && vec * 8 < c.head_dim;
        const uint16_t* src = p.q + (there ? (long long)(x.first + token) * p.q_stride + head * c.head_dim + vec * 8 : 0);
        copy16(q_to + place<G::kQVectors>(r, vec), src, there);
      }
    }
    copies_arrive(&sh.opened[slot]);
    if (lane == 0 && producer == 0) mbar_arrive(&sh.opened[slot]);
    if (++slot == G::kOpen) {
      slot = 0;
      slot_phase ^= 1;
    }
    if (x.nt == 0) break;

#pragma unroll 1
    for (int i = 0; i < x.nt; ++i, ++in_batch) {
      if (in_batch == batch) {
        in_batch = 0;
        pages = pages_next;
        pages_next = page_of(i + batch);
      }
      if (!arrived_at(sh, &sh.empty[stage], stage_phase, p.status)) break;
      const uint32_t to = ring + stage * G::kStage + part * 16 * G::kRowBytes;
      const int key0 = key_first + i * kTile;
      const int page = __shfl_sync(~0u, pages, in_batch);
      if (big_pages && key0 >= low && key0 + 16 <= high && (unsigned)page < (unsigned)c.pages) {
        // sixteen keys of one page: their places are s_token apart
        const long long first = (page * c.s_page + (key0 & ((1 << c.page_shift) - 1)) * c.s_token) * kElement + head_bytes;
        const uint8_t* ks = static_cast<const uint8_t*>(c.k) + (my_part ? first : 0);
        const uint8_t* vs = static_cast<const uint8_t*>(c.v) + (my_part ? first : 0);
        const long long pass = my_part ? kPer * c.s_token * kElement : 0;
#pragma unroll
        for (int r = 0; r < 16; r += kPer) {
          const uint32_t dst = to + place<G::kVectors>(r + my_row, my_vec);
          if (with_keys) copy16(dst, ks, my_part);
          if (with_values) copy16(dst + G::kHalf, vs, my_part);
          ks += pass;
          vs += pass;
        }
      } else {
#pragma unroll 1
        for (int r = 0; r < 16; r += kPer) {
          const int key = key0 + r + my_row;
          const int mine = __shfl_sync(~0u, pages, big_pages ? in_batch : r + my_row);
          const bool asked = key >= low && key < high;
          const long long from = asked ? cache_offset(c, mine, x.h, key, p.status) : -1;
          const bool there = from >= 0 && my_part;
          const long long bytes = there ? from * kElement + my_vec * 16 : 0;
          const uint32_t dst = to + place<G::kVectors>(r + my_row, my_vec);
          if (with_keys) copy16(dst, static_cast<const uint8_t*>(c.k) + bytes, there);
          if (with_values) copy16(dst + G::kHalf, static_cast<const uint8_t*>(c.v) + bytes, there);
        }
      }
      if (!withheld(p, producer == 0 && stage == 0)) copies_arrive(&sh.full[stage]);
      if (++stage == G::kStages) {
        stage = 0;
        stage_phase ^= 1;
      }
    }
  }
  copies_wait_all();
}

// ---- the warps that multiply ----------------------------------------------------------------------
template <class G, int NT, int TW, bool F8>
__device__ __forceinline__ void consume(const AttentionParams& p, Shared<G>& sh, uint32_t q_slots, float* join, uint32_t ring) {
  constexpr int DP = G::DP, kTile = G::kTile;
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int wm = warp % TW, team = warp / TW, part = team % G::kParts, group = team / G::kParts;
  const int g = lane >> 2, t4 = lane & 3;
  constexpr int kMine = G::kConsumers * 32;
  // where this lane reads keys and values: the 16 keys of its part, vectors 0 and 1
  const uint32_t k_lane = place<G::kVectors>(part * 16 + (lane & 15), lane >> 4);
  const uint32_t v_lane = F8 ? k_lane : place<G::kVectors>(part * 16 + (lane & 7) + (lane >> 4) * 8, (lane >> 3) & 1);

  auto wait = [&](uint64_t* bar, uint32_t parity) { mbar_wait(bar, parity, &sh.abort, p.status); };
  auto meet = [&] {  // all warps that multiply
    named_bar_sync(1, kMine);
    return true;
  };

  // the next tile of this group, in the numbering of all tiles of the CTA (tile t has stage t % kStages), its stage and phase
  uint32_t next = group, done = 0;
  int stage = group;
  uint32_t stage_phase = 0, slot_phase = 0;
  int slot = 0, odd = 0;
#pragma unroll 1
  for (;; odd ^= 1) {
    wait(&sh.opened[slot], slot_phase);
    if (any_of(1, kMine, *(volatile int*)&sh.abort)) return;  // (what there was of the segment before was read as well)
    const Segment& x = sh.segments[slot];
    const int nt = x.nt, tile = x.tile, rows = x.rows;
    if (nt == 0) return;
    const Visible sees = visible(p, x);
    const int low_min = sees.low_min, low_max = sees.low_max, high_min = sees.high_min, high_max = sees.high_max;
    const bool several = x.n > 1;

    // positions below which the rows of this thread see (rows that are not there: as the last one)
    int high[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        high[j][i] = several ? x.base_high + (x.row0 + min(rows - 1, wm * 8 * NT + j * 8 + t4 * 2 + i)) / p.group : high_min;
    const float factor = p.scale_log2 * (F8 && c.k_scale ? load(c.k_scale + x.h) : 1.f);

    // operands of Q: rows on the 8-wide side; of 16 elements a thread has 2 t, 2 t + 1, 2 t + 8, 2 t + 9, or, to match the
    // bytes of an 8-bit key, 4 t .. 4 t + 3
    const uint32_t q_base = q_slots + slot * G::kQBytes;
    const int q_row = wm * 8 * NT;
    uint32_t q[G::kQInRegisters ? DP / 16 : 1][NT][2];
    auto load_q = [&](int ks, uint32_t (&x)[NT][2]) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (F8) {
          const uint2 y = lds64(q_base + place<G::kQVectors>(q_row + j * 8 + g, 2 * ks + (t4 >> 1)) + (t4 & 1) * 8);
          x[j][0] = y.x;
          x[j][1] = y.y;
        } else if (NT % 2 == 0) {
          if (j % 2 == 0) {
            uint32_t y[4];
            ldmatrix_x4(q_base + place<G::kQVectors>(q_row + j * 8 + (lane & 7) + (lane >> 4) * 8, 2 * ks + ((lane >> 3) & 1)), y);
            x[j][0] = y[0];
            x[j][1] = y[1];
            x[NT % 2 == 0 ? j + 1 : 0][0] = y[2];
            x[NT % 2 == 0 ? j + 1 : 0][1] = y[3];
          }
        } else {
          x[j][0] = lds32(q_base + place<G::kQVectors>(q_row + j * 8 + g, 2 * ks) + t4 * 4);
          x[j][1] = lds32(q_base + place<G::kQVectors>(q_row + j * 8 + g, 2 * ks + 1) + t4 * 4);
        }
      }
    };

    float m[NT][2], l[NT][2];
    float o[DP / 16][NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      m[j][0] = m[j][1] = kNone;
      l[j][0] = l[j][1] = 0.f;
#pragma unroll
      for (int v = 0; v < DP / 16; ++v) o[v][j][0] = o[v][j][1] = o[v][j][2] = o[v][j][3] = 0.f;
    }
    if (G::kQInRegisters) {
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) load_q(ks, q[G::kQInRegisters ? ks : 0]);
    }
    bool open = true;  // some row has not seen a key yet

#pragma unroll 1
    while (next < done + nt) {
      wait(&sh.full[stage], stage_phase);
      const uint32_t keys = ring + stage * G::kStage, values = keys + G::kHalf;
      // S^T = K Q^T: a thread has keys g, g + 8 of 16 and rows 2 t, 2 t + 1 of 8.  (One tile of rows alone would be a chain of
      // dependent products: it is summed in two.)
      constexpr int kChains = NT == 1 ? 2 : 1;
      float y[NT][kChains][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < kChains; ++i) y[j][i][0] = y[j][i][1] = y[j][i][2] = y[j][i][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ks += F8 ? 2 : 1) {
        uint32_t qs[F8 ? 2 : 1][NT][2];
        if (!G::kQInRegisters) {
          load_q(ks, qs[0]);
          if (F8) load_q(ks + 1, qs[F8 ? 1 : 0]);
        }
        uint32_t r[4];
        ldmatrix_x4(further<G::kVectors>(keys + k_lane, F8 ? ks : 2 * ks), r);
#pragma unroll
        for (int i = 0; i < (F8 ? 2 : 1); ++i) {
          uint32_t a[4];
          if (F8) {  // r[2 i]: keys 0 - 7, r[2 i + 1]: keys 8 - 15 of 16 elements
            a[0] = e4m3x2_to_f16x2(r[F8 ? 2 * i : 0]);
            a[1] = e4m3x2_to_f16x2(r[F8 ? 2 * i + 1 : 0]);
            a[2] = e4m3x2_to_f16x2(r[F8 ? 2 * i : 0] >> 16);
            a[3] = e4m3x2_to_f16x2(r[F8 ? 2 * i + 1 : 0] >> 16);
          } else {
            a[0] = r[0]; a[1] = r[1]; a[2] = r[2]; a[3] = r[3];
          }
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const uint32_t(&z)[2] = G::kQInRegisters ? q[G::kQInRegisters ? ks + i : 0][j] : qs[F8 ? i : 0][j];
            mma_16816(y[j][(F8 ? i : ks) % kChains], a, z[0], z[1]);
          }
        }
      }

      // logits in units of log2, relative to the base; -inf where a row does not see the key
      const int pos0 = (tile + (int)(next - done)) * kTile + part * 16;
      const bool all = pos0 >= low_max && pos0 + 16 <= high_min;  // (the same for the warp)
      bool over = open;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float& x = y[j][0][e];
          if (kChains == 2) x += y[j][kChains - 1][e];
          x = fmaf(x, factor, m[j][e & 1] == kNone ? 0.f : -m[j][e & 1]);
          over |= x > kSlack;
        }
      if (!all) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int pos = pos0 + g + (e >> 1) * 8;
            const bool seen = pos < high[j][e & 1] && (p.window == 0 || pos >= high[j][e & 1] - p.window);
            if (!seen) y[j][0][e] = kNone;
          }
      }
      if (__any_sync(~0u, over)) {  // move the bases
        bool none = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(y[j][0][i], y[j][0][i + 2]);
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
            const float old = m[j][i] == kNone ? 0.f : m[j][i];
            const float now = fmaxf(m[j][i], top + old - kBelow);
            const float base = now == kNone ? 0.f : now;
            const float alpha = exp2_fast(m[j][i] - base), shift = old - base;
            m[j][i] = now;
            none |= now == kNone;
            l[j][i] *= alpha;
            y[j][0][i] += shift;
            y[j][0][i + 2] += shift;
#pragma unroll
            for (int v = 0; v < DP / 16; ++v) {
              o[v][j][i] *= alpha;
              o[v][j][i + 2] *= alpha;
            }
          }
        open = __any_sync(~0u, none);
      }

      // weights, rounded to fp16 for the product (kBelow in attention.cuh), and turned round: keys on the side that is summed over
      uint32_t w[NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float (&x)[4] = y[j][0];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = exp2_fast(x[e]);
          l[j][e & 1] += x[e];
        }
        w[j][0] = transpose8x8(half2_bits(x[0], x[1]));
        w[j][1] = transpose8x8(half2_bits(x[2], x[3]));
      }

      if (several && !all) {  // values of keys that not every row sees (warps that share them all do the same)
        bool found = false;
#pragma unroll 1
        for (int i = lane; i < 16 * G::kVectors; i += 32) {
          const int row = part * 16 + i / G::kVectors, pos = pos0 + i / G::kVectors;
          if ((pos >= high_min && pos < high_max) || (pos >= low_min && pos < low_max))
            found |= clean_vector<F8>(values + place<G::kVectors>(row, i % G::kVectors));
        }
        if (found) sh.not_finite[odd] = 1;
        __syncwarp();
      }

      // O^T += V^T P^T: a thread has elements g, g + 8 (8-bit: 2 g, 2 g + 1) of 16 and rows 2 t, 2 t + 1 of 8
#pragma unroll
      for (int v = 0; v < DP / 16; v += F8 ? 2 : 1) {
        uint32_t r[4];
        // 8-bit: r[2 i], r[2 i + 1] of vector v + i: bytes (key 2 t: elements 2 g, 2 g + 1), (key 2 t + 1: the same); keys + 8
        ldmatrix_x4_trans(further<G::kVectors>(values + v_lane, F8 ? v : 2 * v), r);
#pragma unroll
        for (int i = 0; i < (F8 ? 2 : 1); ++i) {
          uint32_t a[4];
          if (F8) {
            const uint32_t lo = __byte_perm(r[F8 ? 2 * i : 0], 0, 0x3120), hi = __byte_perm(r[F8 ? 2 * i + 1 : 0], 0, 0x3120);
            a[0] = e4m3x2_to_f16x2(lo);
            a[1] = e4m3x2_to_f16x2(lo >> 16);
            a[2] = e4m3x2_to_f16x2(hi);
            a[3] = e4m3x2_to_f16x2(hi >> 16);
          } else {
            a[0] = r[0]; a[1] = r[1]; a[2] = r[2]; a[3] = r[3];
          }
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_16816(o[F8 ? v + i : v][j], a, w[j][0], w[j][1]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.empty[stage]);
      if (stage + G::kGroups < G::kStages) {
        stage += G::kGroups;
        next += G::kGroups;
      } else {  // round the ring, to this group's first stage again
        next += G::kStages - stage + group;
        stage = group;
        stage_phase ^= 1;
      }
    }
    done += nt;

    // ---- the warps' sums meet: [team][row][kColumns elements], a round for each range of elements; groups of eight elements are
    // permuted so that rows 2 t lie in different banks
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 4);
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 8);
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 16);
      }
    const bool whole = x.c0 == x.c1;
    constexpr int kLine = part_line(DP);
    auto write_out = [&](int r, int d, float4 z, float li) { write_four(p, x, r, d, z, li); };
    auto bank = [](int r, int d) { return G::kColumns >= 32 ? d ^ ((r >> 1 & 3) * 8) : d; };
#pragma unroll
    for (int round = 0; round < G::kRounds; ++round) {
      if (round > 0) meet();  // (what was there was read)
      if (tid == 0 && round == 0) sh.not_finite[odd ^ 1] = 0;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = wm * 8 * NT + j * 8 + t4 * 2 + i;
          float* dst = join + (team * G::kRows + r) * G::kColumns;
          if (r < rows) {
            if (g == 0 && round == 0) sh.ml[team * G::kRows + r] = make_float2(m[j][i], l[j][i]);
#pragma unroll
            for (int v = 0; v < G::kColumns / 16; ++v) {
              dst[bank(r, v * 16 + (F8 ? 2 * g : g))] = o[round * (G::kColumns / 16) + v][j][i];
              dst[bank(r, v * 16 + (F8 ? 2 * g + 1 : g + 8))] = o[round * (G::kColumns / 16) + v][j][i + 2];
            }
          }
        }
      meet();
      const bool odd_values = several && sh.not_finite[odd];
#pragma unroll 1
      for (int i = tid; i < rows * (G::kColumns / 4); i += kMine) {
        const int r = i / (G::kColumns / 4), at_d = (i % (G::kColumns / 4)) * 4, d = round * G::kColumns + at_d;
        if (d >= c.head_dim) continue;
        // (all of it is asked for at once: one latency, not one for each team)
        float2 sums[G::kTeams];
        float4 u[G::kTeams];
        float mi = kNone;
#pragma unroll
        for (int t = 0; t < G::kTeams; ++t) {
          sums[t] = sh.ml[t * G::kRows + r];
          u[t] = *reinterpret_cast<const float4*>(join + (t * G::kRows + r) * G::kColumns + bank(r, at_d));
          mi = fmaxf(mi, sums[t].x);
        }
        const float base = mi == kNone ? 0.f : mi;
        float li = 0.f;
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int t = 0; t < G::kTeams; ++t) {
          const float f = exp2_fast(sums[t].x - base);
          li += sums[t].y * f;
          z.x += u[t].x * f; z.y += u[t].y * f; z.z += u[t].z * f; z.w += u[t].w * f;
        }
        if (odd_values) {
#pragma unroll 1
          for (int e = 0; e < 4; ++e) {
            const float v = not_finite_sum<F8>(p, x, sees, kTile, r, d + e);
            z.x += e == 0 ? v : 0.f; z.y += e == 1 ? v : 0.f; z.z += e == 2 ? v : 0.f; z.w += e == 3 ? v : 0.f;
          }
        }
        if (whole) {
          write_out(r, d, z, li);
        } else {
          float* to = part_of(p, x, blockIdx.x, G::kRows, DP);
          *reinterpret_cast<float4*>(to + r * kLine + d) = z;
          if (d == 0) *reinterpret_cast<float2*>(to + r * kLine + DP) = make_float2(mi, li);
        }
      }
    }
    if (!whole) join_parts<G::kRows, DP, kMine, 1, 4>(p, x, tid, &sh.arrived, sh.ml, meet, write_out);
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.closed[slot]);
    if (++slot == G::kOpen) {
      slot = 0;
      slot_phase ^= 1;
    }
  }
}

template <int DP, int NT, int TW, bool F8>
__global__ void __launch_bounds__(Geometry<DP, NT, TW, F8>::kThreads, 1) attention_kernel(const AttentionParams p) {
  using G = Geometry<DP, NT, TW, F8>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Shared<G> sh;
  uint8_t* const join = smem + G::kOpen * G::kQBytes;
  const uint32_t ring = smem_u32(join) + G::kJoin;
  if (threadIdx.x == 0) {
    for (int i = 0; i < G::kStages; ++i) {
      mbar_init(&sh.full[i], 32 * G::kProducers);
      mbar_init(&sh.empty[i], G::kParts * TW);
    }
    for (int i = 0; i < G::kOpen; ++i) {
      mbar_init(&sh.opened[i], 32 * G::kProducers + 1);  // the copies of all lanes, and the note itself
      mbar_init(&sh.closed[i], G::kConsumers);
    }
    sh.abort = 0;
    sh.not_finite[0] = sh.not_finite[1] = 0;
  }
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  prefetch_table(p, G::kThreads);
  if (threadIdx.x >= G::kConsumers * 32) {
    setmaxnreg_dec<G::kProducerRegs>();
    produce<G, F8>(p, sh, (int)threadIdx.x / 32 - G::kConsumers, smem_u32(smem), ring);
  } else {
    setmaxnreg_inc<G::kConsumerRegs>();
    consume<G, NT, TW, F8>(p, sh, smem_u32(smem), reinterpret_cast<float*>(join), ring);
  }
}

template <int DP, int NT, int TW, bool F8>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  using G = Geometry<DP, NT, TW, F8>;
  // the warps share out the registers of the launch: with fewer of them the increase would wait for ever
  return launch_ranges<attention_kernel<DP, NT, TW, F8>, G::kSmem, G::kThreads, G::kRows, G::kTile>(
      p, sm_count, stream, G::kLaunchRegs);
}
template <int DP, bool F8>
cudaError_t launch_rows(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  // (Both sides of each choice at one size: 16 sequences of 1000 to 4099 keys, eight heads of keys.  With sequences of a few dozen keys an
  // item of one tile costs far more on tcgen05 than its bytes, 57 us for 121 of them with 8 or 16 rows against a floor of 3, and
  // nothing here looks at how long they can be.)
  // Up to eight rows: a warp has them all beside the keys.  More of them, over fp16: the tensor cores' fifth generation (16 rows of 128
  // elements: 39.3 us there, 39.9 here; 32 rows: 43 and 47; 48 rows: 47 and 53).  More of them over 8 bits: here, where
  // every warp converts what it multiplies (16 rows: 31 us here, 46 there; 32 rows: 45 and 49), until the products are what takes
  // the time, with more than 32 rows of 128 elements (48 rows: 72 and 55; of 64 elements: 44 and 46).  A warp holds 8 NT rows of
  // sums (DP * NT / 4 registers a thread); more rows than that share keys and values between the warps of a team.
  const long long rows = usual_rows(p);
  if (rows <= 8) return launch<DP, 1, 1, F8>(p, sm_count, stream);
  if (DP < 256 && (!F8 || (DP == 128 && rows > 32))) return launch_attention_tc(p, sm_count, stream);
  if constexpr (F8 || DP == 256) {
    constexpr int kWide = DP == 64 ? 4 : 2, kShared = DP == 64 ? 1 : 2;
    if (rows <= 16) return launch<DP, 2, 1, F8>(p, sm_count, stream);
    if (rows <= 32) return launch<DP, kWide, kShared, F8>(p, sm_count, stream);
    if constexpr (DP != 128) return launch<DP, kWide, 2 * kShared, F8>(p, sm_count, stream);
  }
  return cudaErrorInvalidValue;  // (not reached)
}
template <int DP>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return p.cache.eight_bit ? launch_rows<DP, true>(p, sm_count, stream) : launch_rows<DP, false>(p, sm_count, stream);
}

}  // namespace

// Two parts per CTA that a grid can have, of its rows.
size_t attention_slot_bytes(int head_dim) {
  const int dp = padded_dim(head_dim);
  return (size_t)2 * kMostCtas * 64 * part_line(dp) * sizeof(float);
}

cudaError_t launch_attention(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  switch (padded_dim(p.cache.head_dim)) {
    case 64: return launch_format<64>(p, sm_count, stream);
    case 128: return launch_format<128>(p, sm_count, stream);
    default: return launch_format<256>(p, sm_count, stream);
  }
}

}  // namespace marlin_b200
