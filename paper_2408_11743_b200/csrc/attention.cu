// Attention of new tokens over the paged cache, split over the keys and joined in the same launch.
//
// For one key head and the R = (tokens) * (query heads per key head) rows that read it:  s_j = scale q . k_j,
// o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), m the largest s_j.  Sums over different ranges of keys join exactly:
// (m, l, o) of two ranges give m = max(m1, m2), l = l1 e^(m1 - m) + l2 e^(m2 - m), o alike.  So the work is numbered in
// tiles of 64 keys of (sequence, key head, block of rows), and every CTA takes an equal range of that numbering, whatever
// the lengths are: the lengths are read on the device, so a captured launch stays balanced as sequences grow.
//
// What bounds it: the cache is read once (2 * 2 * head_dim bytes per key and key head), at 8 rows for 4 * 8 * head_dim
// operations of the tensor cores: 8 operations a byte, so the copies have to be kept in flight and nothing else counts.
// Every warp streams keys and values of its own share of a tile through a ring in shared memory (16-byte asynchronous
// copies, addresses by key, so that a page may end anywhere), and multiplies with mma.sync.m16n8k16 with the keys (of S^T = K Q^T)
// and the values (of O^T = V^T P^T) on the 16-wide side and the rows on the 8-wide one: a decode step has few rows, and
// eight of them fill an operand.
#include <limits.h>

#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kTile = 64;       // keys of a tile
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kLeastTiles = 2;  // tiles that a CTA takes at least, where there are fewer tiles than CTAs would like
constexpr uint32_t kMostUnits = 1u << 30;
constexpr float kNone = -INFINITY;
// A row's sums are kept relative to 2^base, base its largest logit (in units of log2) when the base was last moved.  It moves only
// when a logit exceeds it by more than this, so that most tiles neither look for a maximum across lanes nor rescale:
// weights are then at most 2^8, far from the end of fp16, and their rounding is relative.
constexpr float kSlack = 8.f;

constexpr int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
constexpr int blocks_per_sm(int dp, int nt, bool f8) { return dp == 256 ? 1 : nt == 1 ? (f8 ? 4 : 3) : 2; }

// DP: head_dim rounded up to 64, 128 or 256.  NT: tiles of 8 rows per warp.  TW: warps that share keys and values and have
// rows of their own (a team); the kWarps / TW teams share out the keys of a tile.  F8: e4m3 cache.
template <int DP_, int NT, int TW, bool F8>
struct Geometry {
  static constexpr int DP = DP_;
  static constexpr int kRows = 8 * NT * TW;
  static constexpr int kTeams = kWarps / TW;
  static constexpr int kKeys = 16 * TW;              // keys of a tile that a team multiplies
  static constexpr int kRowBytes = DP * (F8 ? 1 : 2);
  static constexpr int kVectors = kRowBytes / 16;    // 16-byte vectors of a key
  static constexpr int kHalf = kTile * kRowBytes;    // the keys (or the values) of a tile
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kBlocks = blocks_per_sm(DP, NT, F8);  // CTAs per SM
  static constexpr int kQVectors = DP / 8;
  static constexpr int kQBytes = kRows * DP * 2;
  static constexpr int kJoinStride = DP + 4;         // floats between rows of the teams' sums: rows 2 t fall on other banks
  static constexpr int kJoin = kTeams * kRows * (kJoinStride + 2) * 4;  // where the teams' sums meet, in the ring
  static constexpr int kRoom = 224 / kBlocks * 1024 - kQBytes;
  static constexpr int kStages = kRoom / kStage > 8 ? 8 : kRoom / kStage;
  static constexpr int kSmem = kQBytes + kStages * kStage;
  static constexpr bool kQInRegisters = NT * DP <= 256;
  static_assert(kStages >= 2 && kStages * kStage >= kJoin, "ring");
};


__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  const int bytes = there ? 16 : 0;  // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
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
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
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

// What a sequence asks for: new tokens [first, first + n) of the call, tiles [tile0, tile0 + tiles) of its len keys, blocks of
// rows per key head.  A sequence with new tokens has a tile at least: it writes the zeros.
struct Sequence {
  int len, n, first, tile0, tiles, blocks;
};
__device__ __forceinline__ Sequence sequence(const AttentionParams& p, int b, int rows) {
  Sequence s;
  s.len = cache_length(p.cache, b, p.status);
  s.first = b;
  s.n = 1;
  if (p.starts) {
    const int from = min(max(__ldg(p.starts + b), 0), p.tokens), to = min(max(__ldg(p.starts + b + 1), from), p.tokens);
    s.first = from;
    s.n = to - from;
  }
  s.tile0 = (p.window ? max(0, s.len - s.n - p.window + 1) : 0) / kTile;
  s.tiles = max(1, (s.len + kTile - 1) / kTile - s.tile0);
  s.blocks = (s.n * p.group + rows - 1) / rows;
  return s;
}

// The ranges of the CTAs: worker w of W begins at unit w * (U / W) + min(w, U % W).  A range that would begin within `snap` tiles of
// the beginning or the end of an item (the tiles of one block of rows) begins there instead: a part of an item costs a
// round trip through the workspace, which is worth a tile or two where a CTA has few.
struct Stripes {
  uint32_t total, workers, size, more, snap;
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * size + min(w, more); }
  __device__ __forceinline__ uint32_t owner(uint32_t x) const {  // whose range, before any move, holds unit x
    const uint32_t wide = more * (size + 1);
    return x < wide ? x / (size + 1) : more + (x - wide) / size;
  }
  // boundary x of the ranges where it lies inside of item [i0, i1)
  __device__ __forceinline__ uint32_t moved(uint32_t x, uint32_t i0, uint32_t i1) const {
    if (x <= i0 || x >= i1) return x;
    if (x - i0 <= snap && x - i0 <= i1 - x) return i0;
    return i1 - x <= snap ? i1 : x;
  }
};

template <int DP, int NT, int TW, bool F8>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(DP, NT, F8)) attention_kernel(const AttentionParams p) {
  using G = Geometry<DP, NT, TW, F8>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t scan[kWarps];
  __shared__ uint32_t found_offset;
  __shared__ int found_sequence;
  __shared__ int arrived;
  __shared__ int not_finite;  // values that were left out of the products of this segment
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = warp / TW, wm = warp % TW;
  const int g = lane >> 2, t4 = lane & 3;
  const uint32_t ring = smem_u32(smem) + G::kQBytes;
  float* const join = reinterpret_cast<float*>(smem + G::kQBytes);

  pdl_launch_dependents();
  pdl_wait_prior_grids();

  // ---- this CTA's range of tiles: thread i counts the tiles of sequences [i * per, (i + 1) * per)
  const int per = (c.sequences + kThreads - 1) / kThreads;
  uint32_t mine = 0;
  for (int b = tid * per; b < min(c.sequences, (tid + 1) * per); ++b) {
    const Sequence s = sequence(p, b, G::kRows);
    const unsigned long long units = (unsigned long long)c.kv_heads * s.blocks * s.tiles + mine;
    mine = (uint32_t)min(units, (unsigned long long)kMostUnits);
  }
  uint32_t before = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t x = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before = min(before + x, kMostUnits);
  }
  if (lane == 31) scan[warp] = before;
  if (tid == 0) not_finite = 0;
  __syncthreads();
  Stripes stripes;
  stripes.total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before = min(before + scan[w], kMostUnits);
    stripes.total = min(stripes.total + scan[w], kMostUnits);
  }
  if (stripes.total == kMostUnits) {  // more tiles than are numbered (2^30: weeks of work): refused
    report_cache(p.status);
    return;
  }
  before -= mine;
  stripes.workers = min(gridDim.x, max(1u, stripes.total / kLeastTiles));
  if (blockIdx.x >= stripes.workers) return;
  stripes.size = stripes.total / stripes.workers;
  stripes.more = stripes.total % stripes.workers;
  stripes.snap = stripes.size < 8 ? 2 : 0;
  uint32_t at = stripes.begin(blockIdx.x);
  const uint32_t end = stripes.begin(blockIdx.x + 1);
  if (at >= end) return;  // (nothing to do at all)
  if (mine > 0 && before <= at && at < before + mine) {
    int b = tid * per;
    uint32_t off = at - before;
    for (;; ++b) {
      const Sequence s = sequence(p, b, G::kRows);
      const uint32_t units = (uint32_t)c.kv_heads * s.blocks * s.tiles;
      if (off < units) break;
      off -= units;
    }
    found_sequence = b;
    found_offset = off;
  }
  __syncthreads();
  int b = found_sequence;
  uint32_t off = found_offset;
  Sequence s = sequence(p, b, G::kRows);
  uint32_t item = off / (uint32_t)s.tiles;     // (key head, block of rows) of the sequence
  uint32_t skip = off - item * (uint32_t)s.tiles;
  {
    const uint32_t i0 = at - skip, to = stripes.moved(at, i0, i0 + s.tiles);
    skip += to - at;
    at = to;
  }

#pragma unroll 1
  for (;;) {
    if (skip == (uint32_t)s.tiles) {  // the next item
      if (at >= end) return;
      skip = 0;
      if (++item == (uint32_t)(c.kv_heads * s.blocks)) {
        item = 0;
        do s = sequence(p, ++b, G::kRows);
        while (s.blocks == 0);
      }
    }
    // ---- one segment: tiles [tile, tile + nt) of (sequence b, key head h, block of rows rb)
    const uint32_t i0 = at - skip, i1 = i0 + s.tiles;
    const uint32_t to = min(stripes.moved(end, i0, i1), i1);
    if (at >= to) return;
    const int nt = (int)(to - at);
    const int h = (int)(item / (uint32_t)s.blocks), rb = (int)item - h * s.blocks;
    const int tile = s.tile0 + (int)skip;
    const int row0 = rb * G::kRows;  // row r is query head h * group + r % group of new token r / group
    const int rows = min(G::kRows, s.n * p.group - row0);
    // row r sees the positions [high - window, high) (all below high without a window), high = base_high + its token; the block
    // as a whole [low_min, high_max), and all of its rows [low_max, high_min)
    const int base_high = s.len - s.n + 1;
    const int token_first = row0 / p.group, token_last = (row0 + rows - 1) / p.group;
    const int high_min = base_high + token_first, high_max = base_high + token_last;
    const int low_min = p.window ? max(0, high_min - p.window) : 0, low_max = p.window ? max(0, high_max - p.window) : 0;

    // ---- copies: every warp brings 16 keys and values of a tile, in most layouts just those that it multiplies
    constexpr int kPer = G::kVectors < 32 ? 32 / G::kVectors : 1;  // keys per pass of the warp
    constexpr int kElement = F8 ? 1 : 2;
    const int my_row = lane / G::kVectors, my_vec = lane % G::kVectors;
    const bool my_part = my_vec * (16 / kElement) < c.head_dim;
    const int* const table = c.table + b * c.table_stride;
    const long long head_bytes = h * c.s_head * kElement + my_row * c.s_token * kElement + my_vec * 16;
    auto page_of = [&](int step) {  // the page of key lane % 16 of the warp's sixteen, INT_MIN where it is not asked for
      const int key = (tile + step) * kTile + warp * 16 + (lane & 15);
      return step < nt && key >= low_min && key < high_max ? __ldg(table + (key >> c.page_shift)) : INT_MIN;
    };
    auto bring = [&](int step, int page, uint32_t stage) {
      if (step < nt) {
        const int key0 = (tile + step) * kTile + warp * 16;
        if (c.page_shift >= 4 && __all_sync(~0u, (unsigned)page < (unsigned)c.pages)) {
          // sixteen keys of one page: their places are s_token apart
          const long long first = (page * c.s_page + (key0 & ((1 << c.page_shift) - 1)) * c.s_token) * kElement + head_bytes;
          const uint8_t* k = static_cast<const uint8_t*>(c.k) + (my_part ? first : 0);
          const uint8_t* v = static_cast<const uint8_t*>(c.v) + (my_part ? first : 0);
          if (c.s_token == DP) {
#pragma unroll
            for (int r = 0; r < 16; r += kPer) {
              const uint32_t dst = stage + place<G::kVectors>(warp * 16 + r + my_row, my_vec);
              copy16(dst, k + r * G::kRowBytes, my_part);
              copy16(dst + G::kHalf, v + r * G::kRowBytes, my_part);
            }
          } else {
            const long long pass = my_part ? kPer * c.s_token * kElement : 0;
#pragma unroll
            for (int r = 0; r < 16; r += kPer) {
              const uint32_t dst = stage + place<G::kVectors>(warp * 16 + r + my_row, my_vec);
              copy16(dst, k, my_part);
              copy16(dst + G::kHalf, v, my_part);
              k += pass;
              v += pass;
            }
          }
        } else {
          const long long off = page == INT_MIN ? -1 : cache_offset(c, page, h, key0 + (lane & 15), p.status);
#pragma unroll 1
          for (int r = 0; r < 16; r += kPer) {
            const long long from = __shfl_sync(~0u, off, r + my_row);
            const bool there = from >= 0 && my_part;
            const long long bytes = there ? from * kElement + my_vec * 16 : 0;
            const uint32_t dst = stage + place<G::kVectors>(warp * 16 + r + my_row, my_vec);
            copy16(dst, static_cast<const uint8_t*>(c.k) + bytes, there);
            copy16(dst + G::kHalf, static_cast<const uint8_t*>(c.v) + bytes, there);
          }
        }
      }
      copies_commit();
    };
    int page = page_of(0);

    // Q goes with the first tile; rows and elements that are not there are zeros
#pragma unroll 1
    for (int i = tid; i < G::kRows * G::kQVectors; i += kThreads) {
      const int r = i / G::kQVectors, vec = i % G::kQVectors;
      const int token = (row0 + r) / p.group, head = h * p.group + (row0 + r) - token * p.group;
      const bool there = r < rows && vec * 8 < c.head_dim;
      const uint16_t* src = p.q + (there ? (long long)(s.first + token) * p.q_stride + head * c.head_dim + vec * 8 : 0);
      copy16(smem_u32(smem) + place<G::kQVectors>(r, vec), src, there);
    }
#pragma unroll 1
    for (int i = 0; i < G::kStages - 1; ++i) {
      const int next = page_of(i + 1);
      bring(i, page, ring + i * G::kStage);
      page = next;
    }

    // positions below which the rows of this thread see (rows that are not there: as the last one)
    int high[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        high[j][i] = s.n == 1 ? base_high : base_high + (row0 + min(rows - 1, wm * 8 * NT + j * 8 + t4 * 2 + i)) / p.group;
    const float factor = p.scale_log2 * (F8 && c.k_scale ? __ldg(c.k_scale + h) : 1.f);

    // operands of Q: rows on the 8-wide side; of 16 elements a thread has 2 t, 2 t + 1, 2 t + 8, 2 t + 9, or, to match the
    // bytes of an 8-bit key, 4 t .. 4 t + 3
    const uint32_t q_base = smem_u32(smem);
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
    bool open = true;  // some row has not seen a key yet
    // stages of this step and of the one that is brought: offsets in the ring
    uint32_t keys = ring, free_stage = ring + (G::kStages - 1) * G::kStage;
    const int key0 = team * G::kKeys;
    // where this lane reads keys and values: 16 keys, vectors 0 and 1
    const uint32_t k_lane = place<G::kVectors>(key0 + (lane & 15), lane >> 4);
    const uint32_t v_lane = F8 ? k_lane : place<G::kVectors>(key0 + (lane & 7) + (lane >> 4) * 8, (lane >> 3) & 1);

#pragma unroll 1
    for (int step = 0; step < nt; ++step) {
      copies_wait<G::kStages - 2>();
      if (step == 0 || TW == kWarps)
        __syncthreads();  // (the first time for Q)
      else if (TW == 1)
        __syncwarp();
      else
        named_bar_sync(1 + team, 32 * TW);
      {
        const int next = page_of(step + G::kStages);
        bring(step + G::kStages - 1, page, free_stage);
        page = next;
      }
      free_stage = keys;
      if (G::kQInRegisters && step == 0) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) load_q(ks, q[G::kQInRegisters ? ks : 0]);
      }
      const uint32_t values = keys + G::kHalf;

      // S^T = K Q^T: a thread has keys g, g + 8 of 16 and rows 2 t, 2 t + 1 of 8.  (One tile alone would be a chain of dependent
      // products: it is summed in two.)
      constexpr int kChains = NT * TW == 1 ? 2 : 1;
      float x[TW][NT][kChains][4];
#pragma unroll
      for (int kk = 0; kk < TW; ++kk)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < kChains; ++i) x[kk][j][i][0] = x[kk][j][i][1] = x[kk][j][i][2] = x[kk][j][i][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ks += F8 ? 2 : 1) {
        uint32_t qs[F8 ? 2 : 1][NT][2];
        if (!G::kQInRegisters) {
          load_q(ks, qs[0]);
          if (F8) load_q(ks + 1, qs[F8 ? 1 : 0]);
        }
#pragma unroll
        for (int kk = 0; kk < TW; ++kk) {
          uint32_t r[4];
          ldmatrix_x4(further<G::kVectors>(keys + k_lane, F8 ? ks : 2 * ks) + kk * 16 * G::kRowBytes, r);
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
              const uint32_t(&y)[2] = G::kQInRegisters ? q[G::kQInRegisters ? ks + i : 0][j] : qs[F8 ? i : 0][j];
              mma_16816(x[kk][j][(F8 ? i : ks) % kChains], a, y[0], y[1]);
            }
          }
        }
      }

      // logits in units of log2, relative to the base; -inf where a row does not see the key
      const int pos0 = (tile + step) * kTile + key0;
      const bool all = pos0 >= low_max && pos0 + G::kKeys <= high_min;  // (the same for the team)
      bool over = open;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float base = m[j][i] == kNone ? 0.f : m[j][i];
#pragma unroll
          for (int kk = 0; kk < TW; ++kk)
#pragma unroll
            for (int e = i; e < 4; e += 2) {
              float& y = x[kk][j][0][e];
              if (kChains == 2) y += x[kk][j][kChains - 1][e];
              y = fmaf(y, factor, -base);
              over |= y > kSlack;
            }
        }
      if (!all) {
#pragma unroll
        for (int kk = 0; kk < TW; ++kk)
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int pos = pos0 + kk * 16 + g + (e >> 1) * 8;
              const bool seen = pos < high[j][e & 1] && (p.window == 0 || pos >= high[j][e & 1] - p.window);
              if (!seen) x[kk][j][0][e] = kNone;
            }
      }
      if (__any_sync(~0u, over)) {  // move the bases
        bool none = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = kNone;
#pragma unroll
            for (int kk = 0; kk < TW; ++kk) top = fmaxf(top, fmaxf(x[kk][j][0][i], x[kk][j][0][i + 2]));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
            const float old = m[j][i] == kNone ? 0.f : m[j][i];
            const float now = fmaxf(m[j][i], top + old);
            const float base = now == kNone ? 0.f : now;
            const float alpha = exp2_fast(m[j][i] - base), shift = old - base;
            m[j][i] = now;
            none |= now == kNone;
            l[j][i] *= alpha;
#pragma unroll
            for (int kk = 0; kk < TW; ++kk) {
              x[kk][j][0][i] += shift;
              x[kk][j][0][i + 2] += shift;
            }
#pragma unroll
            for (int v = 0; v < DP / 16; ++v) {
              o[v][j][i] *= alpha;
              o[v][j][i + 2] *= alpha;
            }
          }
        open = __any_sync(~0u, none);
      }

      // weights, rounded to fp16 for the product (2^-12 of each on average, or 2^-25 of the largest), and turned round: keys on the
      // side that is summed over
      uint32_t w[TW][NT][2];
#pragma unroll
      for (int kk = 0; kk < TW; ++kk)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float (&y)[4] = x[kk][j][0];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = exp2_fast(y[e]);
            l[j][e & 1] += y[e];
          }
          w[kk][j][0] = transpose8x8(half2_bits(y[0], y[1]));
          w[kk][j][1] = transpose8x8(half2_bits(y[2], y[3]));
        }

      if (s.n > 1 && !all) {  // values of keys that not every row sees
        bool found = false;
#pragma unroll 1
        for (int i = lane + 32 * wm; i < G::kKeys * G::kVectors; i += 32 * TW) {
          const int row = key0 + i / G::kVectors, pos = (tile + step) * kTile + row;
          if ((pos >= high_min && pos < high_max) || (pos >= low_min && pos < low_max))
            found |= clean_vector<F8>(values + place<G::kVectors>(row, i % G::kVectors));
        }
        if (found) not_finite = 1;
        if (TW == 1) __syncwarp(); else named_bar_sync(1 + team, 32 * TW);
      }

      // O^T += V^T P^T: a thread has elements g, g + 8 (8-bit: 2 g, 2 g + 1) of 16 and rows 2 t, 2 t + 1 of 8
#pragma unroll
      for (int v = 0; v < DP / 16; v += F8 ? 2 : 1) {
#pragma unroll
        for (int kk = 0; kk < TW; ++kk) {
          uint32_t r[4];
          // 8-bit: r[2 i], r[2 i + 1] of vector v + i: bytes (key 2 t: elements 2 g, 2 g + 1), (key 2 t + 1: the same); keys + 8
          ldmatrix_x4_trans(further<G::kVectors>(values + v_lane, F8 ? v : 2 * v) + kk * 16 * G::kRowBytes, r);
#pragma unroll
          for (int i = 0; i < (F8 ? 2 : 1); ++i) {
            uint32_t a[4];
            if (F8) {
              const uint32_t y = __byte_perm(r[F8 ? 2 * i : 0], 0, 0x3120), z = __byte_perm(r[F8 ? 2 * i + 1 : 0], 0, 0x3120);
              a[0] = e4m3x2_to_f16x2(y);
              a[1] = e4m3x2_to_f16x2(y >> 16);
              a[2] = e4m3x2_to_f16x2(z);
              a[3] = e4m3x2_to_f16x2(z >> 16);
            } else {
              a[0] = r[0]; a[1] = r[1]; a[2] = r[2]; a[3] = r[3];
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) mma_16816(o[F8 ? v + i : v][j], a, w[kk][j][0], w[kk][j][1]);
          }
        }
      }
      keys = keys == ring + (G::kStages - 1) * G::kStage ? ring : keys + G::kStage;
    }

    // ---- the teams' sums meet: [team][row] in the ring, with m and l behind
    copies_wait<0>();
    __syncthreads();
    constexpr int kTeamFloats = G::kRows * G::kJoinStride;
    float* const ml = join + G::kTeams * kTeamFloats;  // [team][row][2]
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 4);
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 8);
        l[j][i] += __shfl_xor_sync(~0u, l[j][i], 16);
        const int r = wm * 8 * NT + j * 8 + t4 * 2 + i;
        if (r < rows) {
          if (g == 0) {
            ml[(team * G::kRows + r) * 2] = m[j][i];
            ml[(team * G::kRows + r) * 2 + 1] = l[j][i];
          }
          float* dst = join + team * kTeamFloats + r * G::kJoinStride;
#pragma unroll
          for (int v = 0; v < DP / 16; ++v) {
            dst[v * 16 + (F8 ? 2 * g : g)] = o[v][j][i];
            dst[v * 16 + (F8 ? 2 * g + 1 : g + 8)] = o[v][j][i + 2];
          }
        }
      }
    __syncthreads();

    // who else has tiles of this item: CTAs c0 .. c1; c0 leaves its part in the second slot of its two, the others in the first
    uint32_t c0 = blockIdx.x, c1 = blockIdx.x;
    const bool whole = nt == s.tiles;
    if (!whole) {
      c0 = stripes.owner(i0);
      while (c0 + 1 < stripes.workers && stripes.begin(c0 + 1) < i1 && stripes.moved(stripes.begin(c0 + 1), i0, i1) == i0) ++c0;
      c1 = stripes.owner(i1 - 1);
      while (stripes.begin(c1) > i0 && stripes.moved(stripes.begin(c1), i0, i1) == i1) --c1;
    }
    constexpr int kSlot = G::kRows * (DP + 4);  // rows of DP sums, the base, the sum of the weights, and two that are not used
    auto slot = [&](uint32_t cta) { return p.partials + (size_t)(2 * cta + (cta == c0)) * kSlot; };
    auto write_out = [&](int r, int d, float4 x, float li) {
      const int token = (row0 + r) / p.group, head = h * p.group + (row0 + r) - token * p.group;
      const bool nothing = base_high + token <= 0;
      const float f = nothing ? 0.f : (F8 && c.v_scale ? __ldg(c.v_scale + h) : 1.f) / li;
      if (nothing) x = make_float4(0.f, 0.f, 0.f, 0.f);
      uint2 w;
      w.x = half2_bits(x.x * f, x.y * f);
      w.y = half2_bits(x.z * f, x.w * f);
      *reinterpret_cast<uint2*>(p.out + ((long long)(s.first + token) * p.q_heads + head) * c.head_dim + d) = w;
    };
    const bool odd_values = s.n > 1 && not_finite;
#pragma unroll 1
    for (int i = tid; i < rows * (DP / 4); i += kThreads) {
      const int r = i / (DP / 4), d = (i % (DP / 4)) * 4;
      if (d >= c.head_dim) continue;
      float mi = kNone;
#pragma unroll
      for (int w = 0; w < G::kTeams; ++w) mi = fmaxf(mi, ml[(w * G::kRows + r) * 2]);
      const float base = mi == kNone ? 0.f : mi;
      float li = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < G::kTeams; ++w) {
        const float f = exp2_fast(ml[(w * G::kRows + r) * 2] - base);
        const float4 y = *reinterpret_cast<const float4*>(join + w * kTeamFloats + r * G::kJoinStride + d);
        li += ml[(w * G::kRows + r) * 2 + 1] * f;
        x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
      }
      if (odd_values) {
        const int high = base_high + (row0 + r) / p.group, low = p.window ? max(0, high - p.window) : 0;
#pragma unroll 1
        for (int pos = max(low, tile * kTile); pos < min(high, (tile + nt) * kTile); ++pos) {
          if (pos >= low_max && pos < high_min) {  // (every row sees these: they were left where they are)
            pos = high_min - 1;
            continue;
          }
          const long long off = cache_offset(c, __ldg(table + (pos >> c.page_shift)), h, pos, p.status);
          if (off < 0) continue;
          float v[4];
          for (int e = 0; e < 4; ++e) {
            if (F8) {
              const uint32_t y = e4m3x2_to_f16x2(static_cast<const uint8_t*>(c.v)[off + d + e]);
              v[e] = __low2float(*reinterpret_cast<const __half2*>(&y));
            } else {
              v[e] = __half2float(static_cast<const __half*>(c.v)[off + d + e]);
            }
            if (isfinite(v[e])) v[e] = 0.f;
          }
          x.x += v[0]; x.y += v[1]; x.z += v[2]; x.w += v[3];
        }
      }
      if (whole) {
        write_out(r, d, x, li);
      } else {
        float* to = slot(blockIdx.x);
        *reinterpret_cast<float4*>(to + r * (DP + 4) + d) = x;
        if (d == 0) *reinterpret_cast<float2*>(to + r * (DP + 4) + DP) = make_float2(mi, li);
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      if (tid == 0) arrived = atom_add_acq_rel_gpu(p.counters + c0, 1);
      __syncthreads();
      if (arrived == (int)(c1 - c0)) {  // the last one: every part is there
        __threadfence();
        if (tid == 0) p.counters[c0] = 0;
        // All parts of as many rows as the ring holds come at once (a load and its use at a time would take a round trip to the
        // L2 for each of up to some hundred parts): [part][row][DP + 2 used, 4 rounded]
        const int parts = (int)(c1 - c0) + 1;
        constexpr int kLine = DP + 4;
        constexpr int kFit = G::kStages * G::kStage / (kLine * 4);
        const int part_step = min(parts, kFit), row_step = max(1, kFit / parts);
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += row_step) {
          const int nr = min(row_step, rows - r0);
          float mi = kNone, li = 0.f;  // (kept from one batch to the next only where a row does not fit: one vector a thread then)
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int w0 = 0; w0 < parts; w0 += part_step) {
            const int nw = min(part_step, parts - w0);
#pragma unroll 1
            for (int wr = warp, w = w0, r = warp; wr < nw * nr; wr += kWarps, r += kWarps) {  // a row of a part per warp
              while (r >= nr) {
                r -= nr;
                ++w;
              }
              const float* from = slot(c0 + w) + (r0 + r) * kLine;
              for (int vec = lane; vec < kLine / 4; vec += 32) copy16(ring + wr * (kLine * 4) + vec * 16, from + vec * 4, true);
            }
            copies_commit();
            copies_wait<0>();
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < nr * (DP / 4); i += kThreads) {
              const int r = i / (DP / 4), d = (i % (DP / 4)) * 4;
              if (w0 == 0) {
                mi = kNone;
                li = 0.f;
                x = make_float4(0.f, 0.f, 0.f, 0.f);
              }
              float top = mi;
              for (int w = 0; w < nw; ++w) top = fmaxf(top, join[(w * nr + r) * kLine + DP]);
              const float base = top == kNone ? 0.f : top, old = exp2_fast(mi - base);
              mi = top;
              li *= old;
              x.x *= old; x.y *= old; x.z *= old; x.w *= old;
              for (int w = 0; w < nw; ++w) {
                const float* from = join + (w * nr + r) * kLine;
                const float f = exp2_fast(from[DP] - base);
                const float4 y = *reinterpret_cast<const float4*>(from + d);
                li += from[DP + 1] * f;
                x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
              }
              if (w0 + nw == parts && d < c.head_dim) write_out(r0 + r, d, x, li);
            }
            __syncthreads();
          }
        }
      }
    }
    if (tid == 0) not_finite = 0;
    __syncthreads();  // the ring and Q are free again
    at = to;
    skip += nt;
    if (skip != (uint32_t)s.tiles) return;  // the range ends within the item
  }
}

template <int DP, int NT, int TW, bool F8>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  using G = Geometry<DP, NT, TW, F8>;
  auto kernel = attention_kernel<DP, NT, TW, F8>;
  static bool attr_set[64] = {};
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmem);
    if (err != cudaSuccess) return err;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  // no more CTAs than there can be tiles: blocks of rows of all sequences, each with the most tiles that the table holds
  const long long most = (long long)(sm_count < kMaxWorkers ? sm_count : kMaxWorkers) * G::kBlocks;
  const long long blocks = ((long long)p.tokens * p.group + G::kRows - 1) / G::kRows + p.cache.sequences;
  const long long per_block = (((long long)p.cache.max_pages << p.cache.page_shift) + kTile - 1) / kTile + 1;
  const long long tiles = (blocks < most ? blocks : most) * (per_block < most ? per_block : most) * p.cache.kv_heads;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles < most ? tiles : most));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = G::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <int DP, int NT, int TW>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return p.cache.eight_bit ? launch<DP, NT, TW, true>(p, sm_count, stream) : launch<DP, NT, TW, false>(p, sm_count, stream);
}
template <int DP>
cudaError_t launch_rows(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  // rows of a usual sequence; one with more takes several blocks of rows.  A warp holds 8 NT rows of sums (DP * NT / 4 registers
  // a thread); more rows than that share keys and values between the warps of a team.
  const long long rows = (p.tokens + p.cache.sequences - 1) / p.cache.sequences * (long long)p.group;
  constexpr int kMost = DP == 256 ? 2 : 4;
  if (rows <= 8) return launch_format<DP, 1, 1>(p, sm_count, stream);
  if (rows <= 16) return launch_format<DP, 2, 1>(p, sm_count, stream);
  if (rows <= 32) return launch_format<DP, kMost, 4 / kMost>(p, sm_count, stream);
  return launch_format<DP, kMost, 8 / kMost>(p, sm_count, stream);
}

}  // namespace

// Two slots per CTA that a grid can have, of its rows with their maxima and sums: most with 64 rows.
size_t attention_slot_bytes(int head_dim) {
  const int dp = padded_dim(head_dim);
  static_assert(blocks_per_sm(64, 1, true) * 8 <= blocks_per_sm(64, 4, true) * 64 &&
                blocks_per_sm(128, 1, true) * 8 <= blocks_per_sm(128, 4, true) * 64, "slots");
  return (size_t)2 * kMaxWorkers * blocks_per_sm(dp, 4, false) * 64 * (dp + 4) * sizeof(float);
}

cudaError_t launch_attention(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  switch (padded_dim(p.cache.head_dim)) {
    case 64: return launch_rows<64>(p, sm_count, stream);
    case 128: return launch_rows<128>(p, sm_count, stream);
    default: return launch_rows<256>(p, sm_count, stream);
  }
}

}  // namespace marlin_b200
