// Attention of new tokens over the paged cache, split over the keys and joined in the same launch.
//
// For one key head and the R = (tokens) * (query heads per key head) rows that read it:  s_j = scale q . k_j,
// o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), m the largest s_j.  Sums over different ranges of keys join exactly:
// (m, l, o) of two ranges give m = max(m1, m2), l = l1 e^(m1 - m) + l2 e^(m2 - m), o alike.  So the work is numbered in
// tiles of 64 keys of (sequence, key head, block of rows), and every CTA takes an equal range of that numbering, whatever
// the lengths are: the lengths are read on the device, so a captured launch stays balanced as sequences grow.
//
// What bounds it: the cache is read once (2 * 2 * head_dim bytes per key and key head), at 16 rows for 4 * 16 * head_dim
// operations of the tensor cores: 16 operations a byte, so the copies have to be kept in flight and nothing else counts.
// Every warp streams keys and values of its own share of a tile through a ring in shared memory (16-byte asynchronous
// copies, addresses by key, so that a page may end anywhere), and multiplies with mma.sync: up to 64 rows are far below
// the 128 rows of a tcgen05 tile.
#include <limits.h>

#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kTile = 64;      // keys of a tile
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kLeastTiles = 2;  // tiles that a CTA takes at least, where there are fewer tiles than CTAs would like
constexpr float kNone = -INFINITY;

// DP: head_dim rounded up to 64, 128 or 256.  WM: warps side by side over the rows (16 each); the kWarps / WM teams share
// out the keys of a tile.  F8: e4m3 cache.
template <int DP, int WM, bool F8>
struct Geometry {
  static constexpr int kRows = 16 * WM;
  static constexpr int kTeams = kWarps / WM;
  static constexpr int kKeys = kTile / kTeams;       // keys of a tile that a team multiplies
  static constexpr int kRowBytes = DP * (F8 ? 1 : 2);
  static constexpr int kVectors = kRowBytes / 16;    // 16-byte vectors of a key
  static constexpr int kHalf = kTile * kRowBytes;    // the keys (or the values) of a tile
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kBlocks = DP == 256 ? 1 : 2;  // CTAs per SM
  static constexpr int kQStride = DP * 2 + 16;       // bytes between rows of Q in shared memory: ldmatrix without conflicts
  static constexpr int kQBytes = kRows * kQStride;
  static constexpr int kJoin = kTeams * kRows * (DP + 2) * 4;  // where the teams' sums meet, in the ring
  static constexpr int kRoom = (kBlocks == 1 ? 220 : 110) * 1024 - kQBytes;
  static constexpr int kStages = kRoom / kStage > 8 ? 8 : kRoom / kStage;
  static constexpr int kSmem = kQBytes + kStages * kStage;
  static_assert(kStages >= 2 && kStages * kStage >= kJoin, "ring");
};

constexpr int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
constexpr int blocks_per_sm(int dp) { return dp == 256 ? 1 : 2; }

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

// A row that does not see a key has weight 0 there, and 0 times an infinity or a NaN is NaN.  Keys that no row sees are never
// loaded; where rows see different keys (several new tokens) such values are left out of the product, and what they stand for
// is added to the rows that see them: counts of +inf (or NaN) and of -inf (or NaN), by the same MMA on operands of zeros and ones.
__device__ __forceinline__ bool not_finite(uint32_t two) {
  return (two & 0x7c00u) == 0x7c00u || (two & 0x7c000000u) == 0x7c000000u;
}
struct Operand {
  uint32_t a[4];
};
__device__ __forceinline__ Operand seen_operand(int pos, const int (&low)[2], const int (&high)[2]) {
  Operand r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i & 1, x = pos + (i >> 1) * 8;
    r.a[i] = (x >= low[row] && x < high[row] ? 0x3c00u : 0u) | (x + 1 >= low[row] && x + 1 < high[row] ? 0x3c000000u : 0u);
  }
  return r;
}
__device__ __noinline__ float4 add_not_finite_parts(float4 acc, uint4 p, uint4 seen, uint32_t b0, uint32_t b1) {
  const uint32_t b[2] = {b0, b1};
  uint32_t finite[2], up[2], down[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    finite[i] = up[i] = down[i] = 0;
#pragma unroll
    for (int j = 0; j < 32; j += 16) {
      const uint32_t x = (b[i] >> j) & 0xffffu, big = x & 0x7fffu;
      if (big < 0x7c00u) finite[i] |= x << j;
      if (big > 0x7c00u || x == 0x7c00u) up[i] |= 0x3c00u << j;
      if (big > 0x7c00u || x == 0xfc00u) down[i] |= 0x3c00u << j;
    }
  }
  const uint32_t a[4] = {p.x, p.y, p.z, p.w}, one[4] = {seen.x, seen.y, seen.z, seen.w};
  float x[4] = {acc.x, acc.y, acc.z, acc.w}, u[4] = {0.f, 0.f, 0.f, 0.f}, d[4] = {0.f, 0.f, 0.f, 0.f};
  mma_16816(x, a, finite[0], finite[1]);
  mma_16816(u, one, up[0], up[1]);
  mma_16816(d, one, down[0], down[1]);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] += (u[i] > 0.f ? INFINITY : 0.f) + (d[i] > 0.f ? -INFINITY : 0.f);
  return make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void add_not_finite(float (&acc)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const Operand& seen) {
  const float4 r = add_not_finite_parts(make_float4(acc[0], acc[1], acc[2], acc[3]), make_uint4(a[0], a[1], a[2], a[3]),
                                        make_uint4(seen.a[0], seen.a[1], seen.a[2], seen.a[3]), b0, b1);
  acc[0] = r.x; acc[1] = r.y; acc[2] = r.z; acc[3] = r.w;
}

// What a sequence asks for: new tokens [first, first + n) of the call, keys [low, len), tiles [tile0, tile0 + tiles) of
// them, blocks of rows per key head.  A sequence with new tokens has a tile at least: it writes the zeros.
struct Sequence {
  int len, n, first, low, tile0, tiles, blocks;
};
__device__ __forceinline__ Sequence sequence(const AttentionParams& p, int b, int rows, int* status) {
  Sequence s;
  s.len = cache_length(p.cache, b, status);
  s.first = b;
  s.n = 1;
  if (p.starts) {
    const int from = min(max(__ldg(p.starts + b), 0), p.tokens), to = min(max(__ldg(p.starts + b + 1), from), p.tokens);
    s.first = from;
    s.n = to - from;
  }
  s.low = p.window ? max(0, s.len - s.n - p.window + 1) : 0;
  s.tile0 = s.low / kTile;
  s.tiles = max(1, (s.len + kTile - 1) / kTile - s.tile0);
  s.blocks = s.n ? (int)(((long long)s.n * p.group + rows - 1) / rows) : 0;
  return s;
}

template <int DP, int WM, bool F8>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(DP)) attention_kernel(const AttentionParams p) {
  using G = Geometry<DP, WM, F8>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long scan[kWarps];
  __shared__ long long found_offset;
  __shared__ int found_sequence;
  __shared__ int arrived;
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = warp / WM, wm = warp % WM;
  const int g = lane >> 2, t4 = lane & 3;
  const uint32_t ring = smem_u32(smem) + G::kQBytes;
  float* const join = reinterpret_cast<float*>(smem + G::kQBytes);

  pdl_launch_dependents();
  pdl_wait_prior_grids();

  // ---- this CTA's range of tiles: thread i counts the tiles of sequences [i * per, (i + 1) * per)
  const int per = (c.sequences + kThreads - 1) / kThreads;
  long long mine = 0;
  for (int b = tid * per; b < min(c.sequences, (tid + 1) * per); ++b) {
    const Sequence s = sequence(p, b, G::kRows, p.status);
    mine += (long long)c.kv_heads * s.blocks * s.tiles;
  }
  long long before = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long x = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before += x;
  }
  if (lane == 31) scan[warp] = before;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += scan[w];
    total += scan[w];
  }
  before -= mine;
  const long long workers = min((long long)gridDim.x, max(1ll, total / kLeastTiles));
  if (blockIdx.x >= workers) return;
  long long at = stripe_begin(blockIdx.x, total, workers);
  const long long end = stripe_begin(blockIdx.x + 1, total, workers);
  if (at >= end) return;  // (nothing to do at all)
  if (mine > 0 && before <= at && at < before + mine) {
    int b = tid * per;
    long long off = at - before;
    for (;; ++b) {
      const Sequence s = sequence(p, b, G::kRows, p.status);
      const long long units = (long long)c.kv_heads * s.blocks * s.tiles;
      if (off < units) break;
      off -= units;
    }
    found_sequence = b;
    found_offset = off;
  }
  __syncthreads();
  int b = found_sequence;
  long long off = found_offset;
  Sequence s = sequence(p, b, G::kRows, p.status);

  while (at < end) {
    // ---- one segment: tiles [tile, tile + nt) of (sequence b, key head h, block of rows rb)
    const int item = (int)(off / s.tiles), skip = (int)(off % s.tiles);
    const int h = item / s.blocks, rb = item % s.blocks;
    const int tile = s.tile0 + skip;
    const int nt = (int)min((long long)(s.tiles - skip), end - at);
    const int rows = (int)min((long long)G::kRows, (long long)s.n * p.group - (long long)rb * G::kRows);
    const int row0 = rb * G::kRows;  // row r is query head h * group + r % group of new token r / group

    // ---- copies: every warp brings 16 keys and values of a tile, in most layouts just those that it multiplies
    auto page_of = [&](int step) {  // lanes 0 - 15: the page of the warp's key, or -1
      const int key = (tile + step) * kTile + warp * 16 + (lane & 15);
      return step < nt && key >= s.low && key < s.len ? __ldg(c.table + b * c.table_stride + (key >> c.page_shift)) : -2;
    };
    auto bring = [&](int step, int page) {
      if (step < nt) {
        const int key = (tile + step) * kTile + warp * 16 + (lane & 15);
        const long long mine = page == -2 ? -1 : cache_offset(c, page, h, key, p.status);
        const uint32_t stage = ring + (step % G::kStages) * G::kStage;
        constexpr int kPer = G::kVectors < 32 ? 32 / G::kVectors : 1;  // keys per pass of the warp
#pragma unroll
        for (int r = 0; r < 16; r += kPer) {
          const int row = r + lane / G::kVectors, vec = lane % G::kVectors;
          const long long from = __shfl_sync(~0u, mine, row);
          const bool there = from >= 0 && vec * (F8 ? 16 : 8) < c.head_dim;
          const long long bytes = there ? (from * (F8 ? 1 : 2) + vec * 16) : 0;
          const uint32_t to = stage + place<G::kVectors>(warp * 16 + row, vec);
          copy16(to, static_cast<const uint8_t*>(c.k) + bytes, there);
          copy16(to + G::kHalf, static_cast<const uint8_t*>(c.v) + bytes, there);
        }
      }
      copies_commit();
    };

    // Q goes with the first tile; rows and elements that are not there are zeros
    constexpr int kQVectors = DP / 8;
    for (int i = tid; i < G::kRows * kQVectors; i += kThreads) {
      const int r = i / kQVectors, vec = i % kQVectors;
      const int token = (row0 + r) / p.group, head = h * p.group + (row0 + r) % p.group;
      const bool there = r < rows && vec * 8 < c.head_dim;
      const uint16_t* src = p.q + (there ? (long long)(s.first + token) * p.q_stride + head * c.head_dim + vec * 8 : 0);
      copy16(smem_u32(smem) + r * G::kQStride + vec * 16, src, there);
    }
    int page = page_of(0);
#pragma unroll 1
    for (int i = 0; i < G::kStages - 1; ++i) {
      const int next = page_of(i + 1);
      bring(i, page);
      page = next;
    }

    // the positions that the rows of this thread see: [low, high)
    int high[2], low[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = wm * 16 + g + 8 * i;
      const int pos = s.len - s.n + (row0 + r) / p.group;
      high[i] = r < rows ? pos + 1 : INT_MAX;  // (rows that are not there: Q is zero, the results are not used)
      low[i] = r < rows && p.window ? max(0, pos - p.window + 1) : 0;
    }
    const float factor = p.scale_log2 * (F8 && c.k_scale ? __ldg(c.k_scale + h) : 1.f);

    constexpr bool kQInRegisters = DP <= 128;
    uint32_t q[kQInRegisters ? DP / 16 : 1][4];
    float m[2] = {kNone, kNone}, l[2] = {0.f, 0.f};
    float o[DP / 8][4];
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

    auto load_q = [&](int ks, uint32_t (&a)[4]) {
      const uint32_t base = smem_u32(smem) + (wm * 16) * G::kQStride;
      if (F8) {  // the order of the elements within 16 is that of the keys' bytes: 4 t .. 4 t + 3 in a thread
        const uint2 x = lds64(base + g * G::kQStride + ks * 32 + t4 * 8);
        const uint2 y = lds64(base + (g + 8) * G::kQStride + ks * 32 + t4 * 8);
        a[0] = x.x; a[1] = y.x; a[2] = x.y; a[3] = y.y;
      } else {
        ldmatrix_x4(base + (lane & 15) * G::kQStride + ks * 32 + (lane >> 4) * 16, a);
      }
    };

#pragma unroll 1
    for (int step = 0; step < nt; ++step) {
      copies_wait<G::kStages - 2>();
      if (WM == 1 && step > 0) __syncwarp(); else __syncthreads();  // (the first time for Q)
      {
        const int next = page_of(step + G::kStages);
        bring(step + G::kStages - 1, page);
        page = next;
      }
      if (kQInRegisters && step == 0) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) load_q(ks, q[kQInRegisters ? ks : 0]);
      }
      const uint32_t keys = ring + (step % G::kStages) * G::kStage, values = keys + G::kHalf;
      const int key0 = team * G::kKeys;

      // S = Q K^T
      float sc[G::kKeys / 8][4];
#pragma unroll
      for (int i = 0; i < G::kKeys / 8; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < DP / 16; ks += F8 ? 2 : 1) {
        uint32_t a[F8 ? 2 : 1][4];
#pragma unroll
        for (int i = 0; i < (F8 ? 2 : 1); ++i) {
          if (kQInRegisters) {
#pragma unroll
            for (int j = 0; j < 4; ++j) a[i][j] = q[kQInRegisters ? ks + i : 0][j];
          } else {
            load_q(ks + i, a[i]);
          }
        }
#pragma unroll
        for (int kk = 0; kk < G::kKeys / 16; ++kk) {
          uint32_t r[4];
          if (F8) {
            const int row = key0 + kk * 16 + (lane & 15);
            ldmatrix_x4(keys + place<G::kVectors>(row, ks + (lane >> 4)), r);
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // r[2 i]: keys 0 - 7, r[2 i + 1]: keys 8 - 15 of 16 elements
              mma_16816(sc[2 * kk], a[F8 ? i : 0], e4m3x2_to_f16x2(r[2 * i]), e4m3x2_to_f16x2(r[2 * i] >> 16));
              mma_16816(sc[2 * kk + 1], a[F8 ? i : 0], e4m3x2_to_f16x2(r[2 * i + 1]), e4m3x2_to_f16x2(r[2 * i + 1] >> 16));
            }
          } else {
            const int row = key0 + kk * 16 + (lane & 7) + (lane >> 4) * 8;
            ldmatrix_x4(keys + place<G::kVectors>(row, 2 * ks + ((lane >> 3) & 1)), r);
            mma_16816(sc[2 * kk], a[0], r[0], r[1]);
            mma_16816(sc[2 * kk + 1], a[0], r[2], r[3]);
          }
        }
      }

      // softmax of this tile: logits in units of log2, -inf where a row does not see the key
      const int pos0 = (tile + step) * kTile + key0;
      const bool all = pos0 >= max(low[0], low[1]) && pos0 + G::kKeys <= min(high[0], high[1]);
      float top[2] = {kNone, kNone};
#pragma unroll
      for (int i = 0; i < G::kKeys / 8; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int pos = pos0 + i * 8 + t4 * 2 + (j & 1);
          const bool seen = all || (pos >= low[j >> 1] && pos < high[j >> 1]);
          sc[i][j] = seen ? sc[i][j] * factor : kNone;
          top[j >> 1] = fmaxf(top[j >> 1], sc[i][j]);
        }
      }
      float alpha[2], base[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 1));
        top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 2));
        const float now = fmaxf(m[i], top[i]);
        base[i] = now == kNone ? 0.f : now;
        alpha[i] = exp2_fast(m[i] - base[i]);
        m[i] = now;
        l[i] *= alpha[i];
      }
      if (__any_sync(~0u, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
          o[i][0] *= alpha[0]; o[i][1] *= alpha[0];
          o[i][2] *= alpha[1]; o[i][3] *= alpha[1];
        }
      }
#pragma unroll
      for (int i = 0; i < G::kKeys / 8; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc[i][j] = exp2_fast(sc[i][j] - base[j >> 1]);
          l[j >> 1] += sc[i][j];
        }
      }

      const bool differ = s.n > 1 && __any_sync(~0u, !all);

      // O += P V, P rounded to fp16 (weights of at most 1: off by 2^-12 of the largest, 2^-25 at the least)
#pragma unroll
      for (int kk = 0; kk < G::kKeys / 16; ++kk) {
        const uint32_t a[4] = {half2_bits(sc[2 * kk][0], sc[2 * kk][1]), half2_bits(sc[2 * kk][2], sc[2 * kk][3]),
                               half2_bits(sc[2 * kk + 1][0], sc[2 * kk + 1][1]), half2_bits(sc[2 * kk + 1][2], sc[2 * kk + 1][3])};
        const int row = key0 + kk * 16 + (lane & 15);
#pragma unroll
        for (int v = 0; v < G::kVectors; v += 2) {
          uint32_t r[4];
          ldmatrix_x4_trans(values + place<G::kVectors>(row, v + (lane >> 4)), r);
          uint32_t bv[F8 ? 4 : 2][2];  // operands of the n-tiles
          if (F8) {
            // r[2 i], r[2 i + 1] of vector v + i: bytes (key 2 t: elements 2 g, 2 g + 1), (key 2 t + 1: the same), keys + 8 in
            // the second; the n-tiles take the even and the odd elements of the 16
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t x = __byte_perm(r[i], 0, 0x3120);
              bv[(i >> 1) * 2 + 0][i & 1] = e4m3x2_to_f16x2(x);
              bv[F8 ? (i >> 1) * 2 + 1 : 0][i & 1] = e4m3x2_to_f16x2(x >> 16);
            }
          } else {
            bv[0][0] = r[0]; bv[0][1] = r[1]; bv[1][0] = r[2]; bv[1][1] = r[3];
          }
#pragma unroll
          for (int i = 0; i < (F8 ? 4 : 2); ++i) {
            float (&acc)[4] = o[(F8 ? 2 * v : v) + i];
            if (differ && __any_sync(~0u, not_finite(bv[i][0]) || not_finite(bv[i][1])))
              add_not_finite(acc, a, bv[i][0], bv[i][1], seen_operand(pos0 + kk * 16 + t4 * 2, low, high));
            else
              mma_16816(acc, a, bv[i][0], bv[i][1]);
          }
        }
      }
    }

    // ---- the teams' sums meet: [team][row][DP] in the ring, with m and l behind
    copies_wait<0>();
    __syncthreads();
    constexpr int kTeamFloats = G::kRows * DP;
    float* const ml = join + G::kTeams * kTeamFloats;  // [team][row][2]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(~0u, l[i], 1);
      l[i] += __shfl_xor_sync(~0u, l[i], 2);
      const int r = wm * 16 + g + 8 * i;
      if (r < rows) {
        if (t4 == 0) {
          ml[(team * G::kRows + r) * 2] = m[i];
          ml[(team * G::kRows + r) * 2 + 1] = l[i];
        }
        float* dst = join + team * kTeamFloats + r * DP;
        if (F8) {
#pragma unroll
          for (int v = 0; v < DP / 16; ++v)
            *reinterpret_cast<float4*>(dst + v * 16 + t4 * 4) =
                make_float4(o[2 * v][2 * i], o[2 * v + 1][2 * i], o[2 * v][2 * i + 1], o[2 * v + 1][2 * i + 1]);
        } else {
#pragma unroll
          for (int v = 0; v < DP / 8; ++v)
            *reinterpret_cast<float2*>(dst + v * 8 + t4 * 2) = make_float2(o[v][2 * i], o[v][2 * i + 1]);
        }
      }
    }
    __syncthreads();

    // who else has tiles of this item: CTAs c0 .. c1; c0 leaves its part in the second slot of its two, the others in the first
    const long long item0 = at - skip;
    const int c0 = stripe_owner(item0, total, workers), c1 = stripe_owner(item0 + s.tiles - 1, total, workers);
    const bool whole = c0 == c1;
    constexpr int kSlot = G::kRows * (DP + 2);
    auto slot = [&](int cta) { return p.partials + (size_t)(2 * cta + (cta == c0)) * kSlot; };
    auto write_out = [&](int r, int d, float4 x, float li) {
      const int token = (row0 + r) / p.group, head = h * p.group + (row0 + r) % p.group;
      const int pos = s.len - s.n + token;
      const float f = pos < 0 ? 0.f : (F8 && c.v_scale ? __ldg(c.v_scale + h) : 1.f) / li;
      if (pos < 0) x = make_float4(0.f, 0.f, 0.f, 0.f);
      uint2 w;
      w.x = half2_bits(x.x * f, x.y * f);
      w.y = half2_bits(x.z * f, x.w * f);
      *reinterpret_cast<uint2*>(p.out + ((long long)(s.first + token) * p.q_heads + head) * c.head_dim + d) = w;
    };
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
        const float4 y = *reinterpret_cast<const float4*>(join + w * kTeamFloats + r * DP + d);
        li += ml[(w * G::kRows + r) * 2 + 1] * f;
        x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
      }
      if (whole) {
        write_out(r, d, x, li);
      } else {
        float* to = slot(blockIdx.x);
        *reinterpret_cast<float4*>(to + r * DP + d) = x;
        if (d == 0) {
          to[G::kRows * DP + 2 * r] = mi;
          to[G::kRows * DP + 2 * r + 1] = li;
        }
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      if (tid == 0) arrived = atom_add_acq_rel_gpu(p.counters + c0, 1);
      __syncthreads();
      if (arrived == c1 - c0) {  // the last one: every part is there
        __threadfence();
        if (tid == 0) p.counters[c0] = 0;
        for (int i = tid; i < rows * (DP / 4); i += kThreads) {
          const int r = i / (DP / 4), d = (i % (DP / 4)) * 4;
          if (d >= c.head_dim) continue;
          float mi = kNone;
          for (int w = c0; w <= c1; ++w) mi = fmaxf(mi, __ldcg(slot(w) + G::kRows * DP + 2 * r));
          const float base = mi == kNone ? 0.f : mi;
          float li = 0.f;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int w = c0; w <= c1; ++w) {
            const float* from = slot(w);
            const float2 part = __ldcg(reinterpret_cast<const float2*>(from + G::kRows * DP + 2 * r));
            const float f = exp2_fast(part.x - base);
            const float4 y = ld_cg_f4(reinterpret_cast<const float4*>(from + r * DP + d));
            li += part.y * f;
            x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
          }
          write_out(r, d, x, li);
        }
      }
    }
    __syncthreads();  // the ring and Q are free again

    at += nt;
    off += nt;
    if (at < end && off == (long long)c.kv_heads * s.blocks * s.tiles) {
      off = 0;
      do s = sequence(p, ++b, G::kRows, p.status);
      while (s.blocks == 0);
    }
  }
}

template <int DP, int WM, bool F8>
cudaError_t launch(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  using G = Geometry<DP, WM, F8>;
  auto kernel = attention_kernel<DP, WM, F8>;
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

template <int DP, int WM>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return p.cache.eight_bit ? launch<DP, WM, true>(p, sm_count, stream) : launch<DP, WM, false>(p, sm_count, stream);
}
template <int DP>
cudaError_t launch_rows(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  // rows of a usual sequence; one with more takes several blocks of rows
  const long long rows = (p.tokens + p.cache.sequences - 1) / p.cache.sequences * (long long)p.group;
  if (rows <= 16) return launch_format<DP, 1>(p, sm_count, stream);
  if (rows <= 32) return launch_format<DP, 2>(p, sm_count, stream);
  return launch_format<DP, 4>(p, sm_count, stream);
}

}  // namespace

// Two slots per CTA that a grid can have, of up to 64 rows with their maxima and sums.
size_t attention_slot_bytes(int head_dim) {
  const int dp = padded_dim(head_dim);
  return (size_t)2 * kMaxWorkers * blocks_per_sm(dp) * 64 * (dp + 2) * sizeof(float);
}

cudaError_t launch_attention(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  switch (padded_dim(p.cache.head_dim)) {
    case 64: return launch_rows<64>(p, sm_count, stream);
    case 128: return launch_rows<128>(p, sm_count, stream);
    default: return launch_rows<256>(p, sm_count, stream);
  }
}

}  // namespace marlin_b200
