// New keys and values into a paged cache of 8 bits with a scale for each block of tokens and key head, and the rotation of queries and keys.
//
// The scale of a block is s = a / L (a times the fp32 number nearest to 1 / L), a the largest magnitude in it and L the largest code (127 in
// two's complement, 448 in e4m3); x is held as the code nearest to x * (1 / s).  A block that has tokens already keeps its scale while the new ones fit under s L.
// Otherwise s is doubled as often as that takes, and the codes that are there are divided by the same power of two and rounded once:
// an e4m3 code loses nothing by it unless it becomes subnormal, one in two's complement at most half a step of the new scale, and however
// often a block grows, the losses of a code add up to less than a step of its last scale (1/2 + 1/4 + ...).
//
// The tokens of one call in one block of one sequence are a run.  A CTA takes a run, or a part of its heads, and a team of its warps takes a
// head at a time (one warp several heads, where a run has few tokens): so the scale of a head's keys or values over all tokens of
// the run is found by a few warps, from registers that keep the elements until they are put away.  Queries go the same way without a
// scale.  Runs are numbered without a sum over the sequences: sequence b has the numbers from starts[b] / block + 2 b on, and n tokens
// lie in at most (n - 1) / block + 2 blocks, so no two sequences share a number; the numbers that nobody has end at once.
//
// What bounds it: instructions.  Prompts of five sequences (10.8 thousand tokens, 32 heads and 32 key heads of 128, e4m3, blocks of 64, all
// rotated): 108 us, 4.1 TB/s, where a copy of its bytes would take 67; keys are turned twice, to find the scale and to be put away, since they do not
// fit into registers as 32-bit numbers.  Blocks of 16 take 106 us, of 4 tokens 204.  One token 3.9 us, 64 tokens 3.5: a launch.
// (With the elements read again from the L2 in a second pass: 125 to 148 us for blocks of 64, 119 for 4.)
#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHold = 4;  // pairs of vectors of a lane that are read once; the rest are read again when the scale is known

// What a CTA has to do: tokens rows [row, row + m) at positions [pos, pos + m), which lie in one block; rows [zero, row) have no position.
struct Run {
  int row, m, pos, zero;
  long long place, scale;  // of the first token, head 0 (in codes; -1: its page is not there) and of its block's scale
};

// Unit j of a head, of head_dim / 16: two vectors of eight elements.  They are the two halves of eight pairs, or, where pairs lie side by
// side and in what is not turned, two vectors of their own.
struct Unit {
  int at, second;  // elements of the head where the vectors begin
  bool pair;
};
__device__ __forceinline__ Unit unit_of(const AppendParams& p, int j, bool turns) {
  const int pairs = turns ? p.pair_units : 0, rest = p.cache.head_dim - pairs * 16;
  Unit r;
  r.pair = j < pairs;
  r.at = r.pair ? j * 8 : pairs * 16 + (j - pairs) * 8;
  r.second = r.at + (r.pair ? p.rotary_dim : rest) / 2;
  return r;
}

// x and y turned by the token's angles: `turn` has those of one unit `units` vectors apart, so that the lanes of a warp read neighbouring ones
__device__ __forceinline__ void rotate_side_by_side(const AppendParams& p, const float4* turn, int at, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += 4) {
    const float4 cs = turn[j / 4 * (p.rotary_dim / 8) + at / 8];
    const float a = x[j], d = x[j + 1], b = x[j + 2], e = x[j + 3];
    x[j] = a * cs.x - d * cs.y;
    x[j + 1] = d * cs.x + a * cs.y;
    x[j + 2] = b * cs.z - e * cs.w;
    x[j + 3] = e * cs.z + b * cs.w;
  }
}
__device__ __forceinline__ void rotate(const AppendParams& p, const float4* turn, const Unit& r, float (&x)[8], float (&y)[8]) {
  if (r.pair) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float4 cs = turn[j / 2 * p.pair_units + r.at / 8];
      const float a = x[j], d = y[j], b = x[j + 1], e = y[j + 1];
      x[j] = a * cs.x - d * cs.y;
      y[j] = d * cs.x + a * cs.y;
      x[j + 1] = b * cs.z - e * cs.w;
      y[j + 1] = e * cs.z + b * cs.w;
    }
  } else if (!p.pair_units) {  // (no pair units: pairs side by side, or no rotation at all)
    if (r.at < p.rotary_dim) rotate_side_by_side(p, turn, r.at, x);
    if (r.second < p.rotary_dim) rotate_side_by_side(p, turn, r.second, y);
  }
}

// The largest magnitude of eight elements that is finite, and `top`.
__device__ __forceinline__ float largest_of(const float (&x)[8], float top) {
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));  // (a NaN has no part in it)
  if (most > 3.402823466e38f) {
    most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, finite_or_zero(x[j]));
  }
  return fmaxf(top, most);
}

// four values -> four codes.  Infinities become the largest code; a NaN is 0 in two's complement, which has none.
template <bool INT8>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  if (!INT8) return e4m3x2(a, b) | e4m3x2(c, d) << 16;
  const int i = max(-127, min(127, __float2int_rn(a))), j = max(-127, min(127, __float2int_rn(b)));
  const int k = max(-127, min(127, __float2int_rn(c))), l = max(-127, min(127, __float2int_rn(d)));
  return __byte_perm(__byte_perm(i, j, 0x0040), __byte_perm(k, l, 0x0040), 0x5410);
}
template <bool INT8>
__device__ __forceinline__ void store_codes(uint8_t* to, const float (&x)[8], float f) {
  uint2 w;
  w.x = codes_of<INT8>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
  w.y = codes_of<INT8>(x[4] * f, x[5] * f, x[6] * f, x[7] * f);
  *reinterpret_cast<uint2*>(to) = w;
}
// four codes times a power of two (or 0), rounded
template <bool INT8>
__device__ __forceinline__ uint32_t shrunk(uint32_t w, float f) {
  float x[4];
  if (INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  } else {
    const uint32_t lo = e4m3x2_to_f16x2(w), hi = e4m3x2_to_f16x2(w >> 16);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  }
  return codes_of<INT8>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

// Cosines and sines of the angles position * inv_freq of m tokens from position pos on.  An angle is formed in 64 bits and reduced by whole
// turns there: the rounding of a 32-bit product alone would be off by 2^-24 of it, half a percent of a radian at position 10^5.  Then the fast
// functions of the hardware will do: off by 2^-21 between -pi and pi, a thousandth of the rounding of a query to fp16.  (A CTA
// forms them for itself, 4096 for a run of 64 tokens with 64 pairs; with the exact functions that was more than half of its instructions.)
__device__ __forceinline__ void form_sines(const AppendParams& p, float4* turn, int pos, int m) {
  const int pairs = p.rotary_dim / 2, each = p.pair_units ? 4 : 2;
  if (pairs == 0) return;
  // a thread has one pair (or, of more than there are threads, none) of every token that its group of threads has
  const int group = (int)threadIdx.x / pairs, groups = kThreads / pairs, pair = (int)threadIdx.x - group * pairs;
  if (group >= groups) return;
  constexpr double kTurnsPerRadian = 0.15915494309189533577;
  const double turns_each = (double)load(p.inv_freq + pair) * kTurnsPerRadian;
  const int v = pair / 2;
  float2* const to = reinterpret_cast<float2*>(&turn[v % each * (p.rotary_dim / 4 / each) + v / each]) + pair % 2;
  for (int t = group; t < m; t += groups) {
    const double turns = (double)(pos + t) * turns_each;
    const float angle = (float)(turns - rint(turns)) * 6.283185307179586f;
    to[t * (p.rotary_dim / 2)] = make_float2(__cosf(angle), __sinf(angle));
  }
}

template <bool INT8>
__global__ void __launch_bounds__(kThreads) kv_append_blocks_kernel(const AppendParams p) {
  extern __shared__ float4 turn[];  // of each token, two pairs (cosine, sine) a vector
  __shared__ Run run;
  __shared__ int owner;
  __shared__ float tops[2][kWarps];  // of the warps of a team
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int shift = p.scales.block_shift, block = 1 << shift, id = blockIdx.x;
  if (tid == 0) run.m = owner = -1;
  __syncthreads();
  // whose run this is: every thread looks at a sequence, and the one that has it follows the table
  for (int b = p.starts ? tid : id; b < (p.starts ? c.sequences : id + 1); b += kThreads) {
    if (!p.starts && tid > 0) break;
    int from = b, to = b + 1, nth = 0;
    if (p.starts) {
      from = min(max(load(p.starts + b), 0), p.tokens);
      to = min(max(load(p.starts + b + 1), from), p.tokens);
      const long long first = (from >> shift) + 2ll * b, next = (to >> shift) + 2ll * b + 2;
      if (id < first || id >= next || from == to) continue;
      nth = (int)(id - first);
    }
    if (atomicCAS(&owner, -1, b) != -1) continue;  // (only where begins descend, which they must not: one sequence, not parts of two)
    bool bad = false;
    const int len = cache_length(c, b, bad);
    if (bad && nth == 0) report_cache(p.status);
    const int begin = max(len - (to - from), 0);  // position of the first new token that has one
    const int at = nth ? (begin & -block) + nth * block : begin;
    if (nth && at >= len) continue;
    run.pos = at;
    run.row = to - (len - at);
    run.m = max(0, min(len, (at & -block) + block) - at);
    run.zero = nth ? run.row : from;
    long long place = -1;
    if (run.m > 0) {
      const int page = load(c.table + b * c.table_stride + (at >> c.page_shift));
      place = cache_offset(c, page, 0, at, p.status);
      run.scale = page * p.scales.s_page + ((at & ((1 << c.page_shift) - 1)) >> shift) * p.scales.s_block;
    }
    run.place = place;
  }
  __syncthreads();
  if (run.m < 0) return;  // nobody's
  const int m = run.m, row = run.row, pos = run.pos;

  form_sines(p, turn, pos, m);
  __syncthreads();

  // Where this lane stands: unit j of token first + i * pass of one of the `heads` heads that the warp has at a time.
  const int units = c.head_dim / 16, per = 32 / units, tokens = max(1, min(m, per)), heads = per / tokens;
  int team = 1;  // warps that have a head together: as many as keep all its tokens in registers
  while (team < kWarps && team * per * kHold < m) team *= 2;
  const int place = lane / units, j = lane - place * units, sub = place / tokens, pass = tokens * team;
  const bool has = place < tokens * heads;  // (lanes that are left over have nothing)
  const int mine = place - sub * tokens + warp % team * tokens, first = has ? mine : m;
  // lanes that have the same head
  const uint32_t together = (tokens * units == 32 ? ~0u : (1u << tokens * units) - 1) << sub * tokens * units;
  const int fill = pos & (block - 1);  // tokens that the block has already
  const int q_groups = (p.q_heads + heads - 1) / heads, kv_groups = (c.kv_heads + heads - 1) / heads;
  const int teams = kWarps / team;
  int odd = 0;
  for (int g = blockIdx.y * teams + warp / team; g < q_groups + 2 * kv_groups; g += gridDim.y * teams) {
    const bool query = g < q_groups, key = !query && g < q_groups + kv_groups;
    const int h = (query ? g : key ? g - q_groups : g - q_groups - kv_groups) * heads + sub;
    const bool there = h < (query ? p.q_heads : c.kv_heads);
    if (!query && (m == 0 || run.place < 0)) continue;  // (the same for the CTA)
    const int begin = there ? first : m;
    const Unit r = unit_of(p, j, query || key);
    const long long stride = query ? p.q_stride : key ? p.k_stride : p.v_stride;
    const uint16_t* const src = (query ? p.q : key ? p.k : p.v) + row * stride + h * c.head_dim;
    uint4 lo[kHold], hi[kHold];
    auto ask = [&](int t, uint4& a, uint4& b) {
      a = load(reinterpret_cast<const uint4*>(src + t * stride + r.at));
      b = load(reinterpret_cast<const uint4*>(src + t * stride + r.second));
    };
    float x[8], y[8];
    auto turned = [&](int t, const uint4& a, const uint4& b) {
      to_floats(a, x);
      to_floats(b, y);
      if (query || key) rotate(p, turn + t * (p.rotary_dim / 4), r, x, y);
    };
    float* const scale_at = (key ? p.scales.k : p.scales.v) + run.scale + h * p.scales.s_head;
    const float old = !query && fill && there ? load(scale_at) : 0.f;
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (begin + i * pass < m) ask(begin + i * pass, lo[i], hi[i]);

    if (query) {
      const long long out_stride = (long long)p.q_heads * c.head_dim;
      uint16_t* const dst = p.q_out + h * c.head_dim;
      if (there && has)
        for (int t = run.zero + mine; t < row; t += pass) {  // (tokens without a position)
          *reinterpret_cast<uint4*>(dst + t * out_stride + r.at) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(dst + t * out_stride + r.second) = make_uint4(0, 0, 0, 0);
        }
      for (int t0 = begin; t0 < m; t0 += kHold * pass) {
        if (t0 != begin) {
#pragma unroll
          for (int i = 0; i < kHold; ++i)
            if (t0 + i * pass < m) ask(t0 + i * pass, lo[i], hi[i]);
        }
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
          const int t = t0 + i * pass;
          if (t >= m) break;
          turned(t, lo[i], hi[i]);
          *reinterpret_cast<uint4*>(dst + (row + t) * out_stride + r.at) = to_halves(x);
          *reinterpret_cast<uint4*>(dst + (row + t) * out_stride + r.second) = to_halves(y);
        }
      }
      continue;
    }

    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int t = begin + i * pass;
      if (t >= m) break;
      turned(t, lo[i], hi[i]);
      top = largest_of(y, largest_of(x, top));
    }
#pragma unroll 2
    for (int t = begin + kHold * pass; t < m; t += pass) {
      uint4 a, b;
      ask(t, a, b);
      turned(t, a, b);
      top = largest_of(y, largest_of(x, top));
    }
    if (heads == 1) {
      top = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top)));
      if (team > 1) {
        if (lane == 0) tops[odd][warp] = top;
        named_bar_sync(1 + warp / team, team * 32);
        for (int i = warp / team * team; i < warp / team * team + team; ++i) top = fmaxf(top, tops[odd][i]);
        odd ^= 1;  // (the next head's go elsewhere: nobody is more than a barrier ahead)
      }
    } else if (has) {
      top = __uint_as_float(__reduce_max_sync(together, __float_as_uint(top)));
    }

    const float need = top * (INT8 ? 1.f / 127.f : 1.f / 448.f);
    const bool begun = fill && old > 0.f && old <= 3.402823466e38f;
    float now = begun ? old : need, shrink = begun ? 1.f : 0.f;
    while (now < need) {
      now *= 2.f;
      shrink *= 0.5f;
    }
    // (everybody has asked for the scale that was: those of a team before they met)
    if (there && has && j == 0 && mine == 0 && !(fill && now == old)) *scale_at = now;
    uint8_t* const base = static_cast<uint8_t*>(key ? c.k : c.v) + run.place + h * c.s_head;
    if (fill && shrink != 1.f && there && has) {  // what the block has is held under the new scale
      for (int t = mine; t < fill; t += pass) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint2* const at = reinterpret_cast<uint2*>(base + (t - fill) * c.s_token + (i ? r.second : r.at));
          uint2 v = make_uint2(0, 0);  // (under a scale that is none every code stands for 0, a NaN's too)
          if (begun) {
            v = *at;
            v.x = shrunk<INT8>(v.x, shrink);
            v.y = shrunk<INT8>(v.y, shrink);
          }
          *at = v;
        }
      }
    }
    // (a scale below 2^-128 that was there before, over zeros: they stay zeros)
    const float inverse = now > 0.f ? fminf(__fdiv_rn(1.f, now), 3.402823466e38f) : 0.f;
    auto put = [&](int t) {
      store_codes<INT8>(base + t * c.s_token + r.at, x, inverse);
      store_codes<INT8>(base + t * c.s_token + r.second, y, inverse);
    };
    // A scale of 0: infinities and zeros of either sign have the code 0, a NaN stays one.  (A loop of its own: looked for in `put` it cost
    // prompts 3 %.)
    if (now == 0.f) {
#pragma unroll 1
      for (int t = begin; t < m; t += pass) {
        uint4 a, b;
        ask(t, a, b);
        turned(t, a, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = x[i] != x[i] ? x[i] : 0.f;
          y[i] = y[i] != y[i] ? y[i] : 0.f;
        }
        put(t);
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int t = begin + i * pass;
      if (t >= m) break;
      turned(t, lo[i], hi[i]);
      put(t);
    }
#pragma unroll 2
    for (int t = begin + kHold * pass; t < m; t += pass) {
      uint4 a, b;
      ask(t, a, b);
      turned(t, a, b);
      put(t);
    }
  }
}

template <bool INT8>
cudaError_t launch(const AppendParams& p, unsigned runs, unsigned parts, int smem, cudaStream_t stream) {
  static bool attr_set[64] = {};
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev < 0 || dev >= 64 || !attr_set[dev]) {  // the most that any call asks for: 128 tokens with 128 pairs
    err = cudaFuncSetAttribute(kv_append_blocks_kernel<INT8>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 128 * 8);
    if (err != cudaSuccess) return err;
    if (dev >= 0 && dev < 64) attr_set[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(runs, parts);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv_append_blocks_kernel<INT8>, p);
}

}  // namespace

cudaError_t launch_kv_append_blocks(AppendParams p, int interleaved, int sm_count, cudaStream_t stream) {
  p.rotary_dim = p.inv_freq ? p.rotary_dim : 0;
  p.pair_units = interleaved ? 0 : p.rotary_dim / 16;
  const long long block = 1ll << p.scales.block_shift;
  const long long runs = p.starts ? p.tokens / block + 2ll * p.cache.sequences : p.cache.sequences;
  const int most = p.starts ? (int)(p.tokens < block ? p.tokens : block) : 1;  // tokens of a run
  const int per = 32 / (p.cache.head_dim / 16);
  int team = 1;
  while (team < kWarps && team * per * kHold < most) team *= 2;
  // the heads of a run are shared out to as many CTAs as give every SM eight of them, about (each forms the sines of the run for itself)
  const long long busy = p.starts ? p.tokens / block + p.cache.sequences : runs;
  const int heads = most < per ? per / most : 1;
  const long long groups = (p.q_heads + heads - 1) / heads + 2ll * ((p.cache.kv_heads + heads - 1) / heads);
  const long long parts = (groups * team + kWarps - 1) / kWarps;
  const long long wanted = min(parts, (8ll * sm_count + busy - 1) / busy);
  const int smem = most * p.rotary_dim / 2 * 8;
  const auto run = p.scales.int8 ? launch<true> : launch<false>;
  return run(p, (unsigned)runs, (unsigned)max(1ll, wanted), smem, stream);
}

}  // namespace marlin_b200
