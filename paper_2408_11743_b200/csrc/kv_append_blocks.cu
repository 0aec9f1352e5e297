// New keys and values into a paged cache of 8 bits with a scale for each block of tokens and key head, and the rotation of queries and keys.
//
// The scale of a block is s = a / L, a the largest magnitude in it and L the largest code (127 in two's complement, 448 in e4m3);
// x is held as the code nearest to x * (1 / s).  A block that has tokens already keeps its scale while the new ones fit under s L.
// Otherwise s is doubled as often as that takes, and the codes that are there are divided by the same power of two and rounded once:
// an e4m3 code loses nothing by it unless it becomes subnormal, one in two's complement at most half a step of the new scale, and however
// often a block grows, the losses of a code add up to less than a step of its last scale (1/2 + 1/4 + ...).
//
// The tokens of one call in one block of one sequence are a run.  A CTA takes a run, or a part of its heads: one warp finds the scale of
// one head's keys (or values) over all tokens of the run, so that nothing has to meet across warps, and the queries are shared out
// to all threads.  Runs are numbered without a sum over the sequences: sequence b has the numbers from starts[b] / block + 2 b on, and n tokens
// lie in at most (n - 1) / block + 2 blocks, so no two sequences share a number; the numbers that nobody has end at once.
#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHold = 4;  // vectors (or pairs of them) of a lane that are read once; the rest are read again when the scale is known

// What a CTA has to do: tokens rows [row, row + m) at positions [pos, pos + m), which lie in one block; rows [zero, row) have no position.
struct Run {
  int row, m, pos, zero;
  long long place, scale;  // of the first token, head 0 (in codes; -1: its page is not there) and of its block's scale
};

// unit j of a head that is turned: eight pairs (two vectors), or a vector
struct Unit {
  int at;     // element of the head where its (first) vector begins
  bool pair;  // second vector at at + rotary_dim / 2
  bool turned;
};
__device__ __forceinline__ Unit unit_of(const AppendParams& p, int j) {
  Unit r;
  r.pair = j < p.pair_units;
  r.at = r.pair ? j * 8 : p.pair_units * 16 + (j - p.pair_units) * 8;
  r.turned = r.pair || r.at < p.rotary_dim;  // (pairs side by side: no pair units, the first rotary_dim elements)
  return r;
}

// x (and, of a pair unit, y) turned by the token's angles: `turn` has those of one unit `units` vectors apart, so that the lanes of a warp
// read neighbouring ones
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
  } else if (r.turned) {
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const float4 cs = turn[j / 4 * (p.rotary_dim / 8) + r.at / 8];
      const float a = x[j], d = x[j + 1], b = x[j + 2], e = x[j + 3];
      x[j] = a * cs.x - d * cs.y;
      x[j + 1] = d * cs.x + a * cs.y;
      x[j + 2] = b * cs.z - e * cs.w;
      x[j + 3] = e * cs.z + b * cs.w;
    }
  }
}

__device__ __forceinline__ float largest_of(const float (&x)[8], float top) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float a = fabsf(x[j]);
    top = fmaxf(top, a <= 3.402823466e38f ? a : 0.f);  // (what is not finite has no part in the scale)
  }
  return top;
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

template <bool INT8>
__global__ void __launch_bounds__(kThreads) kv_append_blocks_kernel(const AppendParams p) {
  extern __shared__ float4 turn[];  // of each token, two pairs (cosine, sine) a vector
  __shared__ Run run;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const KvCacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int shift = p.scales.block_shift, block = 1 << shift, id = blockIdx.x;
  if (tid == 0) run.m = -1;
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

  for (int i = tid; i < m * (p.rotary_dim / 2); i += kThreads) {
    constexpr double kTurnsPerRadian = 0.15915494309189533577;
    const int token = i / (p.rotary_dim / 2), pair = i - token * (p.rotary_dim / 2);
    const double turns = (double)(pos + token) * (double)load(p.inv_freq + pair) * kTurnsPerRadian;
    float s, co;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &co);
    const int v = pair / 2, each = p.pair_units ? 4 : 2;
    reinterpret_cast<float2*>(&turn[token * (p.rotary_dim / 4) + v % each * (p.rotary_dim / 4 / each) + v / each])[pair % 2] = make_float2(co, s);
  }
  __syncthreads();

  // keys and values: a warp has the keys (or the values) of a head
  const int fill = pos & (block - 1);  // tokens that the block has already
  for (int w = blockIdx.y * kWarps + warp; w < 2 * c.kv_heads && m > 0 && run.place >= 0; w += gridDim.y * kWarps) {
    const bool key = w < c.kv_heads;
    const int h = key ? w : w - c.kv_heads;
    const int units = key ? p.head_units : c.head_dim / 8;
    const int per = 32 / units, mine = lane / units, j = lane - mine * units;  // tokens a pass, and where this lane stands
    Unit r = unit_of(p, j);
    if (!key) {
      r.at = j * 8;
      r.pair = r.turned = false;
    }
    const long long stride = key ? p.k_stride : p.v_stride;
    const uint16_t* const src = (key ? p.k : p.v) + row * stride + h * c.head_dim + r.at;
    float* const scale_at = (key ? p.scales.k : p.scales.v) + run.scale + h * p.scales.s_head;
    uint8_t* const base = static_cast<uint8_t*>(key ? c.k : c.v) + run.place + h * c.s_head;
    const float old = fill ? load(scale_at) : 0.f;
    uint4 lo[kHold], hi[kHold];
    const int first = mine < per ? mine : m;  // (lanes without a unit have no token)
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int t = first + i * per;
      if (t >= m) break;
      lo[i] = load(reinterpret_cast<const uint4*>(src + t * stride));
      if (r.pair) hi[i] = load(reinterpret_cast<const uint4*>(src + t * stride + p.rotary_dim / 2));
    }
    float x[8], y[8];
    auto turned = [&](int t, const uint4& a, const uint4& b) {
      to_floats(a, x);
      if (r.pair) to_floats(b, y);
      rotate(p, turn + t * (p.rotary_dim / 4), r, x, y);
    };
    auto again = [&](int t) {
      const uint4 a = load(reinterpret_cast<const uint4*>(src + t * stride));
      uint4 b = a;
      if (r.pair) b = load(reinterpret_cast<const uint4*>(src + t * stride + p.rotary_dim / 2));
      turned(t, a, b);
    };
    float top = 0.f;
    auto look = [&] {
      top = largest_of(x, top);
      if (r.pair) top = largest_of(y, top);
    };
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int t = first + i * per;
      if (t >= m) break;
      turned(t, lo[i], hi[i]);
      look();
    }
#pragma unroll 2
    for (int t = first + kHold * per; t < m; t += per) {
      again(t);
      look();
    }
    top = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top)));

    const float need = __fdiv_rn(top, INT8 ? 127.f : 448.f);
    const bool begun = fill && old > 0.f && old <= 3.402823466e38f;
    float now = begun ? old : need, shrink = begun ? 1.f : 0.f;
    while (now < need) {
      now *= 2.f;
      shrink *= 0.5f;
    }
    if (lane == 0 && !(fill && now == old)) *scale_at = now;
    if (fill && shrink != 1.f) {  // what the block has is held under the new scale
      const int vectors = c.head_dim / 8;
      for (int i = lane; i < fill * vectors; i += 32) {
        const int t = i / vectors;
        uint2* const at = reinterpret_cast<uint2*>(base + (t - fill) * c.s_token + (i - t * vectors) * 8);
        uint2 v = *at;
        v.x = shrunk<INT8>(v.x, shrink);
        v.y = shrunk<INT8>(v.y, shrink);
        *at = v;
      }
    }
    const float inverse = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
    auto put = [&](int t) {
      uint8_t* const to = base + t * c.s_token + r.at;
      store_codes<INT8>(to, x, inverse);
      if (r.pair) store_codes<INT8>(to + p.rotary_dim / 2, y, inverse);
    };
#pragma unroll
    for (int i = 0; i < kHold; ++i) {
      const int t = first + i * per;
      if (t >= m) break;
      turned(t, lo[i], hi[i]);
      put(t);
    }
#pragma unroll 2
    for (int t = first + kHold * per; t < m; t += per) {
      again(t);
      put(t);
    }
  }

  // queries: a thread has the same unit of every token
  const int units = p.q_heads * p.head_units;
  for (int u = blockIdx.y * kThreads + tid; u < units; u += gridDim.y * kThreads) {
    const int head = u / p.head_units;
    const Unit r = unit_of(p, u - head * p.head_units);
    const uint16_t* const src = p.q + head * c.head_dim + r.at;
    uint16_t* const dst = p.q_out + head * c.head_dim + r.at;
    const long long out_stride = (long long)p.q_heads * c.head_dim;
    for (int t = run.zero; t < row; ++t) {  // (tokens without a position)
      *reinterpret_cast<uint4*>(dst + t * out_stride) = make_uint4(0, 0, 0, 0);
      if (r.pair) *reinterpret_cast<uint4*>(dst + t * out_stride + p.rotary_dim / 2) = make_uint4(0, 0, 0, 0);
    }
#pragma unroll 2
    for (int t = 0; t < m; ++t) {
      float x[8], y[8];
      to_floats(load(reinterpret_cast<const uint4*>(src + (row + t) * p.q_stride)), x);
      if (r.pair) to_floats(load(reinterpret_cast<const uint4*>(src + (row + t) * p.q_stride + p.rotary_dim / 2)), y);
      rotate(p, turn + t * (p.rotary_dim / 4), r, x, y);
      *reinterpret_cast<uint4*>(dst + (row + t) * out_stride) = to_halves(x);
      if (r.pair) *reinterpret_cast<uint4*>(dst + (row + t) * out_stride + p.rotary_dim / 2) = to_halves(y);
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
  p.head_units = p.pair_units + (p.cache.head_dim - p.pair_units * 16) / 8;
  const long long block = 1ll << p.scales.block_shift;
  const long long runs = p.starts ? p.tokens / block + 2ll * p.cache.sequences : p.cache.sequences;
  const int most = p.starts ? (int)(p.tokens < block ? p.tokens : block) : 1;  // tokens of a run
  // the heads of a run are shared out to as many CTAs as give every SM eight of them, about
  const long long busy = p.starts ? p.tokens / block + p.cache.sequences : runs;
  const long long units = (long long)p.q_heads * p.head_units;
  const long long parts = max((units + kThreads - 1) / kThreads, (2ll * p.cache.kv_heads + kWarps - 1) / kWarps);
  const long long wanted = min(parts, (8ll * sm_count + busy - 1) / busy);
  const int smem = most * p.rotary_dim / 2 * 8;
  const auto run = p.scales.int8 ? launch<true> : launch<false>;
  return run(p, (unsigned)runs, (unsigned)max(1ll, wanted), smem, stream);
}

}  // namespace marlin_b200
