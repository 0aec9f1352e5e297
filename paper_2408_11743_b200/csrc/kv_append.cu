// New keys and values into the paged cache, with the rotation of queries and keys by their positions on the way.
//
// A rotation turns pairs (a, c) of a head by t = position * inv_freq[j]:  (a cos t - c sin t, c cos t + a sin t).  One CTA
// takes one token (or a part of its heads, where there are few tokens): its first threads form the token's sines and
// cosines once, while the loads of all threads are on their way, and every 16-byte vector is read once and written once.
// t is formed in 64 bits and reduced by whole turns there: the rounding of a 32-bit product alone would be off by 2^-24 t,
// half a percent of a radian at position 10^5.
//
// What bounds it: the bytes where there are many tokens (10800 of them with 32 heads each of queries, keys and values: 82 us, 6.5 TB/s, of
// reads and writes in equal parts, as fast as a copy; 97 us with divisions by run-time numbers in place of multiplications and with
// sines that lay in the order of the pairs, four lanes to a bank: 62 % of the issue slots were taken), and one chain of dependent
// loads (length, page number, then the stores) where there are few: 2.2 us for one token, 2.9 for 64.
#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kThreads = 256;
constexpr int kMostUnits = 4;  // units (a vector, or the two vectors of eight pairs) that a thread holds at a time

struct Unit {
  int head;      // 0 .. q_heads - 1 queries, then keys, then values
  int at;        // element of the head where its (first) vector begins
  bool pair;     // second vector at at + rotary_dim / 2
  bool turned;
};

// u / d for magic = magic_of(d): (u * ceil(2^31 / d)) >> 31 is off by less than u * d / 2^31 of a step of 1 / d, and u * d < 2^28 here
__device__ __forceinline__ int divided(int u, uint32_t magic) { return (int)__umulhi(2u * (uint32_t)u, magic); }
uint32_t magic_of(int d) { return ((1u << 31) + (uint32_t)d - 1) / (uint32_t)d; }

__device__ __forceinline__ Unit unit_of(const AppendParams& p, int u) {
  const int turning = (p.q_heads + p.cache.kv_heads) * p.head_units;
  Unit r;
  if (u >= turning) {
    const int w = u - turning, per = p.cache.head_dim / 8;
    r.head = divided(w, p.value_magic);
    r.at = (w - r.head * per) * 8;
    r.head += p.q_heads + p.cache.kv_heads;
    r.pair = r.turned = false;
    return r;
  }
  r.head = divided(u, p.head_magic);
  const int j = u - r.head * p.head_units;
  r.pair = j < p.pair_units;
  r.at = r.pair ? j * 8 : p.pair_units * 16 + (j - p.pair_units) * 8;
  r.turned = r.pair || r.at < p.rotary_dim;  // (pairs side by side: no pair units, the first rotary_dim elements)
  return r;
}

template <bool F8>
__device__ __forceinline__ void store_cache(void* base, long long off, const float (&x)[8], float scale) {
  if (F8) {
    uint2 w;
    w.x = e4m3x2(x[0] / scale, x[1] / scale) | e4m3x2(x[2] / scale, x[3] / scale) << 16;
    w.y = e4m3x2(x[4] / scale, x[5] / scale) | e4m3x2(x[6] / scale, x[7] / scale) << 16;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + off) = w;
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + off) = to_halves(x);
  }
}

template <bool F8>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendParams p) {
  // cosine and sine of each pair, two pairs a vector: those of one unit (8 pairs, or 4 of pairs side by side) lie `units` apart, so that
  // the units that a warp turns read neighbouring vectors
  __shared__ float4 turn[64];
  __shared__ int sequence, position;
  __shared__ long long place;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = blockIdx.x, tid = threadIdx.x;
  const KvCacheView& c = p.cache;
  const int first = (blockIdx.y * p.units_per_thread) * kThreads + tid;

  uint4 lo[kMostUnits], hi[kMostUnits];
#pragma unroll
  for (int i = 0; i < kMostUnits; ++i) {
    const int u = first + i * kThreads;
    if (i >= p.units_per_thread || u >= p.units) break;
    const Unit r = unit_of(p, u);
    const uint16_t* src;
    if (r.head < p.q_heads)
      src = p.q + (long long)t * p.q_stride + r.head * c.head_dim;
    else if (r.head < p.q_heads + c.kv_heads)
      src = p.k + (long long)t * p.k_stride + (r.head - p.q_heads) * c.head_dim;
    else
      src = p.v + (long long)t * p.v_stride + (r.head - p.q_heads - c.kv_heads) * c.head_dim;
    lo[i] = load(reinterpret_cast<const uint4*>(src + r.at));
    if (r.pair) hi[i] = load(reinterpret_cast<const uint4*>(src + r.at + p.rotary_dim / 2));
  }

  // whose token this is, and where it goes: every thread looks at a sequence, and the one whose rows hold the token follows the
  // table, so that the loads of a step are on their way together
  const float frequency = p.inv_freq && tid < p.rotary_dim / 2 ? load(p.inv_freq + tid) : 0.f;
  if (tid == 0) sequence = -1;
  __syncthreads();
  for (int b = p.starts ? tid : t; b < (p.starts ? c.sequences : t + 1); b += kThreads) {
    if (!p.starts && tid > 0) break;
    const int from = p.starts ? load(p.starts + b) : t, end = p.starts ? load(p.starts + b + 1) : t + 1;
    bool bad = false;
    const int len = cache_length(c, b, bad);
    if (bad) report_cache(p.status);
    if (from > t || t >= end) continue;
    const int pos = len - (end - t);
    position = pos;
    place = pos >= 0 ? cache_offset(c, load(c.table + b * c.table_stride + (pos >> c.page_shift)), 0, pos, p.status) : -1;
    sequence = b;
  }
  __syncthreads();
  if (sequence < 0) return;  // nobody's
  const int pos = position;
  const long long to = place;
  if (p.inv_freq && tid < p.rotary_dim / 2) {
    constexpr double kTurnsPerRadian = 0.15915494309189533577;
    const double turns = (double)pos * (double)frequency * kTurnsPerRadian;
    float s, co;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &co);
    const int v = tid / 2, each = p.pair_units ? 4 : 2;
    reinterpret_cast<float2*>(&turn[v % each * (p.rotary_dim / 4 / each) + v / each])[tid % 2] = make_float2(co, s);
  }
  __syncthreads();

#pragma unroll
  for (int i = 0; i < kMostUnits; ++i) {
    const int u = first + i * kThreads;
    if (i >= p.units_per_thread || u >= p.units) break;
    const Unit r = unit_of(p, u);
    float x[8], y[8];
    to_floats(lo[i], x);
    if (r.pair) {
      to_floats(hi[i], y);
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
    if (r.head < p.q_heads) {
      uint16_t* dst = p.q_out + ((long long)t * p.q_heads + r.head) * c.head_dim + r.at;
      const uint4 none = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(dst) = pos >= 0 ? to_halves(x) : none;
      if (r.pair) *reinterpret_cast<uint4*>(dst + p.rotary_dim / 2) = pos >= 0 ? to_halves(y) : none;
    } else if (to >= 0) {
      const bool key = r.head < p.q_heads + c.kv_heads;
      const int h = r.head - p.q_heads - (key ? 0 : c.kv_heads);
      const float* scales = key ? c.k_scale : c.v_scale;
      const float scale = F8 && scales ? load(scales + h) : 1.f;
      const long long off = to + h * c.s_head + r.at;
      store_cache<F8>(key ? c.k : c.v, off, x, scale);
      if (r.pair) store_cache<F8>(key ? c.k : c.v, off + p.rotary_dim / 2, y, scale);
    }
  }
}

}  // namespace

cudaError_t launch_kv_append(AppendParams p, int tokens, int interleaved, int sm_count, cudaStream_t stream) {
  const int rotary = p.inv_freq ? p.rotary_dim : 0;
  p.rotary_dim = rotary;
  p.pair_units = interleaved ? 0 : rotary / 16;
  p.head_units = p.pair_units + (p.cache.head_dim - p.pair_units * 16) / 8;
  p.head_magic = magic_of(p.head_units);
  p.value_magic = magic_of(p.cache.head_dim / 8);
  p.units = (p.q_heads + p.cache.kv_heads) * p.head_units + p.cache.kv_heads * (p.cache.head_dim / 8);
  // a few tokens: their heads are spread over more CTAs, until the SMs have two each
  p.units_per_thread = kMostUnits;
  while (p.units_per_thread > 1 &&
         (long long)tokens * ((p.units + kThreads * p.units_per_thread - 1) / (kThreads * p.units_per_thread)) < 2 * sm_count)
    p.units_per_thread /= 2;
  const int per = kThreads * p.units_per_thread;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tokens, (p.units + per - 1) / per);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, p.cache.eight_bit ? kv_append_kernel<true> : kv_append_kernel<false>, p);
}

}  // namespace marlin_b200
