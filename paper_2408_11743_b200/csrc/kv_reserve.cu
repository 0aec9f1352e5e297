// Page tables, begins and slots of a step from the lengths of its sequences: what a host would do between two steps, on the GPU, so that
// steps can be queued and replayed without it.
//
// Everything is a sum over the sequences in front: where a sequence's rows begin, which of the free pages it gets, where the pages that it
// gives back go.  A CTA takes the sequences kChunk at a time, a thread each, sums over them in two levels (lanes, warps), and looks its
// tokens up among the begins of the chunk.  With many tokens several CTAs do the same sums and share the tokens out; lengths and the
// stack of free pages, which all of them read, are written by the one that comes last.
//
// What bounds it: the latency of a launch and of a chain of three loads and three sums where there are few tokens.
#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kChunk = 512, kWarps = kChunk / 32;
constexpr int kTokens = 8192;  // of a CTA, at least, before there is a second one

struct Sums {
  long long a, b;
};
// Sums over the threads in front, and over all of them.
__device__ __forceinline__ Sums sums_before(Sums x, Sums* warps, Sums& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums y = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const long long a = __shfl_up_sync(~0u, y.a, d), b = __shfl_up_sync(~0u, y.b, d);
    if (lane >= d) {
      y.a += a;
      y.b += b;
    }
  }
  if (lane == 31) warps[warp] = y;
  __syncthreads();
  Sums before = {y.a - x.a, y.b - x.b};
  all = {0, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const Sums s = warps[w];
    if (w < warp) {
      before.a += s.a;
      before.b += s.b;
    }
    all.a += s.a;
    all.b += s.b;
  }
  __syncthreads();
  return before;
}

// What becomes of a sequence: it keeps `base` tokens and gets those of rows [begin, end); its row of the table goes from `held` pages to `after`,
// the first new one being number `need` of those that are taken, the first one given back number `back` of those.
struct Step {
  long long begin, end, need, back;
  int base, held, after, old;
  bool fits, served;
};

struct Chunk {
  int begin[kChunk], base[kChunk], held[kChunk], after[kChunk], need[kChunk];
  long long back[kChunk];
  bool served[kChunk];
};

// entry i with the largest value[i] <= x, of n in ascending order, value[0] <= x
template <class T>
__device__ __forceinline__ int last_up_to(const T* value, int n, long long x) {
  int low = 0, high = n;
  while (high - low > 1) {
    const int middle = (low + high) / 2;
    if (value[middle] <= x)
      low = middle;
    else
      high = middle;
  }
  return low;
}

__global__ void __launch_bounds__(kChunk) kv_reserve_kernel(const ReserveParams p) {
  __shared__ Chunk chunk;
  __shared__ Sums warps[kWarps];
  __shared__ unsigned long long taken;  // pages, by those that were served
  __shared__ int arrived;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int tid = threadIdx.x, shift = p.page_shift;
  const int said = load(p.free_count), there = min(max(said, 0), p.capacity);
  bool bad = tid == 0 && said != there;
  if (tid == 0) taken = 0;

  // The step of sequence b (n: those of the chunk that are there); `before`: of the chunks in front.
  struct {
    long long rows, need, back;
  } before;
  auto step_of = [&](int b0) {
    const int b = b0 + tid;
    Step s = {};
    long long count = 0;
    bool sound = false;
    if (b < p.sequences) {
      const int len = load(p.lengths + b);
      s.old = s.base = len < 0 ? ~len : len;
      if (p.keep) s.base = min(max(load(p.keep + b), 0), s.old);
      count = p.counts ? load(p.counts + b) : 1;
      sound = count >= 0;
      count = max(count, 0ll);
      const long long total = s.base + count, pages = (total + (1ll << shift) - 1) >> shift;
      s.held = (int)(((long long)s.old + (1ll << shift) - 1) >> shift);
      sound = sound && pages <= p.max_pages && s.held <= p.max_pages && total <= kLongest;
      s.after = sound ? (int)pages : s.held;
    }
    Sums all;
    s.begin = before.rows + sums_before({count, 0}, warps, all).a;
    s.end = s.begin + count;
    before.rows += all.a;
    s.fits = sound && s.end <= p.tokens;
    bad |= b < p.sequences && !s.fits;
    const long long need = s.fits ? max(s.after - s.held, 0) : 0, back = s.fits ? max(s.held - s.after, 0) : 0;
    const Sums x = sums_before({need, back}, warps, all);
    s.need = before.need + x.a;
    s.back = before.back + x.b;
    before.need += all.a;
    before.back += all.b;
    s.served = s.fits && (need == 0 || s.need + need <= there);
    if (s.served && need > 0) atomicMax(&taken, (unsigned long long)(s.need + need));
    chunk.begin[tid] = (int)min(s.begin, (long long)INT_MAX);
    chunk.base[tid] = s.base;
    chunk.held[tid] = s.held;
    chunk.after[tid] = s.after;
    chunk.need[tid] = (int)min(s.need, (long long)INT_MAX);
    chunk.back[tid] = s.back;
    chunk.served[tid] = s.served;
    __syncthreads();
    return s;
  };

  // ---- begins, new entries of the table, slots and positions of this CTA's tokens
  const int each = (p.tokens + (int)gridDim.x - 1) / (int)gridDim.x;
  const int token0 = (int)min((long long)blockIdx.x * each, (long long)p.tokens), token1 = (int)min((long long)token0 + each, (long long)p.tokens);
  before = {0, 0, 0};
  if (blockIdx.x == 0 && tid == 0 && p.starts) p.starts[0] = 0;
  Step s;
  for (int b0 = 0; b0 < p.sequences; b0 += kChunk) {
    const long long rows0 = before.rows;
    __syncthreads();
    s = step_of(b0);
    if (blockIdx.x == 0 && p.starts && b0 + tid < p.sequences) p.starts[b0 + tid + 1] = (int)min(s.end, (long long)INT_MAX);
    const int n = min(kChunk, p.sequences - b0);
    for (long long t = max(rows0, (long long)token0) + tid; t < min(before.rows, (long long)token1); t += kChunk) {
      const int i = last_up_to(chunk.begin, n, t);
      const bool served = chunk.served[i];
      const int pos = chunk.base[i] + (int)(t - chunk.begin[i]), entry = pos >> shift;
      int page = -1;
      if (served) {
        int* const at = p.table + (b0 + i) * p.table_stride + entry;
        if (entry < chunk.held[i]) {
          page = load(at);
        } else {
          page = load(p.free_pages + (there - 1 - (chunk.need[i] + entry - chunk.held[i])));
          if ((pos & ((1 << shift) - 1)) == 0) *at = page;
        }
      }
      if (p.slots) p.slots[t] = page >= 0 ? ((long long)page << shift) + (pos & ((1 << shift) - 1)) : -1;
      if (p.positions) p.positions[t] = served ? pos : -1;
    }
  }
  for (long long t = max(before.rows, (long long)token0) + tid; t < token1; t += kChunk) {  // rows of nobody
    if (p.slots) p.slots[t] = -1;
    if (p.positions) p.positions[t] = -1;
  }

  // ---- lengths and the stack, when everybody has read them
  if (bad) report_cache(p.status);
  __syncthreads();
  if (gridDim.x > 1) {
    if (tid == 0) arrived = atom_add_acq_rel_gpu(p.counter, 1);
    __syncthreads();
    if (arrived != (int)gridDim.x - 1) return;
    if (tid == 0) *p.counter = 0;
  }
  const long long now = there - (long long)taken + before.back;
  if (tid == 0) {
    *p.free_count = (int)min(now, (long long)p.capacity);
    if (now > p.capacity) report_cache(p.status);
  }
  before = {0, 0, 0};
  for (int b0 = 0; b0 < p.sequences; b0 += kChunk) {
    const long long back0 = before.back;
    __syncthreads();
    if (p.sequences > kChunk)
      s = step_of(b0);
    else
      before.back = now - there + (long long)taken;  // (the only chunk is still there)
    if (b0 + tid < p.sequences) p.lengths[b0 + tid] = s.served ? s.base + (int)(s.end - s.begin) : ~s.old;
    const int n = min(kChunk, p.sequences - b0);
    for (long long j = back0 + tid; j < before.back; j += kChunk) {
      const int i = last_up_to(chunk.back, n, j);
      const int page = load(p.table + (b0 + i) * p.table_stride + chunk.after[i] + (j - chunk.back[i]));
      const long long at = now - 1 - j;
      if (at < p.capacity) p.free_pages[at] = page;
    }
  }
}

}  // namespace

cudaError_t launch_kv_reserve(const ReserveParams& p, int sm_count, cudaStream_t stream) {
  const int wanted = (p.tokens + kTokens - 1) / kTokens;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)max(1, min(wanted, sm_count)));
  cfg.blockDim = dim3(kChunk);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv_reserve_kernel, p);
}

}  // namespace marlin_b200
