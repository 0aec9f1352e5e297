// Page tables, begins and slots of a step from the lengths of its sequences: what a host would do between two steps, on the GPU, so that
// steps can be queued and replayed without it.
//
// Everything is a sum over the sequences in front: where a sequence's rows begin, which of the free pages it gets, where the pages that it
// gives back go.  A CTA takes the sequences kChunk at a time, a thread each, sums all three over them at once (lanes, then warps), and looks
// its tokens up among the begins of the chunk.  With many tokens several CTAs do the same sums and share the tokens out; lengths and the
// stack of free pages, which all of them read, are written by the one that comes last.
//
// What bounds it: the latency of a launch, of a chain of three loads, the sums and a search.  Measured, a step and the step that takes it back in a
// graph: 64 sequences with a token each 10.0 us (5.0 a call), a thousand prompts of up to 700 tokens 41.4 (350 thousand slots and
// positions, 4.2 MB; and eleven thousand pages that go back on the stack from one CTA).
#include "kv_cache.cuh"

namespace marlin_b200 {
namespace {

constexpr int kChunk = 512, kWarps = kChunk / 32;
constexpr int kTokens = 1024;  // of a CTA, at least, before there is a second one
constexpr int kMost = 0x7fffffff;

// Sums stay at kMost when they reach it: more rows, or pages, than there can be, of a sequence that is refused.
__device__ __forceinline__ int plus(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kMost); }
struct Sums {
  int rows, need, back, none;
};
__device__ __forceinline__ Sums plus(const Sums& a, const Sums& b) { return {plus(a.rows, b.rows), plus(a.need, b.need), plus(a.back, b.back), 0}; }
// Sums over the threads in front, and over all of them.
__device__ __forceinline__ Sums sums_before(Sums x, Sums* warps, Sums& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums y = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Sums z = {__shfl_up_sync(~0u, y.rows, d), __shfl_up_sync(~0u, y.need, d), __shfl_up_sync(~0u, y.back, d), 0};
    if (lane >= d) y = plus(y, z);
  }
  if (lane == 31) warps[warp] = y;
  const Sums left = {__shfl_up_sync(~0u, y.rows, 1), __shfl_up_sync(~0u, y.need, 1), __shfl_up_sync(~0u, y.back, 1), 0};
  __syncthreads();
  Sums before = lane ? left : Sums{0, 0, 0, 0};
  all = {0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const Sums s = warps[w];
    if (w < warp) before = plus(before, s);
    all = plus(all, s);
  }
  return before;
}

// What becomes of a sequence: it keeps `base` tokens and gets those of rows [begin, end); its row of the table goes from `held` pages to `after`,
// the first new one being number `need` of those that are taken, the first one given back number `back` of those.
struct Step {
  int begin, end, need, back, base, held, after, old;
  bool served;
};

struct Chunk {
  int begin[kChunk], base[kChunk], held[kChunk], after[kChunk], need[kChunk], back[kChunk];
  bool served[kChunk];
};

// entry i with the largest value[i] <= x, of n in ascending order, value[0] <= x
__device__ __forceinline__ int last_up_to(const int* value, int n, int x) {
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
  __shared__ int taken, returned;  // pages, by and of those that were served
  __shared__ int arrived;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int tid = threadIdx.x, shift = p.page_shift;
  const int said = load(p.free_count), there = min(max(said, 0), p.capacity);
  bool bad = tid == 0 && said != there;
  if (tid == 0) taken = returned = 0;

  Sums before;  // of the chunks in front
  // The step of sequence b0 + tid, also into `chunk`.  (All of a chunk's threads call it, behind a barrier.)
  auto step_of = [&](int b0) {
    const int b = b0 + tid;
    Step s = {};
    int count = 0, need = 0, back = 0;
    bool sound = false;
    if (b < p.sequences) {
      const int len = load(p.lengths + b);
      const int kept = p.keep ? load(p.keep + b) : kMost, said = p.counts ? load(p.counts + b) : 1;
      s.old = len < 0 ? ~len : len;
      s.base = min(max(kept, 0), s.old);
      count = max(said, 0);
      const long long total = (long long)s.base + count, pages = (total + (1ll << shift) - 1) >> shift;
      s.held = (int)(((long long)s.old + (1ll << shift) - 1) >> shift);
      sound = said >= 0 && pages <= p.max_pages && s.held <= p.max_pages && total <= kLongest;
      s.after = sound ? (int)pages : s.held;
      need = max(s.after - s.held, 0);
      back = max(s.held - s.after, 0);
    }
    // (Behind a sequence whose rows do not fit none fits: what these need and give back counts for nobody.)
    Sums all;
    const Sums x = plus(before, sums_before({count, need, back, 0}, warps, all));
    before = plus(before, all);
    s.begin = x.rows;
    s.end = plus(x.rows, count);
    s.need = x.need;
    s.back = x.back;
    const bool fits = sound && s.end <= p.tokens;
    bad |= b < p.sequences && !fits;
    const int upto = plus(x.need, need);
    s.served = fits && (need == 0 || upto <= there);
    if (s.served && need > 0) atomicMax(&taken, upto);
    if (s.served && back > 0) atomicMax(&returned, plus(x.back, back));
    chunk.begin[tid] = s.begin;
    chunk.base[tid] = s.base;
    chunk.held[tid] = s.held;
    chunk.after[tid] = s.after;
    chunk.need[tid] = s.need;
    chunk.back[tid] = s.back;
    chunk.served[tid] = s.served;
    __syncthreads();
    return s;
  };

  // ---- begins, new entries of the table, slots and positions of this CTA's tokens
  const int each = (p.tokens + (int)gridDim.x - 1) / (int)gridDim.x;
  const int token0 = (int)min((long long)blockIdx.x * each, (long long)p.tokens), token1 = (int)min((long long)token0 + each, (long long)p.tokens);
  before = {0, 0, 0, 0};
  if (blockIdx.x == 0 && tid == 0 && p.starts) p.starts[0] = 0;
  Step s;
  for (int b0 = 0; b0 < p.sequences; b0 += kChunk) {
    const int rows0 = min(before.rows, p.tokens);  // (a sum that has run full, and a thread's number added to it, would be negative)
    __syncthreads();
    s = step_of(b0);
    if (blockIdx.x == 0 && p.starts && b0 + tid < p.sequences) p.starts[b0 + tid + 1] = s.end;
    const int n = min(kChunk, p.sequences - b0);
#pragma unroll 2
    for (int t = max(rows0, token0) + tid; t < min(before.rows, token1); t += kChunk) {
      const int i = last_up_to(chunk.begin, n, t);
      const bool served = chunk.served[i];
      const int pos = chunk.base[i] + (t - chunk.begin[i]), entry = pos >> shift;
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
  for (int t = max(min(before.rows, p.tokens), token0) + tid; t < token1; t += kChunk) {  // rows of nobody
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
  const int all_back = min(returned, kMost - 9 * kChunk);
  const long long now = (long long)there - taken + all_back;
  if (tid == 0) {
    *p.free_count = (int)min(now, (long long)p.capacity);
    if (now > p.capacity) report_cache(p.status);
  }
  const bool again = p.sequences > kChunk;  // (otherwise the only chunk is still there)
  if (again) before = {0, 0, 0, 0};
  int back0 = 0;
  for (int b0 = 0; b0 < p.sequences; b0 += kChunk) {
    if (again) {
      back0 = min(before.back, all_back);
      __syncthreads();
      s = step_of(b0);
    }
    if (b0 + tid < p.sequences) p.lengths[b0 + tid] = s.served ? s.base + (s.end - s.begin) : ~s.old;
    const int n = min(kChunk, p.sequences - b0);
    // (eight at a time: one latency for all of them)
    const int back1 = min(before.back, all_back);
    for (int j0 = back0 + tid; j0 < back1; j0 += 8 * kChunk) {
      int page[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int j = j0 + k * kChunk;
        if (j >= back1) break;
        const int i = last_up_to(chunk.back, n, j);
        page[k] = load(p.table + (b0 + i) * p.table_stride + chunk.after[i] + (j - chunk.back[i]));
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const long long at = now - 1 - (j0 + k * kChunk);
        if (j0 + k * kChunk < back1 && at < p.capacity) p.free_pages[at] = page[k];
      }
    }
  }
}

}  // namespace

cudaError_t launch_kv_reserve(const ReserveParams& p, int sm_count, cudaStream_t stream) {
  const int wanted = (p.tokens + kTokens - 1) / kTokens;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)max(1, min(wanted, 2 * sm_count)));
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
