// Attention with sinks, and over caches of 8 bits with a scale for each block of tokens: instances of the warp-level kernel (attention_warp.cuh).
#include "attention_warp.cuh"

namespace marlin_b200 {
namespace {

template <int DP>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  if (!p.cache.eight_bit) return launch_rows<DP, false, kExtra>(p, sm_count, stream);
  return p.scales.int8 ? launch_rows<DP, true, kExtraInt8>(p, sm_count, stream) : launch_rows<DP, true, kExtra>(p, sm_count, stream);
}

// Whether the kernel for prompts takes a call: at 256 rows a block it wants rows of a sequence and key head, and blocks enough for the SMs, since it
// takes every block whole.  Both sides, tcgen05 with at most 64 rows a block and this one, 64 heads over 8 of 128 elements unless said otherwise:
//   32 sequences, a window of 2000, 64 rows a key head 97 and 106 us, 128 rows 181 and 108, 256 rows 332 and 112;
//   one sequence, a window of 500, 32 blocks 44 and 28, 64 blocks 71 and 28; two, 32 heads, 128 rows, 32 blocks 48 and 29;
//   one of 4000 with no window to speak of, 96 blocks 164 and 78, 128 blocks 217 and 78;
//   32 of 100 to 300 keys, 128 rows 69 and 32; eight of up to 900, 12 heads of 64 elements, 100 rows, 48 blocks 45 and 23.
// Below 24 blocks a few SMs would do all the work.  Sums over more keys than 32768 would lose more in the products than a result's rounding
// (attention_tc.cuh, kFold), and this kernel does not put them aside.
bool is_prompt(const AttentionParams& p) {
  if (p.cache.eight_bit || padded_dim(p.cache.head_dim) > 128) return false;
  const long long span = p.window ? (long long)p.window + p.sinks : (long long)p.cache.max_pages << p.cache.page_shift;
  const long long items = ((long long)p.tokens * p.group + 255) / 256 * p.cache.kv_heads;
  return usual_rows(p) >= 128 && items >= 24 && span <= 32768;
}

}  // namespace

cudaError_t launch_attention_more(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  if (is_prompt(p)) return launch_attention_prompt(p, sm_count, stream);
  switch (padded_dim(p.cache.head_dim)) {
    case 64: return launch_format<64>(p, sm_count, stream);
    case 128: return launch_format<128>(p, sm_count, stream);
    default: return launch_format<256>(p, sm_count, stream);
  }
}

}  // namespace marlin_b200
