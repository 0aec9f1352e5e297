// Attention with sinks, and over caches of 8 bits with a scale for each block of tokens: instances of the warp-level kernel (attention_warp.cuh).
#include "attention_warp.cuh"

namespace marlin_b200 {
namespace {

template <int DP>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  if (!p.cache.eight_bit) return launch_rows<DP, false, kExtra>(p, sm_count, stream);
  return p.scales.int8 ? launch_rows<DP, true, kExtraInt8>(p, sm_count, stream) : launch_rows<DP, true, kExtra>(p, sm_count, stream);
}

// Whether the kernel for prompts takes a call.
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
