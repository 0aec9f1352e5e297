// Attention of new tokens over the paged cache: which kernel a call takes (attention_warp.cuh, attention_tc.cuh).
#include "attention_warp.cuh"

namespace marlin_b200 {
namespace {

template <int DP>
cudaError_t launch_format(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  return p.cache.eight_bit ? launch_rows<DP, true, kNoExtra>(p, sm_count, stream) : launch_rows<DP, false, kNoExtra>(p, sm_count, stream);
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
