// The tcgen05 kernel of the attention (attention_tc.cuh): its instances.
#include "attention_tc.cuh"

namespace marlin_b200 {

cudaError_t launch_attention_tc(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  if (p.cache.eight_bit) return launch<128, 64, true, kNoExtra>(p, sm_count, stream);
  return padded_dim(p.cache.head_dim) == 64 ? launch_rows<64, kNoExtra>(p, sm_count, stream) : launch_rows<128, kNoExtra>(p, sm_count, stream);
}

}  // namespace marlin_b200
