// Attention with sinks, and over caches of 8 bits with a scale for each block of tokens: instances of the tcgen05 kernel (attention_tc.cuh).
#include "attention_tc.cuh"

namespace marlin_b200 {

cudaError_t launch_attention_tc_more(const AttentionParams& p, int sm_count, cudaStream_t stream) {
  if (p.cache.eight_bit) return p.scales.int8 ? launch<128, 64, true, kExtraInt8>(p, sm_count, stream) : launch<128, 64, true, kExtra>(p, sm_count, stream);
  return padded_dim(p.cache.head_dim) == 64 ? launch_rows<64, kExtra>(p, sm_count, stream) : launch_rows<128, kExtra>(p, sm_count, stream);
}

}  // namespace marlin_b200
