// Attention over the 4-bit cache, heads of 128 channels (serve_attn.cuh).
#include "serve_attn.cuh"

namespace kint {
cudaError_t launch_attn_128(const AttnP& p, int what, cudaStream_t s) { return pick<128>(p, what, s); }
}  // namespace kint
