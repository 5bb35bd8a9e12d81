// The tail attention of layers with a sliding window: the same kernels over fewer key
// tiles (a translation unit of its own, compiled beside the other).
#include "tail_attn_tc.cuh"

namespace kvm {

void launch_window_attention(const AttnParams& p, cudaStream_t s) { launch_all<true>(p, s); }

}  // namespace kvm
