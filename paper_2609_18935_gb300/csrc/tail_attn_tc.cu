// The tail attention over whole caches, and which of its kernels a layer runs.
#include "tail_attn_tc.cuh"

namespace kvm {

void launch_tail_attention(const AttnParams& p, cudaStream_t s) {
    if (p.n_ctas <= 0) return;
    if (p.window > 0) launch_window_attention(p, s);
    else launch_all<false>(p, s);
}

// One block per SM: 384 threads of about 150 registers leave no room for a
// second (and head_dim 256 needs all of TMEM and shared memory).
int attention_ctas_per_sm(int) { return 1; }

}  // namespace kvm
