// The gated delta rule over a tree of drafted tokens, from the carried state,
// which it leaves alone (kvm_draft_gdn).
//
// A node's state is S advanced along the path to it:
//     S_i = alpha_i S_p (I - beta_i k_i k_i^T) + beta_i v_i k_i^T   (p: its parent, S for a root),  o_i = S_i q_i.
// Written out over the path, with G_i the product of alpha up to node i and
// R_ij that of the nodes after j up to i (j an ancestor of i),
//     u_i = beta_i (v_i - G_i S k_i - sum_{j < i} R_ij (k_i . k_j) u_j),
//     o_i = G_i S q_i + sum_{j <= i} R_ij (q_i . k_j) u_j,
// sums over ancestors.  So S is read once for all nodes, whatever the tree, and
// no node's state is formed; u_i stays behind for the commit (draft.cu).
#include "kvm_internal.cuh"
#include "packed_f32.cuh"

namespace kvm {
namespace {

constexpr int kThreads = 128;
constexpr int kRows = 32;                        // rows of S a block

__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
    }
}

template <int DK, bool CONV>
__global__ void __launch_bounds__(kThreads) draft_gdn_kernel(const __grid_constant__ DraftGdnParams p, int most) {
    constexpr int NP = DK / 32, GK = DK / 8, LD = DK + 4;
    extern __shared__ __align__(16) float sm[];
    const int b = blockIdx.z, h = blockIdx.y, r0 = blockIdx.x * kRows;
    const int n0 = p.cu[b], n = p.cu[b + 1] - n0;
    float* ks = sm;                              // [most][LD]
    float* qs = ks + most * LD;
    float* us = qs + most * LD;                  // [most][kRows]: v, then u
    float* as = us + most * kRows;               // S k
    float* ds = as + most * kRows;               // S q
    float* C = ds + most * kRows;                // [most][most]: R_ij (k_i . k_j)
    float* E = C + most * most;                  // R_ij (q_i . k_j)
    float* al = E + most * most;
    float* be = al + most;
    float* G = be + most;
    __shared__ unsigned long long anc[kDraftNodes];
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependents_launch();
    if (n <= 0) return;
    const int H = p.H, dv = p.dv, hk = H * DK;
    const int j = tid & 7, row = tid >> 3;
    const float* Sg = p.S + (((int64_t)b * H + h) * dv + r0 + 2 * row) * DK + 4 * j;
    float4 s[2][NP];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NP; ++i) s[r][i] = *reinterpret_cast<const float4*>(Sg + r * DK + 32 * i);
    for (int i = tid; i < n; i += kThreads) {
        anc[i] = p.anc[n0 + i];
        al[i] = p.alpha[(int64_t)(n0 + i) * H + h];
        be[i] = p.beta[(int64_t)(n0 + i) * H + h];
    }
    __syncthreads();
    // ---- stage k, q, v: eight channels a thread; a k row's GK lanes share its norm
    const int per = 2 * GK + kRows / 8, all = n * per;
    for (int e0 = 0; e0 < (all + 31) / 32 * 32; e0 += kThreads) {
        // whole warps: k pieces first
        const int e = e0 + tid;
        const int nk = n * GK;
        const bool act = e < all, is_k = e < nk, is_v = e >= 2 * nk;
        const int x = is_k ? e : is_v ? e - 2 * nk : e - nk;
        const int i = act ? (is_v ? x / (kRows / 8) : x / GK) : 0, c = 8 * (is_v ? x % (kRows / 8) : x % GK);
        const __nv_bfloat16* in = is_v ? p.v : is_k ? p.k : p.q;
        const int64_t stride = is_v ? (int64_t)H * dv : hk;
        const int at = is_v ? h * dv + r0 + c : h * DK + c;       // channel within the part
        const int ch = at + (is_v ? 2 * hk : is_k ? hk : 0);      // and of the convolution
        float y[8] = {};
        float sq = 0.f;
        if (act) {
            const uint4 own = *reinterpret_cast<const uint4*>(in + (int64_t)(n0 + i) * stride + at);
            if constexpr (CONV) {
                unsigned long long m = anc[i];
#pragma unroll
                for (int t = 3; t >= 0; --t) {       // the node, then its ancestors upwards, then carried inputs
                    uint4 v;
                    if (m) {
                        const int a = 63 - __clzll(m);
                        m &= ~(1ull << a);
                        v = *reinterpret_cast<const uint4*>(in + (int64_t)(n0 + a) * stride + at);
                    } else {
                        const int r = t + __popcll(anc[i]) - 1;    // carried row: 2 is the input before the root
                        v = *reinterpret_cast<const uint4*>(p.state_in + ((int64_t)b * 3 + r) * p.channels + ch);
                    }
                    float f[8];
                    unpack8(v, f);
#pragma unroll
                    for (int q = 0; q < 8; ++q) y[q] = fmaf(p.w[(int64_t)(ch + q) * 4 + t], f[q], y[q]);
                }
#pragma unroll
                for (int q = 0; q < 8; q += 2) {
                    const float2 v = silu2(pack2(y[q], y[q + 1]));
                    y[q] = v.x;
                    y[q + 1] = v.y;
                }
#pragma unroll
                for (int q = 0; q < 8; ++q) sq = fmaf(y[q], y[q], sq);
                // what a commit carries on: the raw inputs (q and k by the first slice's block)
                if (is_v || blockIdx.x == 0)
                    *reinterpret_cast<uint4*>(p.rec_x + (int64_t)(n0 + i) * p.channels + ch) = own;
            } else {
                unpack8(own, y);
            }
        }
        if constexpr (CONV) {
#pragma unroll
            for (int o = GK / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
            const float inv = !is_k ? 1.f : sq > 0.f ? rsqrtf(sq) : 0.f;
            // the delta rule's operands are bf16, as after the convolution of a tail
#pragma unroll
            for (int q = 0; q < 8; ++q) y[q] = __bfloat162float(__float2bfloat16_rn(y[q] * inv));
        }
        if (act) {
            float* dst = is_v ? us + i * kRows + c : (is_k ? ks : qs) + i * LD + c;
#pragma unroll
            for (int q = 0; q < 8; ++q) dst[q] = y[q];
            if (is_k && blockIdx.x == 0) {
#pragma unroll
                for (int q = 0; q < 8; ++q) p.rec_k[((int64_t)(n0 + i) * H + h) * DK + c + q] = __float2bfloat16_rn(y[q]);
            }
        }
    }
    if (blockIdx.x == 0)
        for (int i = tid; i < n; i += kThreads) p.rec_a[(int64_t)(n0 + i) * H + h] = al[i];
    __syncthreads();
    // ---- S k and S q
    for (int i = 0; i < n; ++i) {
        float a[2] = {}, d[2] = {};
#pragma unroll
        for (int x = 0; x < NP; ++x) {
            const float4 k = *reinterpret_cast<const float4*>(ks + i * LD + 4 * j + 32 * x);
            const float4 q = *reinterpret_cast<const float4*>(qs + i * LD + 4 * j + 32 * x);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float4 t = s[r][x];
                a[r] = fmaf(t.x, k.x, fmaf(t.y, k.y, fmaf(t.z, k.z, fmaf(t.w, k.w, a[r]))));
                d[r] = fmaf(t.x, q.x, fmaf(t.y, q.y, fmaf(t.z, q.z, fmaf(t.w, q.w, d[r]))));
            }
        }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                a[r] += __shfl_xor_sync(0xffffffffu, a[r], o);
                d[r] += __shfl_xor_sync(0xffffffffu, d[r], o);
            }
        if (j == 0)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                as[i * kRows + 2 * row + r] = a[r];
                ds[i * kRows + 2 * row + r] = d[r];
            }
    }
    // ---- decays: column j of R down the tree (a product, so a zero decay is one)
    if (tid <= n) {
        const int c = tid;                       // c == n: G
        for (int i = 0; i < n; ++i) {
            const unsigned long long up = anc[i] & ~(1ull << i);
            const int par = up ? 63 - __clzll(up) : -1;
            if (c == n) G[i] = al[i] * (par >= 0 ? G[par] : 1.f);
            else C[i * most + c] = c == i ? 1.f : c < i && (anc[i] >> c & 1) ? al[i] * C[par * most + c] : 0.f;
        }
    }
    __syncthreads();
    for (int e = tid; e < n * n; e += kThreads) {
        const int i = e / n, c = e % n;
        float kk = 0.f, qk = 0.f;
        const float R = C[i * most + c];
        if (R != 0.f) {
            for (int x = 0; x < DK; x += 4) {
                const float4 a = *reinterpret_cast<const float4*>(ks + i * LD + x), t = *reinterpret_cast<const float4*>(qs + i * LD + x);
                const float4 k = *reinterpret_cast<const float4*>(ks + c * LD + x);
                kk = fmaf(a.x, k.x, fmaf(a.y, k.y, fmaf(a.z, k.z, fmaf(a.w, k.w, kk))));
                qk = fmaf(t.x, k.x, fmaf(t.y, k.y, fmaf(t.z, k.z, fmaf(t.w, k.w, qk))));
            }
        }
        C[i * most + c] = c == i ? 0.f : R * kk;
        E[i * most + c] = R * qk;
    }
    __syncthreads();
    // ---- the updates, a row of S a thread
    if (tid < kRows) {
        for (int i = 0; i < n; ++i) {
            float x = us[i * kRows + tid] - G[i] * as[i * kRows + tid];
            for (int c = 0; c < i; ++c) x = fmaf(-C[i * most + c], us[c * kRows + tid], x);
            us[i * kRows + tid] = be[i] * x;
        }
    }
    __syncthreads();
    for (int e = tid; e < n * kRows; e += kThreads) {
        const int i = e / kRows, r = e % kRows;
        float o = G[i] * ds[i * kRows + r];
        for (int c = 0; c <= i; ++c) o = fmaf(E[i * most + c], us[c * kRows + r], o);
        const int64_t at = ((int64_t)(n0 + i) * H + h) * dv + r0 + r;
        p.out[at] = __float2bfloat16_rn(o);
        p.rec_u[at] = us[i * kRows + r];
    }
}

template <int DK, bool CONV>
void launch(const DraftGdnParams& p, int most, cudaStream_t s) {
    auto bytes = [](int m) { return sizeof(float) * ((size_t)m * (2 * (DK + 4) + 3 * kRows + 3) + 2 * (size_t)m * m); };
    static unsigned long long configured = 0;    // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(draft_gdn_kernel<DK, CONV>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes(kDraftNodes));
        configured |= 1ull << (dev & 63);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.dv / kRows, p.H, p.n_chars);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes(most);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, draft_gdn_kernel<DK, CONV>, p, most);
}

}  // namespace

void launch_draft_gdn(const DraftGdnParams& p, int most, cudaStream_t s) {
    if (p.dk == 64) p.w ? launch<64, true>(p, most, s) : launch<64, false>(p, most, s);
    else p.w ? launch<128, true>(p, most, s) : launch<128, false>(p, most, s);
}

}  // namespace kvm
