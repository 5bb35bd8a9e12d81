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
//
// A block of eight warps per (character, head); T = its nodes rounded up to 16.
//  * [K; Q], 2 T rows, lies in shared memory as one 128-byte-swizzled tile: rows
//    of the B operand of S [K; Q]^T and, itself against its K rows, both operands
//    of [K; Q] K^T.  Both products run on the tensor cores (tcgen05, M 128: the
//    rows of S, of [K; Q]) into TMEM, 3 T columns.
//  * S is fp32: 64 columns at a time, loaded as whole lines into registers while
//    the inputs are staged, then split into three bf16 parts (24 bits, so the
//    product is as exact as its fp32 sums: u enters the states of later steps).
//  * C_ij = beta_i R_ij (k_i . k_j) and E_ij = R_ij (q_i . k_j), 0 off the paths,
//    go to shared memory over the consumed parts of S.
//  * Four warps solve for u, a thread a row of S: 16 nodes at a time, first the
//    blocks left of the diagonal, then the triangle in registers; the other four
//    follow with the outputs, one barrier per 16 nodes between them.  fma pairs
//    (f32x2), coefficients as broadcast 16-byte loads: 64 for 256 multiply-adds.
// R_ij = G_i / G_j while no G is small, else products down the path (a decay of 0
// is one).
#include "kvm_internal.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace kvm {
namespace {

using namespace ptx;

constexpr int kThreads = 256;
constexpr int kRowsA = 128;                      // rows of an A operand
constexpr int kPartBytes = kRowsA * 128;         // 64 bf16 columns of S
constexpr int kLdc = kDraftNodes + 4;            // row pitch of C and E: 16-byte rows on all banks
constexpr float kSmallDecay = 0x1p-40f;

// Shared memory for trees of up to T nodes (a multiple of 16).  [K; Q] comes first:
// as an A operand it is read up to row 127, past its own 2 T.
struct Layout {
    int kq, v, s, misc, bytes;
    __host__ __device__ Layout(int T, int dk) {
        const int tile = 2 * T * dk * 2, u = T * kRowsA * 4;         // u takes the tile's place
        kq = 0;
        v = kq + (tile > u ? tile : u);
        s = v + T * kRowsA * 2;
        misc = s + 3 * kPartBytes;
        bytes = misc + 2048;
    }
};
static_assert(2 * kDraftNodes * kLdc * 4 <= 3 * kPartBytes, "C and E take the place of S's parts");

__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// x -> its bf16 value, x -= that
__device__ __forceinline__ float take_bf16(float& x) {
    const float h = __bfloat162float(__float2bfloat16_rn(x));
    x -= h;
    return h;
}

// acc[i] += C[i][0..15] . u[0..15] in pairs (even and odd columns apart)
__device__ __forceinline__ void block16(f2 (&acc)[16], const float* C, const f2 (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(C + i * kLdc + 4 * x);
            acc[i] = fma2(c.x, u[2 * x], acc[i]);
            acc[i] = fma2(c.y, u[2 * x + 1], acc[i]);
        }
}

template <int DK, bool CONV>
__global__ void __launch_bounds__(kThreads, 2) draft_gdn_kernel(const __grid_constant__ DraftGdnParams p) {
    constexpr int HALVES = DK / 64, GK = DK / 8;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const int b = p.order[blockIdx.y], h = blockIdx.x;
    const int n0 = p.cu[b], n = p.cu[b + 1] - n0;
    if (n <= 0) return;
    const Layout at((p.most + 15) / 16 * 16, DK);
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int T = (n + 15) / 16 * 16;
    const uint32_t region = 2 * T * 128;             // bytes of 64 columns of [K; Q]
    uint64_t* anc = reinterpret_cast<uint64_t*>(smem + at.misc);           // [64]
    float* al = reinterpret_cast<float*>(smem + at.misc + 512);            // [64] each
    float* be = al + kDraftNodes;
    float* G = be + kDraftNodes;
    float* rG = G + kDraftNodes;
    const uint32_t bar = base + at.misc + 1536;                            // two barriers, one per half of S
    uint32_t* slot = reinterpret_cast<uint32_t*>(smem + at.misc + 1552);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + at.misc + 1556);
    int* small = reinterpret_cast<int*>(smem + at.misc + 1560);
    float* Cm = reinterpret_cast<float*>(smem + at.s);
    float* Em = Cm + kDraftNodes * kLdc;
    float* U = reinterpret_cast<float*>(smem + at.kq);                     // [T][128]
    __nv_bfloat16* vs = reinterpret_cast<__nv_bfloat16*>(smem + at.v);     // [T][128]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int H = p.H, dv = p.dv, hk = H * DK;
    uint32_t cols = 32;                              // TMEM: S [K; Q]^T, then [K; Q] K^T
    while ((int)cols < 3 * T) cols *= 2;
    if (tid == 0) {
        *abort_flag = 0;
        *small = 0;
        mbar_init(bar, 1);
        mbar_init(bar + 8, 1);
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(smem_u32(slot), cols);
        tmem_relinquish();
    }
    grid_dependency_wait();
    grid_dependents_launch();

    // ---- loads: S (in registers), the nodes' words and gates
    const float* Sg = p.S + ((int64_t)b * H + h) * dv * DK;
    float4 s[HALVES][8];
#pragma unroll
    for (int x = 0; x < HALVES; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = (tid + e * kThreads) >> 4, c4 = tid & 15;
            s[x][e] = row < dv ? *reinterpret_cast<const float4*>(Sg + (int64_t)row * DK + 64 * x + 4 * c4) : make_float4(0, 0, 0, 0);
        }
    if (tid < n) {
        anc[tid] = p.anc[n0 + tid];
        const float a = p.alpha[(int64_t)(n0 + tid) * H + h];
        al[tid] = a;
        be[tid] = p.beta[(int64_t)(n0 + tid) * H + h];
        p.rec_a[(int64_t)(n0 + tid) * H + h] = a;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const uint32_t tg = tmem + 2 * T;

    // ---- stage k, q, v, eight channels a piece: k rows, then q rows, then v rows
    {
        const int nk = n * GK, all = 2 * nk + n * (dv / 8);
        for (int e0 = 0; e0 < all; e0 += kThreads) {
            const int e = e0 + tid;
            const bool act = e < all, is_k = e < nk, is_v = e >= 2 * nk;
            const int x = is_k ? e : is_v ? e - 2 * nk : e - nk;
            const int per = is_v ? dv / 8 : GK;
            const int i = act ? x / per : 0, c = act ? 8 * (x % per) : 0;
            const __nv_bfloat16* in = (is_v ? p.v : is_k ? p.k : p.q) + (is_v ? h * dv : h * DK) + c;
            const int64_t stride = is_v ? (int64_t)H * dv : hk;
            uint4 val = *reinterpret_cast<const uint4*>(in + (int64_t)(n0 + i) * stride);
            if constexpr (CONV) {
                // taps 3, 2, .. are the node, its parent, .. and then the carried inputs from the last back
                const int ch = (is_v ? 2 * hk + h * dv : is_k ? hk + h * DK : h * DK) + c;
                if (act) *reinterpret_cast<uint4*>(p.rec_x + (int64_t)(n0 + i) * p.channels + ch) = val;
                unsigned long long m = anc[i];
                const int up = __popcll(m);
                uint4 r[4];
                r[3] = val;
                m &= ~(1ull << i);
#pragma unroll
                for (int t = 2; t >= 0; --t) {
                    const int a = m ? 63 - __clzll(m) : -1;
                    m &= ~(a >= 0 ? 1ull << a : 0ull);
                    r[t] = *reinterpret_cast<const uint4*>(
                        a >= 0 ? in + (int64_t)(n0 + a) * stride : p.state_in + ((int64_t)b * 3 + t + up - 1) * p.channels + ch);
                }
                float y[8] = {};
                float f[4][8];
#pragma unroll
                for (int t = 0; t < 4; ++t) unpack8(r[t], f[t]);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float4 w = *(reinterpret_cast<const float4*>(p.w) + ch + q);
                    y[q] = fmaf(w.w, f[3][q], fmaf(w.z, f[2][q], fmaf(w.y, f[1][q], w.x * f[0][q])));
                }
                float sq = 0.f;
#pragma unroll
                for (int q = 0; q < 8; q += 2) {
                    const float2 z = silu2(pack2(y[q], y[q + 1]));
                    y[q] = z.x;
                    y[q + 1] = z.y;
                    sq = fmaf(z.x, z.x, fmaf(z.y, z.y, sq));
                }
                // a k row's GK lanes are neighbours (whole warps run this loop)
#pragma unroll
                for (int o = GK / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                const float inv = !is_k ? 1.f : sq > 0.f ? rsqrtf(sq) : 0.f;
                // rounded to bf16, the operands' type, as after the convolution of a tail
                val = make_uint4(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv),
                                 pack_bf16(y[4] * inv, y[5] * inv), pack_bf16(y[6] * inv, y[7] * inv));
            }
            if (!act) continue;
            if (is_v) {
                *reinterpret_cast<uint4*>(vs + i * kRowsA + c) = val;
            } else {
                *reinterpret_cast<uint4*>(smem + at.kq + sw128_off16(is_k ? i : T + i, c, 2 * T)) = val;
                if (is_k) *reinterpret_cast<uint4*>(p.rec_k + ((int64_t)(n0 + i) * H + h) * DK + c) = val;
            }
        }
    }
    // ---- the products, 64 columns of S at a time
    bool ok = true;
#pragma unroll
    for (int x = 0; x < HALVES; ++x) {
        if (x > 0) ok = mbar_wait(bar + 8 * (x - 1), 0, abort_flag, p.err, kErrWait, p.diag, 0x61);   // the parts are consumed
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = (tid + e * kThreads) >> 4, c4 = tid & 15;
            const uint32_t o = sw128_off16(row, 4 * c4, kRowsA);
            float4 v = s[x][e];
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const float a = take_bf16(v.x), c = take_bf16(v.y), d = take_bf16(v.z), f = take_bf16(v.w);
                *reinterpret_cast<uint2*>(smem + at.s + part * kPartBytes + o) = make_uint2(pack_bf16(a, c), pack_bf16(d, f));
            }
        }
        fence_proxy_async_smem();
        ok = __syncthreads_and(ok);
        if (tid == 0 && ok) {
            tc_fence_after();
            const uint64_t kq = smem_desc_sw128(base + at.kq + x * region, 16, 1024);
            const uint64_t sd = smem_desc_sw128(base + at.s, 16, 1024);
            const uint32_t id_s = idesc_bf16_f32(kRowsA, 2 * T, false), id_g = idesc_bf16_f32(kRowsA, T, false);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                mma_bf16(tg, kq + 2 * ks, kq + 2 * ks, id_g, (x > 0 || ks > 0) ? 1u : 0u);
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    mma_bf16(tmem, sd + ((part * kPartBytes) >> 4) + 2 * ks, kq + 2 * ks, id_s, (x > 0 || part > 0 || ks > 0) ? 1u : 0u);
            mma_commit(bar + 8 * x);
        }
    }
    // ---- decays from the root, while the products run
    if (tid < kDraftNodes) {
        float g = 1.f;
        if (tid < n) {
            for (uint64_t m = anc[tid]; m; m &= m - 1) g *= al[__ffsll((long long)m) - 1];   // root first
            if (!(g >= kSmallDecay)) *small = 1;
        }
        G[tid] = g;
        rG[tid] = 1.f / g;
        if (tid >= n) be[tid] = 0.f;
    }
    ok = ok && mbar_wait(bar + 8 * (HALVES - 1), 0, abort_flag, p.err, kErrWait, p.diag, 0x62);
    ok = __syncthreads_and(ok);
    tc_fence_after();
    const int quarter = warp & 3, half = warp >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    if (ok) {
        // ---- C and E: lane l of the product holds k row l, or q row l - T; the two warps of a quarter take 16 columns in turn
        const int l = quarter * 32 + lane;
        const bool is_c = l < T, real = l < 2 * T && (is_c ? l : l - T) < n;
        const int i = is_c ? l : l - T;
        float* row = (is_c ? Cm : Em) + i * kLdc;
        const bool exact = *small != 0;
        uint64_t m = real ? anc[i] : 0;
        if (is_c) m &= ~(1ull << i);                 // C is strict
        const float scale = real ? (is_c ? be[i] : 1.f) : 0.f;
        for (int c0 = 16 * half; c0 < T; c0 += 32) {
            uint32_t g[16];
            tmem_ld16(lanes + 2 * T + c0, g);
            tmem_ld_wait();
            if (l >= 2 * T) continue;
#pragma unroll
            for (int c = 0; c < 16; c += 4) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = c0 + c + e;
                    float R = scale;
                    if (!exact && real) R *= G[i] * rG[j];
                    y[e] = (m >> j & 1) ? R * __uint_as_float(g[c + e]) : 0.f;
                }
                *reinterpret_cast<float4*>(row + c0 + c) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
    }
    __syncthreads();
    if (ok && *small != 0) {
        // some decay is small: the products down each path, node by node
        if (tid < 2 * T) {
            const bool is_c = tid < T;
            const int i = is_c ? tid : tid - T;
            float* row = (is_c ? Cm : Em) + i * kLdc;
            float R = 1.f;
            for (uint64_t m = i < n ? anc[i] : 0; m;) {
                const int j = 63 - __clzll((long long)m);
                m &= ~(1ull << j);
                row[j] *= R;
                R *= al[j];
            }
        }
        __syncthreads();
    }
    if (ok) {
        const int r = quarter * 32 + lane;           // row of S
        const int NB = T / 16;
        if (half == 0) {
            // ---- u
            for (int I = 0; I < NB; ++I) {
                uint32_t a[16];
                tmem_ld16(lanes + 16 * I, a);
                f2 acc[16] = {};
                for (int J = 0; J < I; ++J) {
                    f2 u[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) u[x] = pack2(U[(16 * J + 2 * x) * kRowsA + r], U[(16 * J + 2 * x + 1) * kRowsA + r]);
                    block16(acc, Cm + 16 * I * kLdc + 16 * J, u);
                }
                tmem_ld_wait();
                float u[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int node = 16 * I + i;
                    const float2 t = unpack2(acc[i]);
                    const float v = __bfloat162float(vs[node * kRowsA + r]);
                    const float x = be[node] * (v - G[node] * __uint_as_float(a[i])) - (t.x + t.y);
                    u[i] = node < n ? x : 0.f;       // a padding row holds anything
                }
#pragma unroll
                for (int i = 1; i < 16; ++i)
#pragma unroll
                    for (int j = 0; j < i; ++j) u[i] = fmaf(-Cm[(16 * I + i) * kLdc + 16 * I + j], u[j], u[i]);
#pragma unroll
                for (int i = 0; i < 16; ++i) U[(16 * I + i) * kRowsA + r] = u[i];
                named_bar_arrive(1 + I, kThreads);
                if (r < dv) {
                    float* rec = p.rec_u + ((int64_t)(n0 + 16 * I) * H + h) * dv + r;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (16 * I + i < n) rec[(int64_t)i * H * dv] = u[i];
                }
            }
        } else {
            // ---- outputs
            for (int I = 0; I < NB; ++I) {
                uint32_t a[16];
                tmem_ld16(lanes + T + 16 * I, a);
                f2 acc[16] = {};
                for (int J = 0; J <= I; ++J) {
                    if (J == I) named_bar_sync(1 + I, kThreads);
                    f2 u[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) u[x] = pack2(U[(16 * J + 2 * x) * kRowsA + r], U[(16 * J + 2 * x + 1) * kRowsA + r]);
                    block16(acc, Em + 16 * I * kLdc + 16 * J, u);
                }
                tmem_ld_wait();
                if (r < dv) {
                    __nv_bfloat16* out = p.out + ((int64_t)(n0 + 16 * I) * H + h) * dv + r;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 t = unpack2(acc[i]);
                        if (16 * I + i < n)
                            out[(int64_t)i * H * dv] = __float2bfloat16_rn(fmaf(G[16 * I + i], __uint_as_float(a[i]), t.x + t.y));
                    }
                }
            }
        }
    } else if (*abort_flag) {
        // what was issued completes before TMEM and shared memory are released
        volatile int never = 0;
        for (int x = 0; x < HALVES; ++x) mbar_wait(bar + 8 * x, 0, &never, p.err, kErrWait, nullptr, 0, 1000000000ull);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

template <int DK, bool CONV>
void launch(const DraftGdnParams& p, cudaStream_t s) {
    static unsigned long long configured = 0;    // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(draft_gdn_kernel<DK, CONV>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout(kDraftNodes, DK).bytes + 1024);
        configured |= 1ull << (dev & 63);
    }
    launch_pdl(draft_gdn_kernel<DK, CONV>, dim3(p.H, p.n_chars), dim3(kThreads), Layout((p.most + 15) / 16 * 16, DK).bytes + 1024, s, p);
}

}  // namespace

void launch_draft_gdn(const DraftGdnParams& p, cudaStream_t s) {
    if (p.dk == 64) p.w ? launch<64, true>(p, s) : launch<64, false>(p, s);
    else p.w ? launch<128, true>(p, s) : launch<128, false>(p, s);
}

}  // namespace kvm
