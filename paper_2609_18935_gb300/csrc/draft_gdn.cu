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
//  * S is fp32: 64 columns at a time (side by side where that costs no block an
//    SM, so that the second half is split while the first one's products run),
//    loaded as whole lines into registers while the inputs are staged, then split
//    into three bf16 parts of eight bits each (by truncation: two masks and two exact
//    differences; with rounding, whose conversions run at an eighth of that rate, this
//    phase of a block took 3 us against 1.8).  u enters the states of later steps, so
//    all of S's bits take part.
//  * C_ij = -beta_i R_ij (k_i . k_j) and E_ij = R_ij (q_i . k_j), 0 off the paths,
//    go to shared memory over the consumed parts of S, in three and two bf16 parts.
//  * The triangular solve and the outputs: a warp owns 16 rows of S and works
//    through the nodes 16 at a time, u_I = (1 - C_II)^-1 (rhs_I + sum_{J < I} C_IJ u_J),
//    o_I = G S q + sum_{J <= I} E_IJ u_J.  These are warp-wide products of 16 x 16 x
//    16 whose left operand is the previous product's accumulator, so they run on
//    mma.sync with u in registers: a round through TMEM and shared memory a block
//    would cost more than the product.  (With u in registers a row a thread and
//    the coefficients as broadcast loads, 16 bytes a lane, shared memory returned
//    a coefficient a clock and warp: 9 us at 64 nodes, against 3.1.)  The inverses
//    of the diagonal blocks are formed in fp32, a column a lane.
// What is not finite in C, E and the right-hand sides (a node's key, value or gate was
// not) counts as 0, as a coefficient of 0 off the paths would not hide it.
// R_ij = G_i / G_j while no G is small, else products down the path (a decay of 0
// is one).
//
// 32 characters of up to 64 nodes, 16 heads of 128 x 128, convolved: 30.7 us, 47 MB
// (1.5 TB/s).  Neither memory nor the tensor pipe bounds it (14 % and 11 % of their
// peaks): a block is a chain of short phases between barriers, each run once, and its
// warps wait for instructions and for one another.  One character, the chain alone: 6.1
// us of 16 nodes and 10.0 of 64, convolved 9.0 and 16.9.
#include <type_traits>

#include "draft_rows.cuh"
#include "kvm_internal.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace kvm {
namespace {

using namespace ptx;

constexpr int kThreads = 256;
constexpr int kRowsA = 128;                      // rows of an A operand
constexpr int kPartBytes = kRowsA * 128;         // 64 bf16 columns of S
constexpr int kLdc = kDraftNodes + 8;            // row pitch of C's and E's parts: fragments on all banks
constexpr int kLdv = kRowsA + 8;                 // row pitch of v
constexpr int kLdd = 24;                         // row pitch of the inverse diagonal blocks' parts
constexpr int kLdf = 20;                         // row pitch of the diagonal blocks in fp32
constexpr float kSmallDecay = 0x1p-40f;

// Shared memory for trees of up to T nodes (a multiple of 16).  [K; Q] comes first:
// as an A operand it is read up to row 127, past its own 2 T.
struct Layout {
    int kq, v, s, misc, w, bytes;
    // raw: bytes of a node's unconvolved inputs, or 0; wide: both halves of S side by side
    __host__ __device__ Layout(int T, int dk, int raw, bool wide) {
        const int diag = T / 16 * (16 * kLdf * 4 + 3 * 16 * kLdd * 2), tile = 2 * T * dk * 2;
        const int parts = 3 * kPartBytes * (wide ? dk / 64 : 1), x = (T + 3) * raw;
        kq = 0;
        v = (max_(tile, diag) + 1023) / 1024 * 1024;
        s = (v + T * kLdv * 2 + 1023) / 1024 * 1024;
        misc = (s + max_(parts, x) + 1023) / 1024 * 1024;
        w = misc + 2048;                         // the convolution's taps, 16 bytes a channel (raw: 2 bytes a channel)
        bytes = w + 8 * raw;
    }
    static __host__ __device__ int max_(int a, int b) { return a > b ? a : b; }
};
static_assert(5 * kDraftNodes * kLdc * 2 <= 3 * kPartBytes, "C and E take the place of S's parts");

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// The leading eight bits of a and b as a bf16 pair (a low); a and b keep the rest.
__device__ __forceinline__ uint32_t take_part(float& a, float& b) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    a -= __uint_as_float(x & 0xffff0000u);
    b -= __uint_as_float(y & 0xffff0000u);
    return __byte_perm(x, y, 0x7632);
}

// D (16 x 8, fp32) += A (16 x 16, bf16) B (16 x 8, bf16): lane l holds of D rows
// l / 4 and l / 4 + 8, columns 2 (l % 4) and the next; A's pairs are two such D
// side by side, B's are k rows of column l / 4.
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// What is not finite among x becomes 0, and bad true.
template <int N>
__device__ __forceinline__ void clear_not_finite(float (&x)[N], bool& bad) {
    f2 z = 0;                                    // two zeros, and a NaN where 0 x is one
#pragma unroll
    for (int e = 0; e < N; e += 2) z = fma2(pack2(x[e], x[e + 1]), 0, z);
    const float2 t = unpack2(z);
    if (t.x + t.y == 0.f) return;
    bad = true;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = fabsf(x[e]) < INFINITY ? x[e] : 0.f;
}

// Four 8 x 8 blocks of 16-bit elements, lane l giving row l % 8 of block l / 8: each
// lane gets two neighbours of row l / 4.
__device__ __forceinline__ void ldmatrix(uint32_t (&f)[2][2], uint32_t row) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(f[0][0]), "=r"(f[0][1]), "=r"(f[1][0]), "=r"(f[1][1]) : "r"(row) : "memory");
}
// 16 TMEM lanes x 16 columns, as two such D (to be waited for).
__device__ __forceinline__ void tmem_ld_16x16(uint32_t addr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
}
// d += lo, lo = 0
__device__ __forceinline__ void join(float (&d)[2][4], float (&lo)[2][4]) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            d[t][e] += lo[t][e];
            lo[t][e] = 0.f;
        }
}
// The first N of three parts of a 16 x 16 block, as A operands.
template <int N>
__device__ __forceinline__ void split(const float (&d)[2][4], uint32_t (&a)[N][4]) {
    float x[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][e] = d[t][e];
#pragma unroll
    for (int part = 0; part < N; ++part)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            a[part][2 * t] = take_part(x[t][0], x[t][1]);
            a[part][2 * t + 1] = take_part(x[t][2], x[t][3]);
        }
}
// d += (sum of a's parts) B^T, B a 16 x 16 block [column of d][k] in NB parts, the
// products below 2^-24 (or with two parts 2^-16) of the largest left out.  Small
// products are summed apart (lo): four chains of dependent products instead of one.
template <int NA, int NB>
__device__ __forceinline__ void block_mma(float (&d)[2][4], float (&lo)[2][4], const uint32_t (&a)[NA][4], const __nv_bfloat16* B,
                                          int pitch, int part_step) {
    constexpr int LAST = NB - 1;                 // parts i of a and j of B with i + j <= LAST
    const int lane = threadIdx.x & 31;
    const uint32_t b = smem_u32(B + ((lane >> 4) * 8 + (lane & 7)) * pitch + (lane & 8));
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        uint32_t f[2][2];                        // [columns 8 t ..][k 0 - 7, 8 - 15]
        ldmatrix(f, b + j * part_step * 2);
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (i + j <= LAST) mma16(i + j == 0 ? d[t] : lo[t], a[i], f[t][0], f[t][1]);
    }
}

// Place of channel e's taps in shared memory: lanes read octets of channels, 128
// bytes apart.
__device__ __forceinline__ int tap_slot(int e) { return (e & ~7) | ((e ^ e >> 3) & 7); }
// The convolution, SiLU and (norm) the scaling to unit length of one part of the
// staged raw rows [3 carried + nodes][pitch bytes], in gdn_conv_kernel's order of
// operations (so bit for bit what a tail's inputs become), for put(node, channel, eight
// outputs): eight channels a lane, their taps in registers, two nodes a thread at a
// time.  rows: per node the staged rows of its four taps, a byte each.
template <typename Put>
__device__ __forceinline__ void conv_part(const uint8_t* raw, int pitch, int dim, const float4* w, bool norm, int n, const uint32_t* rows,
                                          Put put) {
    constexpr int AHEAD = 2;
    const int per = dim <= 32 ? 4 : dim <= 64 ? 8 : 16;        // lanes a node; those past dim / 8 idle
    const int c = 8 * (threadIdx.x % per), first = threadIdx.x / per, step = kThreads / per;
    const bool act = c < dim;
    if (act) { raw += 2 * c; w += c; }
    f2 tap[4][4];                                              // [tap][channel pair]
    const int turn = act ? threadIdx.x % per & 7 : 0;          // the channels of an octet lie turned (tap_slot): neighbours on other banks
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float4 f = w[2 * e ^ turn], g = w[(2 * e + 1) ^ turn];
        tap[0][e] = pack2(f.x, g.x); tap[1][e] = pack2(f.y, g.y); tap[2][e] = pack2(f.z, g.z); tap[3][e] = pack2(f.w, g.w);
    }
    const int lead = (threadIdx.x & ~31) / per;                // the warp's first node: it leaves out what is past the last one
#pragma unroll 1
    for (int i0 = 0; lead + i0 < n; i0 += AHEAD * step) {
        const bool two = lead + i0 + step < n;                 // uniform per warp
        uint4 x[AHEAD][4];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (a > 0 && !two) break;
            const uint32_t r = rows[min(first + i0 + a * step, n - 1)];
#pragma unroll
            for (int t = 0; t < 4; ++t) x[a][t] = *reinterpret_cast<const uint4*>(raw + (r >> (8 * t) & 255) * pitch);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (a > 0 && !two) break;
            f2 acc[4] = {};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t* u = reinterpret_cast<const uint32_t*>(&x[a][t]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[e] = fma2(tap[t][e], pack2(__uint_as_float(u[e] << 16), __uint_as_float(u[e] & 0xffff0000u)), acc[e]);
            }
            float y[8], sq = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 v = silu2(acc[e]);
                y[2 * e] = v.x;
                y[2 * e + 1] = v.y;
            }
            if (norm) {                                        // whole warps run this
#pragma unroll
                for (int e = 0; e < 8; ++e) sq = fmaf(y[e], y[e], sq);
                for (int o = per / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                const float inv = sq > 0.f ? rsqrtf(sq) : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= inv;
            }
            // rounded to bf16, the operands' type, as after the convolution of a tail
            if (act && first + i0 + a * step < n)
                put(first + i0 + a * step, c, make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])));
        }
    }
}

template <int DK, bool CONV>
__global__ void __launch_bounds__(kThreads, 2) draft_gdn_kernel(const __grid_constant__ DraftGdnParams p) {
    constexpr int HALVES = DK / 64, GK = DK / 8;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const int b = p.order[blockIdx.y], h = blockIdx.x;
    const int n0 = p.cu[b], n = p.cu[b + 1] - n0;
    if (n <= 0) return;
    const int H = p.H, dv = p.dv, hk = H * DK;
    const int pitch = CONV ? (2 * DK + dv) * 2 : 0;
    const Layout at((p.most + 15) / 16 * 16, DK, pitch, p.wide);
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem);
    const int T = (n + 15) / 16 * 16, NB = T / 16;
    const uint32_t region = 2 * T * 128;             // bytes of 64 columns of [K; Q]
    uint64_t* anc = reinterpret_cast<uint64_t*>(smem + at.misc);           // [64]
    float* al = reinterpret_cast<float*>(smem + at.misc + 512);            // [64] each
    float* be = al + kDraftNodes;
    float* G = be + kDraftNodes;
    float* rG = G + kDraftNodes;
    const uint32_t bar = base + at.misc + 1536;                            // one barrier per half of S
    uint32_t* slot = reinterpret_cast<uint32_t*>(smem + at.misc + 1560);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + at.misc + 1564);
    int* small = reinterpret_cast<int*>(smem + at.misc + 1568);
    uint32_t* rows = reinterpret_cast<uint32_t*>(smem + at.misc + 1572);   // [64] staged rows of each node's taps
    constexpr int kPart = kDraftNodes * kLdc;        // elements of a part of C or E
    __nv_bfloat16* Cp = reinterpret_cast<__nv_bfloat16*>(smem + at.s);     // C: three parts, blocks left of the diagonal
    __nv_bfloat16* Ep = Cp + 3 * kPart;                                    // E: two
    float* Cd = reinterpret_cast<float*>(smem + at.kq);                    // C's diagonal blocks [NB][16][kLdf]
    __nv_bfloat16* Dp = reinterpret_cast<__nv_bfloat16*>(Cd + NB * 16 * kLdf);   // their inverses [NB][three parts][16][kLdd]
    __nv_bfloat16* vs = reinterpret_cast<__nv_bfloat16*>(smem + at.v);     // [T][kLdv]

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t cols = 32;                              // TMEM: S [K; Q]^T, then [K; Q] K^T
    while ((int)cols < 3 * T) cols *= 2;
    if (tid == 0) {
        *abort_flag = 0;
        *small = 0;
        for (int x = 0; x < 2; ++x) mbar_init(bar + 8 * x, 1);
        fence_mbar_init();
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc(smem_u32(slot), cols);
        tmem_relinquish();
    }
    grid_dependency_wait();
    grid_dependents_launch();

    // ---- loads: the inputs (asynchronously), S into registers, the nodes' words and gates
    {
        const __nv_bfloat16* kg = p.k + (int64_t)n0 * hk + h * DK;
        const __nv_bfloat16* qg = p.q + (int64_t)n0 * hk + h * DK;
        const __nv_bfloat16* vg = p.v + ((int64_t)n0 * H + h) * dv;
        if constexpr (CONV) {
            // raw rows q | k | v, three carried ones first, a warp a row (as bulk copies, three a row, they took 4K cycles to
            // issue at 64 nodes), and the taps in the same order
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int x = lane + 32 * u;
                if (x >= pitch / 16) break;
                const bool is_q = x < GK, is_v = x >= 2 * GK;
                const int c = 8 * (is_q ? x : is_v ? x - 2 * GK : x - GK);
                const __nv_bfloat16* src = (is_v ? vg : is_q ? qg : kg) + c;
                const int64_t stride = is_v ? H * dv : hk;
                const uint32_t dst = base + at.s + 16 * x;
                if (warp < 3)
                    cp_async16(dst + warp * pitch, p.state_in + ((int64_t)b * 3 + warp) * p.channels +
                                                       (is_q ? h * DK : is_v ? 2 * hk + h * dv : hk + h * DK) + c);
                for (int i = warp; i < n; i += kThreads / 32) cp_async16(dst + (3 + i) * pitch, src + i * stride);
            }
            for (int e = tid; e < 2 * DK + dv; e += kThreads)
                cp_async16(base + at.w + 16 * tap_slot(e),
                           p.w + (int64_t)(e < DK ? h * DK + e : e < 2 * DK ? hk + h * DK + e - DK : 2 * hk + h * dv + e - 2 * DK) * 4);
        } else {
            for (int e = tid; e < 2 * n * GK; e += kThreads) {
                const int row = e / GK, c = 8 * (e % GK);
                const bool is_k = row < n;
                const int i = is_k ? row : row - n;
                cp_async16(base + at.kq + sw128_off16(is_k ? i : T + i, c, 2 * T), (is_k ? kg : qg) + (int64_t)i * hk + c);
            }
            if ((tid & 15) * 8 < dv)
                for (int i = tid >> 4; i < n; i += kThreads / 16)
                    cp_async16(base + at.v + (i * kLdv + 8 * (tid & 15)) * 2, vg + (int64_t)i * H * dv + 8 * (tid & 15));
        }
    }
    const float* Sg = p.S + ((int64_t)b * H + h) * dv * DK;
    float4 s[HALVES][8];
    auto load_s = [&](auto half) {
        constexpr int x = decltype(half)::value;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = (tid + e * kThreads) >> 4, c4 = tid & 15;
            s[x][e] = row < dv ? *reinterpret_cast<const float4*>(Sg + (int64_t)row * DK + 64 * x + 4 * c4) : make_float4(0, 0, 0, 0);
        }
    };
    using First = std::integral_constant<int, 0>;
    using Last = std::integral_constant<int, HALVES - 1>;
    // the convolution needs the registers: there S comes after it, from L2
    if constexpr (CONV) {
        for (int e = tid * 32; e < dv * DK; e += kThreads * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(Sg + e));
    } else {
        load_s(First());
        if (HALVES > 1) load_s(Last());
    }
    if (tid < n) {
        const uint64_t own = p.anc[n0 + tid];
        anc[tid] = own;
        if constexpr (CONV) {
            // staged rows of the taps: 3 is the node, 2 its parent, .. and then the carried inputs from the last back
            uint64_t m = own;
            uint32_t r = 0;
#pragma unroll
            for (int t = 3; t >= 0; --t) {
                const int a = m ? 63 - __clzll((long long)m) : -1;
                m &= ~(a >= 0 ? 1ull << a : 0ull);
                r |= (uint32_t)(a >= 0 ? 3 + a : t + __popcll(own) - 1) << (8 * t);
            }
            rows[tid] = r;
        }
        const float a = p.alpha[(int64_t)(n0 + tid) * H + h];
        al[tid] = a;
        be[tid] = p.beta[(int64_t)(n0 + tid) * H + h];
        p.rec_a[(int64_t)(n0 + tid) * H + h] = a;
    }
    cp_async_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot;
    const uint32_t tg = tmem + 2 * T;
    bool ok = true;

    if constexpr (CONV) {
        const uint8_t* raw = smem + at.s;
#pragma unroll
        for (int u = 0; u < 2; ++u) {                // what a commit carries on
            const int x = lane + 32 * u;
            if (x >= pitch / 16) break;
            __nv_bfloat16* rec = p.rec_x + (int64_t)n0 * p.channels +
                                 (x < GK ? h * DK + 8 * x : x < 2 * GK ? hk + h * DK + 8 * (x - GK) : 2 * hk + h * dv + 8 * (x - 2 * GK));
            for (int i = warp; i < n; i += kThreads / 32)
                *reinterpret_cast<uint4*>(rec + (int64_t)i * p.channels) = *reinterpret_cast<const uint4*>(raw + (3 + i) * pitch + 16 * x);
        }
        const float4* w = reinterpret_cast<const float4*>(smem + at.w);
#pragma unroll 1
        for (int part = 0; part < 3; ++part)         // q, k, v: one copy of the code
            conv_part(raw + 2 * DK * part, pitch, part == 2 ? dv : DK, w + DK * part, part == 1, n, rows, [&](int i, int c, uint4 y) {
                uint8_t* dst = part == 2 ? smem + at.v + (i * kLdv + c) * 2 : smem + at.kq + sw128_off16(part == 1 ? i : T + i, c, 2 * T);
                *reinterpret_cast<uint4*>(dst) = y;
            });
        load_s(First());
        if (HALVES > 1) load_s(Last());
        __syncthreads();                             // the raw rows make room for S's parts
    }
    // ---- the products, 64 columns of S at a time
#pragma unroll
    for (int x = 0; x < HALVES; ++x) {
        if (x > 0 && !p.wide) ok = ok && mbar_wait(bar + 8 * (x - 1), 0, abort_flag, p.err, kErrWait, p.diag, 0x61);   // the parts are consumed
        const int s0 = at.s + (p.wide ? 3 * x * kPartBytes : 0);
        uint8_t* dst = smem + s0 + sw128_off16(tid >> 4, 4 * (tid & 15), kRowsA);       // and every 16 rows on (two of the swizzle's periods)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float4 v = s[x][e];
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const uint32_t lo = take_part(v.x, v.y), hi = take_part(v.z, v.w);
                *reinterpret_cast<uint2*>(dst + part * kPartBytes + e * (16 * 128)) = make_uint2(lo, hi);
            }
        }
        fence_proxy_async_smem();
        ok = __syncthreads_and(ok);
        if (tid == 0 && ok) {
            tc_fence_after();
            const uint64_t kq = smem_desc_sw128(base + at.kq + x * region, 16, 1024);
            const uint64_t sd = smem_desc_sw128(base + s0, 16, 1024);
            const uint32_t id_s = idesc_bf16_f32(kRowsA, 2 * T, false), id_g = idesc_bf16_f32(kRowsA, T, false);
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    mma_bf16(tmem, sd + ((part * kPartBytes) >> 4) + 2 * ks, kq + 2 * ks, id_s, (x > 0 || part > 0 || ks > 0) ? 1u : 0u);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                mma_bf16(tg, kq + 2 * ks, kq + 2 * ks, id_g, (x > 0 || ks > 0) ? 1u : 0u);
            mma_commit(bar + 8 * x);
        }
    }
    // ---- while the products run: the keys' record, and the decays from the root
    for (int e = tid; e < n * GK; e += kThreads) {
        const int i = e / GK, c = 8 * (e % GK);
        uint4 key = *reinterpret_cast<const uint4*>(smem + at.kq + sw128_off16(i, c, 2 * T));
        kvm::clear_not_finite(key);                  // its u is 0, and 0 times it is to stay 0 in a commit (reported with E_ii)
        *reinterpret_cast<uint4*>(p.rec_k + ((int64_t)(n0 + i) * H + h) * DK + c) = key;
    }
    if (warp == 1) {
        // products up the tree by doubling: g holds the nodes from i up to before `up`
        float g[2];
        int up[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int i = lane + 32 * x;
            const uint64_t m = i < n ? anc[i] & ~(1ull << i) : 0;
            g[x] = i < n ? al[i] : 1.f;
            up[x] = m ? 63 - __clzll((long long)m) : -1;
        }
        while (__any_sync(0xffffffffu, up[0] >= 0 || up[1] >= 0)) {
            float t[2];
            int w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int from = up[x] & 31;
                const float a = __shfl_sync(0xffffffffu, g[0], from), c = __shfl_sync(0xffffffffu, g[1], from);
                const int d = __shfl_sync(0xffffffffu, up[0], from), e = __shfl_sync(0xffffffffu, up[1], from);
                t[x] = up[x] < 0 ? 1.f : up[x] < 32 ? a : c;
                w[x] = up[x] < 0 ? -1 : up[x] < 32 ? d : e;
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                g[x] *= t[x];
                up[x] = w[x];
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int i = lane + 32 * x;
            if (i < n && fabsf(g[x]) < kSmallDecay) *small = 1;
            G[i] = g[x];
            rG[i] = 1.f / g[x];
            if (i >= n) be[i] = 0.f;
        }
    }
    ok = ok && mbar_wait(bar + 8 * (HALVES - 1), 0, abort_flag, p.err, kErrWait, p.diag, 0x62);
    ok = __syncthreads_and(ok);
    tc_fence_after();
    bool bad = false;                                // something was not finite
    if (ok) {
        // ---- C and E: lane l of the product holds k row l, or q row l - T; the two warps of a quarter take 16 columns in turn
        const int l = (warp & 3) * 32 + lane;
        const bool is_c = l < T, real = l < 2 * T && (is_c ? l : l - T) < n;
        const int i = is_c ? l : l - T, I = i / 16;
        const bool exact = *small != 0;
        uint64_t m = real ? anc[i] : 0;
        if (is_c) m &= ~(1ull << i);                 // C is strict
        const float scale = real ? (is_c ? -be[i] : 1.f) * (exact ? 1.f : G[i]) : 0.f;
        for (int J = warp >> 2; J < NB; J += 2) {
            uint32_t g[16];
            __syncwarp();                            // lanes part ways below, a load from TMEM is the warp's
            tmem_ld16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + 2 * T + 16 * J, g);
            tmem_ld_wait();
            if (l >= 2 * T || J > I) continue;
            const uint32_t bits = (uint32_t)(m >> (16 * J)) & 0xffffu;
            float y[16];
            if (!exact) {
#pragma unroll
                for (int c = 0; c < 16; ++c)
                    y[c] = (bits >> c & 1) ? scale * rG[16 * J + c] * __uint_as_float(g[c]) : 0.f;
            } else {
                // some decay is small: the product down the path, which reaches this block's nodes from the largest down
                float R = scale;
                for (uint64_t a = real ? anc[i] >> (16 * J + 15) >> 1 : 0; a;) {
                    const int j = 63 - __clzll((long long)a);
                    a &= ~(1ull << j);
                    R *= al[16 * J + 16 + j];
                }
#pragma unroll
                for (int c = 15; c >= 0; --c) {
                    y[c] = (bits >> c & 1) ? R * __uint_as_float(g[c]) : 0.f;
                    if (real && (anc[i] >> (16 * J + c) & 1)) R *= al[16 * J + c];
                }
            }
            clear_not_finite(y, bad);
            if (is_c && J == I) {
                float* row = Cd + (I * 16 + (i & 15)) * kLdf;
#pragma unroll
                for (int c = 0; c < 16; c += 4) *reinterpret_cast<float4*>(row + c) = make_float4(y[c], y[c + 1], y[c + 2], y[c + 3]);
            } else {
                __nv_bfloat16* row = (is_c ? Cp : Ep) + i * kLdc + 16 * J;
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    if (part == 2 && !is_c) break;
                    uint32_t w[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) w[c] = take_part(y[2 * c], y[2 * c + 1]);
                    uint4* dst = reinterpret_cast<uint4*>(row + part * kPart);
                    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
        }
    }
    __syncthreads();
    if (ok && warp < NB) {
        // ---- (1 - C_II)^-1, block `warp`: column `lane` by forward substitution
        const int j = lane & 15;
        const float* C = Cd + warp * 16 * kLdf;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float t[2] = {i == j ? 1.f : 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < i; m += 4) {
                const float4 c = *reinterpret_cast<const float4*>(C + i * kLdf + m);    // 0 on and right of the diagonal
                t[0] = fmaf(c.x, x[m], t[0]);
                if (m + 1 < i) t[1] = fmaf(c.y, x[m + 1], t[1]);
                if (m + 2 < i) t[0] = fmaf(c.z, x[m + 2], t[0]);
                if (m + 3 < i) t[1] = fmaf(c.w, x[m + 3], t[1]);
            }
            x[i] = t[0] + t[1];
        }
        if (lane < 16) {
            __nv_bfloat16* D = Dp + warp * 3 * 16 * kLdd + j;
#pragma unroll
            for (int i = 0; i < 16; i += 2)
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    const uint32_t w = take_part(x[i], x[i + 1]);
                    D[(part * 16 + i) * kLdd] = __ushort_as_bfloat16((unsigned short)w);
                    D[(part * 16 + i + 1) * kLdd] = __ushort_as_bfloat16((unsigned short)(w >> 16));
                }
        }
    }
    __syncthreads();
    if (ok) {
        // ---- u and the outputs: this warp's rows of S are TMEM lanes 32 (warp % 4) + 16 (warp / 4) ..
        const int r0 = (warp & 3) * 32 + (warp >> 2) * 16;
        const uint32_t lanes = tmem + ((uint32_t)r0 << 16);
        const int row = r0 + (lane >> 2), col = 2 * (lane & 3);
        uint32_t u[4][3][4];                         // the parts of each block's u
        uint32_t xa[8], oa[8];                       // S k and S q of the next 16 nodes
        tmem_ld_16x16(lanes, xa);
        tmem_ld_16x16(lanes + T, oa);
#pragma unroll
        for (int I = 0; I < 4; ++I) {
            if (I >= NB) break;
            float x[2][4], o[2][4], lo[2][4] = {};
            tmem_ld_wait();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int node = 16 * I + 8 * t + col + (e & 1), r = row + 8 * (e >> 1);
                    const float v = __bfloat162float(vs[node * kLdv + r]), gn = G[node];
                    const float sk = __uint_as_float(xa[4 * t + e]), sq = __uint_as_float(oa[4 * t + e]);
                    x[t][e] = node < n && r < dv ? be[node] * (v - gn * sk) : 0.f;       // padding holds anything
                    o[t][e] = gn * sq;
                }
            clear_not_finite(x[0], bad);
            clear_not_finite(x[1], bad);
            __syncwarp();                            // the loads and products below are the warp's
            if (I + 1 < NB) {
                tmem_ld_16x16(lanes + 16 * (I + 1), xa);
                tmem_ld_16x16(lanes + T + 16 * (I + 1), oa);
            }
#pragma unroll
            for (int J = 0; J < I; ++J) block_mma<3, 3>(x, lo, u[J], Cp + 16 * I * kLdc + 16 * J, kLdc, kPart);
            join(x, lo);
            split(x, u[I]);
            float y[2][4] = {};
            block_mma<3, 3>(y, lo, u[I], Dp + I * 3 * 16 * kLdd, kLdd, 16 * kLdd);
            join(y, lo);
            split(y, u[I]);
#pragma unroll
            for (int J = 0; J <= I; ++J) {
                const uint32_t (&a)[2][4] = *reinterpret_cast<const uint32_t (*)[2][4]>(&u[J]);
                block_mma<2, 2>(o, lo, a, Ep + 16 * I * kLdc + 16 * J, kLdc, kPart);
            }
            join(o, lo);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int node = 16 * I + 8 * t + col + (e & 1), r = row + 8 * (e >> 1);
                    vs[node * kLdv + r] = __float2bfloat16_rn(o[t][e]);                 // in v's place, read by this lane alone
                    if (node < n && r < dv) p.rec_u[((int64_t)(n0 + node) * H + h) * dv + r] = y[t][e];
                }
            __syncwarp();
        }
        if (bad) atomicOr(p.err, kErrValue);
    } else if (*abort_flag) {
        // what was issued completes before TMEM and shared memory are released
        volatile int never = 0;
        for (int x = 0; x < HALVES; ++x) mbar_wait(bar + 8 * x, 0, &never, p.err, kErrWait, nullptr, 0, 1000000000ull);
    }
    tc_fence_before();
    __syncthreads();
    if (ok) {
        const int c = 8 * (tid & 15);
        if (c < dv)
            for (int i = tid >> 4; i < n; i += kThreads / 16)
                *reinterpret_cast<uint4*>(p.out + ((int64_t)(n0 + i) * H + h) * dv + c) = *reinterpret_cast<const uint4*>(vs + i * kLdv + c);
    }
    if (warp == 0) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, cols);
    }
}

template <int DK, bool CONV>
void launch(const DraftGdnParams& p, cudaStream_t s) {
    const int pitch = CONV ? (2 * DK + p.dv) * 2 : 0;
    static unsigned long long configured = 0;    // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(draft_gdn_kernel<DK, CONV>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             Layout(kDraftNodes, DK, CONV ? (2 * DK + 128) * 2 : 0, true).bytes + 1024);
        configured |= 1ull << (dev & 63);
    }
    launch_pdl(draft_gdn_kernel<DK, CONV>, dim3(p.H, p.n_chars), dim3(kThreads), Layout((p.most + 15) / 16 * 16, DK, pitch, p.wide).bytes + 1024, s, p);
}

}  // namespace

void launch_draft_gdn(const DraftGdnParams& p, cudaStream_t s) {
    if (p.dk == 64) p.w ? launch<64, true>(p, s) : launch<64, false>(p, s);
    else p.w ? launch<128, true>(p, s) : launch<128, false>(p, s);
}

}  // namespace kvm
