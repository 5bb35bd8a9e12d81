// The verdict over a tree of drafted tokens (kvm_draft_verify): which path the
// target's probabilities accept, and the token that follows it.
//
// The children of a node are guesses drawn one after another from the draft's
// row q after that node; p is the target's.  After j failed guesses what is left
// of p is w_j = max(p - c_j q, 0) up to its sum Z_j (c_0 = 0, Z_0 = 1; c_1 = 1,
// c_{j+1} = c_j + Z_j: taking q once more out of w_j / Z_j is taking Z_j q more out
// of p, and where a residual has reached 0 it stays there).  Guess t is accepted
// where u q(t) Z_j < w_j(t); where all fail the next token is drawn from w_j by
// inverse distribution, the first x at which the running sum passes u_next Z_j.
// The path and the next token are then distributed as the target's own samples.
//
// Every node's p(t) and q(t) lie in its parent's rows, so one round of loads
// fetches them for the whole tree, and the walk reads a row only where a guess
// failed and for the last draw.  A row's pass is spread over a cluster of blocks,
// and its warps' sums meet in distributed shared memory.
//
// Sums decide between neighbouring tokens, so they are carried in pairs of fp32
// (the error-free sum and product; Dekker, "A floating-point technique for
// extending the available precision", 1971) and joined in 64 bits: about 2^-46
// relative, where a sum in 32 bits would move the draw by many tokens of a large
// vocabulary, and the 64-bit pipe (two results a cycle and SM) would bound the pass.
#include "kvm_internal.cuh"
#include "sm100_ptx.cuh"

namespace kvm {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

// hi + lo
struct Pair {
    float hi, lo;
};

__device__ __forceinline__ float probability(float x) {       // what is not a finite positive number counts as 0
    return x > 0.f && x <= 3.402823466e38f ? x : 0.f;
}

// max(p - c q, 0)
__device__ __forceinline__ Pair weight(float p, float q, float ch, float cl) {
    p = probability(p);
    q = probability(q);
    const float m = -ch * q, e = fmaf(-ch, q, -m);             // -c q = m + e - cl q
    const float s = p + m;
    const float bv = s - p, av = s - bv;
    const float lo = ((p - av) + (m - bv)) + fmaf(-cl, q, e);
    return s + lo > 0.f ? Pair{s, lo} : Pair{0.f, 0.f};
}

__device__ __forceinline__ void add(Pair& a, const Pair& x) {
    const float s = a.hi + x.hi;
    const float bv = s - a.hi, av = s - bv;
    a.lo += ((a.hi - av) + (x.hi - bv)) + x.lo;
    a.hi = s;
}

// Four neighbouring values of a row from virtual place y (a multiple of 4): place
// y holds element y - m, so that places on the vector grid lie on it in memory too.
template <typename T>
__device__ __forceinline__ void load4(const T* row, int y, int m, int end, float* x) {
    if (y >= m && y + 4 <= end) {
        if constexpr (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(row + (y - m));
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(row + (y - m));
            const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x));
            const float2 c = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
            x[0] = a.x; x[1] = a.y; x[2] = c.x; x[3] = c.y;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = y + e >= m && y + e < end ? (float)row[y + e - m] : 0.f;
    }
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

__device__ __forceinline__ double ld_cluster(const double* mine, uint32_t rank) {
    uint32_t addr;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T>
__global__ void __launch_bounds__(kThreads) draft_verify_kernel(const __grid_constant__ DraftVerifyParams p) {
    __shared__ double sums[2][kWarps];               // each warp's sum of its range, two passes deep
    __shared__ float pt[kDraftNodes], qt[kDraftNodes], us[kDraftNodes];
    __shared__ int par[kDraftNodes], path[kDraftNodes];
    uint32_t rank, blocks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.y;
    const int n0 = p.cu[b], n = p.cu[b + 1] - n0;
    const int V = p.vocab;
    const T* target = static_cast<const T*>(p.target);
    const T* draft = static_cast<const T*>(p.draft);
    grid_dependency_wait();
    grid_dependents_launch();
    if (n <= 0) {                                    // uniform over the cluster
        if (rank == 0 && tid == 0) { p.count[b] = 0; p.next[b] = -1; }
        return;
    }
    if (tid < n) {
        const unsigned long long up = p.anc[n0 + tid] & ~(1ull << tid);
        const int pa = up ? 63 - __clzll(up) : -1;
        par[tid] = pa;
        us[tid] = p.u[n0 + tid];
        float x = 0.f, y = 0.f;
        if (pa >= 0) {
            const int t = p.tokens[n0 + tid];
            if (t >= 0 && t < V) {
                x = (float)target[(int64_t)(n0 + pa) * V + t];
                y = (float)draft[(int64_t)(n0 + pa) * V + t];
            } else {
                atomicOr(p.err, kErrBounds);         // such a guess is not accepted
            }
        }
        pt[tid] = probability(x);
        qt[tid] = probability(y);
    }
    __syncthreads();

    const int gw = rank * kWarps + warp, n_gw = blocks * kWarps;
    int cur = 0, count = 1, pass = 0;
    double c = 0.0, Z = 1.0;
    if (tid == 0) path[0] = 0;
    // this warp's part of the current row, and the sum over all of max(p - c q, 0)
    int m = 0, end = 0, per = 0;
    const T *rp = nullptr, *rq = nullptr;
    auto row_sum = [&]() {
        const float ch = (float)c, cl = (float)(c - (double)ch);
        Pair acc{0.f, 0.f};
        const int y1 = min(end, (gw + 1) * per);
#pragma unroll 4
        for (int y = gw * per + 4 * lane; y < y1; y += 128) {
            float a[4], d[4];
            load4(rp, y, m, end, a);
            load4(rq, y, m, end, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) add(acc, weight(a[e], d[e], ch, cl));
        }
        const double mine = warp_sum((double)acc.hi + (double)acc.lo);
        if (lane == 0) sums[pass & 1][warp] = mine;
        cluster_sync();
        double z = 0.0;
        for (int g = lane; g < n_gw; g += 32) z += ld_cluster(&sums[pass & 1][g % kWarps], g / kWarps);
        ++pass;
        return warp_sum(z);                          // the same order in every warp
    };
    for (;;) {
        const int64_t at = (int64_t)(n0 + cur) * V;
        m = (int)(at & 3);
        end = m + V;
        per = ((end + n_gw - 1) / n_gw + 127) / 128 * 128;
        rp = target + at;
        rq = draft + at;
        c = 0.0;
        Z = 1.0;
        int taken = -1;
        for (int i = cur + 1; i < n; ++i) {
            if (par[i] != cur) continue;
            const double q = qt[i], w = (double)pt[i] - c * q;
            if ((double)us[i] * q * Z < (w > 0.0 ? w : 0.0)) { taken = i; break; }
            if (Z == 0.0) break;                     // nothing is left of p: no other guess can be accepted
            c = c == 0.0 ? 1.0 : c + Z;
            Z = row_sum();
        }
        if (taken < 0) break;
        cur = taken;
        if (tid == 0) path[count] = cur;
        ++count;
    }
    // ---- the next token, from what is left of the last node's row (all of it where nothing is)
    if (c == 0.0 || Z == 0.0) {
        c = 0.0;
        Z = row_sum();
    }
    const double T0 = (double)p.u_next[b] * Z;
    const double* last = sums[(pass - 1) & 1];
    // the last warp range with something in it whose running sum before it is <= T0
    int found = -1;
    double before = 0.0, base = 0.0;
    for (int g0 = 0; g0 < n_gw; g0 += 32) {
        const int g = g0 + lane;
        const double x = g < n_gw ? ld_cluster(last + g % kWarps, g / kWarps) : 0.0;
        double inc = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double t = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += t;
        }
        const double pre = base + (inc - x);
        const unsigned hit = __ballot_sync(0xffffffffu, x > 0.0 && pre <= T0);
        if (hit) {
            const int l = 31 - __clz(hit);
            found = g0 + l;
            before = __shfl_sync(0xffffffffu, pre, l);
        }
        base += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (found == gw) {
        const float ch = (float)c, cl = (float)(c - (double)ch);
        const int y1 = min(end, (gw + 1) * per);
        int best = -1;
        for (int y0 = gw * per; y0 < y1; y0 += 128) {
            const int y = y0 + 4 * lane;
            float a[4] = {}, d[4] = {};
            if (y < y1) {
                load4(rp, y, m, end, a);
                load4(rq, y, m, end, d);
            }
            double w[4], x = 0.0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Pair v = weight(a[e], d[e], ch, cl);
                w[e] = (double)v.hi + (double)v.lo;
                x += w[e];
            }
            double inc = x;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += t;
            }
            double pre = before + (inc - x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (w[e] > 0.0 && pre <= T0) best = y + e - m;
                pre += w[e];
            }
            before += __shfl_sync(0xffffffffu, inc, 31);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (lane == 0) p.next[b] = best;
    }
    if (rank == 0) {
        if (found < 0 && tid == 0) p.next[b] = -1;   // the row holds no positive number
        __syncthreads();
        if (tid < n) p.path[n0 + tid] = tid < count ? path[tid] : -1;
        if (tid == 0) p.count[b] = count;
    }
    cluster_sync();                                  // no block leaves while another may read its sums
}

}  // namespace

void launch_draft_verify(const DraftVerifyParams& p, bool bf16, int num_sms, cudaStream_t s) {
    int blocks = 1;
    while (blocks < kMaxCluster && blocks * kThreads * 8 < p.vocab && 2 * blocks * p.n_chars <= 2 * num_sms) blocks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, p.n_chars);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = blocks;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (bf16) cudaLaunchKernelEx(&cfg, draft_verify_kernel<__nv_bfloat16>, p);
    else cudaLaunchKernelEx(&cfg, draft_verify_kernel<float>, p);
}

}  // namespace kvm
