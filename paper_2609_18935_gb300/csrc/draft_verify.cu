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
// and its warps' sums meet in distributed shared memory.  Passes depend on one
// another, about 2 us each, so a verdict takes as long as its longest walk: 7 us over
// one tree of 16 nodes and 50001 tokens, 30 us over 32 trees of up to 24 and 131072.
//
// Sums decide between neighbouring tokens, so they are carried in pairs of fp32
// (the error-free sum and product; Dekker, "A floating-point technique for
// extending the available precision", 1971): about 2^-46
// relative, where a sum in 32 bits would move the draw by many tokens of a large
// vocabulary, and the 64-bit pipe gives two results a cycle and SM: with the few
// scalars of the walk alone in 64 bits, in every thread, a verdict took twice as long.
#include <type_traits>

#include "kvm_internal.cuh"
#include "packed_f32.cuh"
#include "sm100_ptx.cuh"

namespace kvm {
namespace {

constexpr int kMaxCluster = 16;              // 8 is what every launch may ask for, 16 a kernel that opts in

// hi + lo
struct Pair {
    float hi, lo;
};
// Two of them side by side (packed fp32).
struct Pairs {
    f2 hi, lo;
};

__device__ __forceinline__ float probability(float x) {       // what is not a finite positive number counts as 0
    return __float_as_uint(x) < 0x7f800000u ? x : 0.f;
}

// w where t > 0, else 0
__device__ __forceinline__ Pairs where_positive(f2 hi, f2 lo) {
    const float2 t = unpack2(add2(hi, lo)), x = unpack2(hi), y = unpack2(lo);
    return {pack2(t.x > 0.f ? x.x : 0.f, t.y > 0.f ? x.y : 0.f), pack2(t.x > 0.f ? y.x : 0.f, t.y > 0.f ? y.y : 0.f)};
}
// max(p - q, 0) of two elements: p may be anything (0 for what is no probability), q is one
__device__ __forceinline__ Pairs weights(f2 p, f2 q) {
    const f2 s = sub2(p, q), bv = sub2(s, p), av = sub2(s, bv);
    return where_positive(s, sub2(sub2(p, av), add2(q, bv)));
}
// max(p - c q, 0), c = ch + cl
__device__ __forceinline__ Pairs weights(f2 p, f2 q, f2 ch, f2 nch, f2 ncl) {
    const f2 m = mul2(nch, q), e = fma2(ch, q, m);             // -c q = m - e + ncl q
    const f2 s = add2(p, m);
    const f2 bv = sub2(s, p), av = sub2(s, bv);
    return where_positive(s, fma2(ncl, q, sub2(add2(sub2(p, av), sub2(m, bv)), e)));
}

__device__ __forceinline__ void add(Pairs& a, const Pairs& x) {
    const f2 s = add2(a.hi, x.hi);
    const f2 bv = sub2(s, a.hi), av = sub2(s, bv);
    a.lo = add2(a.lo, add2(add2(sub2(a.hi, av), sub2(x.hi, bv)), x.lo));
    a.hi = s;
}
__device__ __forceinline__ Pair add(Pair a, Pair x) {
    const float s = a.hi + x.hi;
    const float bv = s - a.hi, av = s - bv;
    const float lo = ((a.hi - av) + (x.hi - bv)) + (a.lo + x.lo);
    const float hi = s + lo;                                   // kept normalised: lo below an ulp of hi
    return {hi, lo - (hi - s)};
}
__device__ __forceinline__ Pair sub(Pair a, Pair x) { return add(a, {-x.hi, -x.lo}); }
__device__ __forceinline__ Pair mul(Pair a, float x) {
    const float h = a.hi * x, l = fmaf(a.hi, x, -h) + a.lo * x;
    const float hi = h + l;
    return {hi, l - (hi - h)};
}
__device__ __forceinline__ Pair mul(Pair a, Pair x) {
    const float h = a.hi * x.hi, l = fmaf(a.hi, x.hi, -h) + (a.hi * x.lo + a.lo * x.hi);
    const float hi = h + l;
    return {hi, l - (hi - h)};
}
__device__ __forceinline__ bool positive(Pair a) { return a.hi > 0.f; }          // of a normalised one
__device__ __forceinline__ bool less(Pair a, Pair x) { return positive(sub(x, a)); }
__device__ __forceinline__ Pair shuffle_xor(Pair a, int o) {
    return {__shfl_xor_sync(0xffffffffu, a.hi, o), __shfl_xor_sync(0xffffffffu, a.lo, o)};
}
// The sum over each N neighbouring lanes (N a power of two), in the same bits in every
// one of them: a sum of two does not depend on their order.
template <int N>
__device__ __forceinline__ Pair lane_sum(Pair a) {
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) a = add(a, shuffle_xor(a, o));
    return a;
}

// Four neighbouring values of a row from virtual place y (a multiple of 4): place y holds element y - m, so that places on the vector grid lie
// on it in memory too.
template <typename T>
__device__ __forceinline__ void load4(const T* row, int y, int m, int end, float (&x)[4]) {
    if (y >= m && y + 4 <= end) {
        if constexpr (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(row + (y - m));
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(row + (y - m));
            x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
            x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = y + e >= m && y + e < end ? (float)row[y + e - m] : 0.f;
    }
}
__device__ __forceinline__ void probabilities(float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = probability(x[e]);
}

// Writes v over the neighbour's copy of *mine, in block `rank` of the cluster, and
// counts its eight bytes in at that block's copy of the barrier.
__device__ __forceinline__ void st_cluster(const Pair* mine, uint32_t bar, uint32_t rank, Pair v) {
    uint32_t addr, at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(ptx::smem_u32(mine)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(bar), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                 ::"r"(addr), "f"(v.hi), "f"(v.lo), "r"(at) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) draft_verify_kernel(const __grid_constant__ DraftVerifyParams p) {
    constexpr int kWarps = THREADS / 32;
    __shared__ Pair sums[kWarps];                    // this block's warps' sums of their ranges
    __shared__ Pair parts[2][kMaxCluster];           // every block's sum, two passes deep
    __shared__ __align__(8) uint64_t arrived[2];     // and their barriers: a phase is all blocks' sums of a pass
    __shared__ int abort_word;
    __shared__ float pt[kDraftNodes], qt[kDraftNodes], us[kDraftNodes];
    __shared__ int path[kDraftNodes];
    __shared__ unsigned long long kids[kDraftNodes];               // each node's children
    uint32_t rank, blocks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.y;
    const int n0 = p.cu[b], n = p.cu[b + 1] - n0;
    const int V = p.vocab;
    const T* target = static_cast<const T*>(p.target);
    const T* draft = static_cast<const T*>(p.draft);
    volatile int* abort_flag = &abort_word;
    const uint32_t bar = ptx::smem_u32(arrived);
    if (tid == 0) {
        *abort_flag = 0;
        ptx::mbar_init(bar, 1);
        ptx::mbar_init(bar + 8, 1);
        ptx::fence_mbar_init();
    }
    if (tid < kDraftNodes) kids[tid] = 0;
    __syncthreads();
    if (blocks > 1) {                                // the neighbours' barriers stand before the first sum arrives
        cluster_arrive();
        cluster_wait();
    }
    grid_dependency_wait();
    grid_dependents_launch();
    if (n <= 0) {                                    // uniform over the cluster
        if (rank == 0 && tid == 0) { p.count[b] = 0; p.next[b] = -1; }
        return;
    }
    const float u_next = p.u_next[b];
    if (tid < n) {
        const unsigned long long up = p.anc[n0 + tid] & ~(1ull << tid);
        const int t = p.tokens[n0 + tid];
        const int pa = up ? 63 - __clzll(up) : -1;
        if (pa >= 0) atomicOr(kids + pa, 1ull << tid);
        us[tid] = p.u[n0 + tid];
        float x = 0.f, y = 0.f;
        if (pa >= 0) {
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
    Pair c{0.f, 0.f}, Z{1.f, 0.f};
    if (tid == 0) path[0] = 0;
    // this warp's part of the current row, and the sum over all of max(p - c q, 0)
    int m = 0, end = 0, per = 0;
    const T *rp = nullptr, *rq = nullptr;
    bool lost = false;
    f2 ch2 = 0, nch2 = 0, ncl2 = 0;
    auto set_c = [&]() {
        ch2 = pack2(c.hi, c.hi);
        nch2 = pack2(-c.hi, -c.hi);
        ncl2 = pack2(-c.lo, -c.lo);
    };
    // This thread's sum of w over the row: c is 0 (q is not read), 1 (no rounding in c q)
    // or another number.  Its instructions bound a pass over a large vocabulary: with
    // the last form for all three 32 trees over 131072 tokens took 31.9 us against 29.9.
    auto thread_sum = [&](auto kind) {
        constexpr int C = decltype(kind)::value;
        Pairs acc{0, 0};                             // four zeros
        const int y1 = min(end, (gw + 1) * per);
#pragma unroll 4
        for (int y = gw * per + 4 * lane; y < y1; y += 128) {
            float a[4], d[4];
            load4(rp, y, m, end, a);
            if constexpr (C == 0) {
                probabilities(a);
                add(acc, {pack2(a[0], a[1]), 0});
                add(acc, {pack2(a[2], a[3]), 0});
                continue;
            }
            load4(rq, y, m, end, d);
            probabilities(d);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const f2 x = pack2(a[e], a[e + 1]), z = pack2(d[e], d[e + 1]);
                add(acc, C == 1 ? weights(x, z) : weights(x, z, ch2, nch2, ncl2));
            }
        }
        return acc;
    };
    auto row_sum = [&]() {
        set_c();
        const Pairs acc = !positive(c) ? thread_sum(std::integral_constant<int, 0>())
                          : c.hi == 1.f && c.lo == 0.f ? thread_sum(std::integral_constant<int, 1>())
                                                       : thread_sum(std::integral_constant<int, 2>());
        const float2 hi = unpack2(acc.hi), lo = unpack2(acc.lo);
        const Pair mine = lane_sum<32>(add(Pair{hi.x, lo.x}, Pair{hi.y, lo.y}));
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
        Pair* all = parts[pass & 1];
        if (warp == 0) {
            const Pair z = lane_sum<kWarps>(sums[lane & (kWarps - 1)]);
            if (blocks == 1) {
                if (lane == 0) all[0] = z;
            } else {
                if (lane == 0) ptx::mbar_arrive_expect_tx(bar + 8 * (pass & 1), blocks * sizeof(Pair));
                if (lane < blocks) st_cluster(all + rank, bar + 8 * (pass & 1), lane, z);
            }
        }
        // A block sends its sum of pass k + 2, over that of pass k, once it has all
        // sums of pass k + 1, so every block has read those of pass k by then.
        // An expired wait ends the walk of the whole block, and by its missing sums the
        // others'.
        if (blocks == 1) __syncthreads();
        else lost = __syncthreads_or(!ptx::mbar_wait(bar + 8 * (pass & 1), pass >> 1 & 1, abort_flag, p.err, kErrWait, p.diag, 0x71));
        ++pass;
        Pair z = all[lane & (blocks - 1)];           // blocks is a power of two; the same order in every warp
        for (int o = blocks / 2; o > 0; o >>= 1) z = add(z, shuffle_xor(z, o));
        return z;
    };
    for (;;) {
        const int64_t at = (int64_t)(n0 + cur) * V;
        m = (int)(at & 3);
        end = m + V;
        per = ((end + n_gw - 1) / n_gw + 127) / 128 * 128;
        rp = target + at;
        rq = draft + at;
        c = {0.f, 0.f};
        Z = {1.f, 0.f};
        int taken = -1;
        for (unsigned long long m = kids[cur]; m; m &= m - 1) {
            const int i = __ffsll((long long)m) - 1;
            const Pair w = sub({pt[i], 0.f}, mul(c, qt[i]));
            if (positive(w) && less(mul(mul(Z, qt[i]), us[i]), w)) { taken = i; break; }
            if (!positive(Z)) break;                 // nothing is left of p: no other guess can be accepted
            c = positive(c) ? add(c, Z) : Pair{1.f, 0.f};
            Z = row_sum();
            if (lost) break;
        }
        if (taken < 0 || lost) break;
        cur = taken;
        if (tid == 0) path[count] = cur;
        ++count;
    }
    // ---- the next token, from what is left of the last node's row (all of it where nothing is)
    if (!lost && (!positive(c) || !positive(Z))) {
        c = {0.f, 0.f};
        Z = row_sum();
    }
    const Pair T0 = mul(Z, u_next);
    // running sum of x over the lanes before this one
    auto before_lane = [&](Pair x) {
        Pair inc = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const Pair t{__shfl_up_sync(0xffffffffu, inc.hi, o), __shfl_up_sync(0xffffffffu, inc.lo, o)};
            if (lane >= o) inc = add(t, inc);
        }
        const Pair t{__shfl_up_sync(0xffffffffu, inc.hi, 1), __shfl_up_sync(0xffffffffu, inc.lo, 1)};
        return lane ? t : Pair{0.f, 0.f};
    };
    const Pair* last = parts[(pass - 1) & 1];
    // the last of n_of sums with something in it whose running sum, on top of `base`, before it is <= T0; that running sum
    auto find = [&](const Pair* of, int n_of, Pair& base) {
        const Pair x = lane < n_of ? of[lane] : Pair{0.f, 0.f};
        const Pair pre = add(base, before_lane(x));
        const unsigned hit = __ballot_sync(0xffffffffu, positive(x) && !less(T0, pre));
        const int l = 31 - __clz(hit);               // -1 where there is none
        base = {__shfl_sync(0xffffffffu, pre.hi, l & 31), __shfl_sync(0xffffffffu, pre.lo, l & 31)};
        return l;
    };
    Pair before{0.f, 0.f};
    const int block = find(last, blocks, before);
    int found = -1;                                  // the warp whose part holds the token
    if (!lost && block == (int)rank) {
        const int w = find(sums, kWarps, before);
        if (w >= 0) found = (int)rank * kWarps + w;
        else if (tid == 0) p.next[b] = -1;           // sums that are no numbers
    }
    if (found == gw) {
        const int y1 = min(end, (gw + 1) * per);
        int best = -1;
        for (int y0 = gw * per; y0 < y1; y0 += 128) {
            const int y = y0 + 4 * lane;
            float a[4] = {}, d[4] = {};
            if (y < y1) {
                load4(rp, y, m, end, a);
                load4(rq, y, m, end, d);
                probabilities(d);
            }
            Pair w[4], x{0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const Pairs v = weights(pack2(a[e], a[e + 1]), pack2(d[e], d[e + 1]), ch2, nch2, ncl2);
                const float2 hi = unpack2(v.hi), lo = unpack2(v.lo);
                w[e] = add(Pair{0.f, 0.f}, Pair{hi.x, lo.x});
                w[e + 1] = add(Pair{0.f, 0.f}, Pair{hi.y, lo.y});
                x = add(add(x, w[e]), w[e + 1]);
            }
            Pair pre = add(before, before_lane(x));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (positive(w[e]) && !less(T0, pre)) best = y + e - m;
                pre = add(pre, w[e]);
            }
            before = {__shfl_sync(0xffffffffu, pre.hi, 31), __shfl_sync(0xffffffffu, pre.lo, 31)};
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        if (lane == 0) p.next[b] = best;
    }
    if (rank == 0) {
        if ((block < 0 || lost) && tid == 0) p.next[b] = -1;       // the row holds no positive number
        __syncthreads();
        if (tid < n) p.path[n0 + tid] = tid < count ? path[tid] : -1;
        if (tid == 0) p.count[b] = count;
    }
    __syncwarp();
    if (blocks > 1) {                                // no block leaves while another may still write to it
        cluster_arrive();
        cluster_wait();
    }
}

}  // namespace

namespace {
template <typename T, int THREADS>
void launch(const DraftVerifyParams& p, int blocks, cudaStream_t s) {
    static unsigned long long configured = 0;    // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(draft_verify_kernel<T, THREADS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        configured |= 1ull << (dev & 63);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, p.n_chars);
    cfg.blockDim = dim3(THREADS);
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
    cudaLaunchKernelEx(&cfg, draft_verify_kernel<T, THREADS>, p);
}
}  // namespace

// Blocks of a character's cluster: a power of two up to 16 that leaves each thread at
// least four elements, while all characters' blocks fit the SMs at once (two of 512
// threads or four of 256 an SM).  Blocks of 512 threads where 16 of them fit for every
// character and 256 threads would have more than eight elements each, else of 256, whose
// sums meet sooner; with 512 | 256: 131072 tokens of one character 15.1 | 18.7 us, 50001
// 7.9 | 9.1, 32768 of 8 (16-bit, 64 nodes) 19.4 | 17.5, of one 9.4 | 9.7; of 32 15.3 | 14.2,
// 131072 of 32 32.4 | 30.0.
void launch_draft_verify(const DraftVerifyParams& p, bool bf16, int num_sms, cudaStream_t s) {
    const bool large = (int64_t)kMaxCluster * p.n_chars <= 2 * num_sms && p.vocab > 8 * 256 * kMaxCluster;
    const int threads = large ? 512 : 256;
    int blocks = 1;
    while (blocks < kMaxCluster && blocks * threads * 4 < p.vocab && (int64_t)2 * blocks * p.n_chars * threads <= (int64_t)1024 * num_sms)
        blocks *= 2;
    if (large) bf16 ? launch<__nv_bfloat16, 512>(p, blocks, s) : launch<float, 512>(p, blocks, s);
    else bf16 ? launch<__nv_bfloat16, 256>(p, blocks, s) : launch<float, 256>(p, blocks, s);
}

}  // namespace kvm
