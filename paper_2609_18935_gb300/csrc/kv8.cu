// Caches in 8 bits: into blocks and out of them (the numbers: kv8.cuh).
//
//  kv8_append : a tail's keys, rotated in fp32, and its values into the blocks behind
//               the live entries, each block formed whole (its older rows too, if the
//               new ones need a larger scale); the tail's rotated queries into q_rot.
//  kv8_widen  : blocks as bf16 rows (exact): what the tensor-core attention and the
//               probe read, and kvm_get_kv.
//  kv8_gather : a removal's survivors, widened, in their new places; kv8_pack then
//               forms the blocks there (two launches over a bf16 copy: a block's scale
//               is known only once all its rows are, and in place its rows' sources
//               are other blocks' rows).
//  kv8_pack   : bf16 rows into blocks; kvm_set_kv.
//
// All move a 64 x D block a thread block, bound by memory.  A row past the last one in
// use is 0 in its block, so no number in a cache is ever other than finite: what is
// not finite in a key or value goes in as 0 and is reported (kErrValue), as a draft's.
#include "draft_rows.cuh"
#include "kv8.cuh"
#include "kvm_internal.cuh"

namespace kvm {
namespace {

constexpr int kThreads = 256;

// The item's character (the last with blk_off <= item), block, head, and K or V.
struct Item {
    int b, block, head;
    bool is_v;
};
template <typename P>
__device__ __forceinline__ Item item_of(const P& p, int item, int sides = 2) {
    int lo = 0, hi = p.n_chars - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.ch[mid].blk_off <= item) lo = mid; else hi = mid - 1;
    }
    const int local = item - p.ch[lo].blk_off, per = sides * p.Hkv;
    return {lo, p.ch[lo].block0 + local / per, local % per / sides, sides == 2 && (local & 1)};
}

__device__ __forceinline__ float block_max(float m, float* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, red[w]);
    return m;
}

__device__ __forceinline__ float2 bf2_f2(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w)); }
__device__ __forceinline__ uint32_t f2_bf2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// (cos, sin) of a position's turn of a pair: pos * turn modulo a whole turn is the low
// 64 bits of a product of integers, exact but for the 2^-64 that `turn` is rounded to
// (2^-33 of a turn at position 2^31), where 64-bit floats take a hundred times as long.
__device__ __forceinline__ void turn_of(int64_t pos, uint64_t turn, float& c, float& s) {
    const int64_t frac = (int64_t)((uint64_t)pos * turn);              // in [-1/2, 1/2) turns
    sincospif(__ll2float_rn(frac) * 0x1p-63f, &s, &c);
}

// A block of 64 rows of fp32 in shared memory, formed and stored.
template <int D>
__device__ __forceinline__ void store_block(const float* tile, float amax, uint8_t* dst, float* scale) {
    const int e = kv8_exponent(amax);
    const float inv = pow2(-e);
    uint32_t* d = reinterpret_cast<uint32_t*>(dst);
#pragma unroll 4
    for (int i = threadIdx.x; i < kKv8Rows * D / 4; i += kThreads) {
        const float4 x = reinterpret_cast<const float4*>(tile)[i];
        d[i] = to_e4m3(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    }
    if (threadIdx.x == 0) *scale = pow2(e);
}

// Blocks first, then a block of threads for each token's queries.
template <int D>
__global__ void __launch_bounds__(kThreads) kv8_append_kernel(const __grid_constant__ Kv8AppendParams p) {
    extern __shared__ __align__(16) float tile[];              // [64][D]
    __shared__ float red[kThreads / 32];
    __shared__ float cs[kMaxRotaryHalf], sn[kMaxRotaryHalf];
    grid_dependency_wait();
    grid_dependents_launch();
    const int t = threadIdx.x, half = p.R / 2;
    if ((int)blockIdx.x >= p.n_items) {
        const int n = blockIdx.x - p.n_items;                  // packed tail token
        int lo = 0, hi = p.n_chars - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.tail_off[mid] <= n) lo = mid; else hi = mid - 1;
        }
        const int64_t pos = p.tail_pos ? (int64_t)p.tail_pos[n] : p.p[lo] + n - p.tail_off[lo];
        for (int d = t; d < half; d += kThreads) turn_of(pos, p.turn[d], cs[d], sn[d]);
        const __nv_bfloat16* q = p.q + (int64_t)n * p.Hq * D;
        __nv_bfloat16* o = p.q_rot + (int64_t)n * p.Hq * D;
        if (half % 8 == 0) {
            const int per = half / 8 + (D - p.R) / 8;          // 16-byte pieces of a head: those turned in pairs first
            uint4 a, b;
            auto place = [&](int i) { return i / per * D + (i % per < half / 8 ? 8 * (i % per) : p.R + 8 * (i % per - half / 8)); };
            auto load = [&](int i) {
                if (i >= p.Hq * per) return;
                a = *reinterpret_cast<const uint4*>(q + place(i));
                if (i % per < half / 8) b = *reinterpret_cast<const uint4*>(q + place(i) + half);
            };
            load(t);
            __syncthreads();                                   // the angles are there
            for (int i = t; i < p.Hq * per; i += kThreads) {
                if (i > t) load(i);
                const int c = i % per;
                if (c < half / 8) {
                    uint32_t* x = reinterpret_cast<uint32_t*>(&a);
                    uint32_t* y = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 u = bf2_f2(x[k]), v = bf2_f2(y[k]);
                        const int d = 8 * c + 2 * k;
                        x[k] = f2_bf2(u.x * cs[d] - v.x * sn[d], u.y * cs[d + 1] - v.y * sn[d + 1]);
                        y[k] = f2_bf2(v.x * cs[d] + u.x * sn[d], v.y * cs[d + 1] + u.y * sn[d + 1]);
                    }
                    *reinterpret_cast<uint4*>(o + place(i) + half) = b;
                }
                *reinterpret_cast<uint4*>(o + place(i)) = a;
            }
        } else {
            __syncthreads();
            for (int i = t; i < p.Hq * D; i += kThreads) {
                const int d = i % D;
                const float x = __bfloat162float(q[i]);
                o[i] = d >= p.R     ? q[i]
                       : d < half   ? __float2bfloat16_rn(x * cs[d] - __bfloat162float(q[i + half]) * sn[d])
                                    : __float2bfloat16_rn(x * cs[d - half] + __bfloat162float(q[i - half]) * sn[d - half]);
            }
        }
        return;
    }
    const Item it = item_of(p, blockIdx.x);
    const Kv8Char& c = p.ch[it.b];
    const int row0 = it.block * kKv8Rows, L = p.L_prev[it.b];
    const int old = min(max(L - row0, 0), kKv8Rows), end = min(c.rows - row0, kKv8Rows);   // rows [old, end) are new
    const int64_t slot = (int64_t)it.head * p.slab_rows + c.cap_off + row0;
    uint8_t* dst = (it.is_v ? p.to.V : p.to.K) + slot * D;
    float* scale = (it.is_v ? p.to.Vs : p.to.Ks) + slot / kKv8Rows;
    const int n0 = p.tail_off[it.b] + row0 - L;                // packed token of the block's first row
    bool bad = false;
    {
        const float s = old ? *scale : 0.f;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(dst);
#pragma unroll 4
        for (int i = t; i < old * (D / 4); i += kThreads) {
            const uint32_t w = src[i];
            const float2 a = bf2_f2(e4m3_low(w)), b = bf2_f2(e4m3_high(w));
            reinterpret_cast<float4*>(tile)[i] = make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
        }
        const __nv_bfloat16* x = it.is_v ? p.v_new : p.k_new;
#pragma unroll 2
        for (int i = old * (D / 8) + t; i < kKv8Rows * (D / 8); i += kThreads) {
            const int r = i / (D / 8), d = i % (D / 8) * 8;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (r < end) w = *reinterpret_cast<const uint4*>(x + ((int64_t)(n0 + r) * p.Hkv + it.head) * D + d);
            bad = clear_not_finite(w) || bad;
            const float2 a = bf2_f2(w.x), b = bf2_f2(w.y), e = bf2_f2(w.z), f = bf2_f2(w.w);
            reinterpret_cast<float4*>(tile)[2 * i] = make_float4(a.x, a.y, b.x, b.y);
            reinterpret_cast<float4*>(tile)[2 * i + 1] = make_float4(e.x, e.y, f.x, f.y);
        }
    }
    __syncthreads();
    if (!it.is_v) {
        for (int i = t; i < (end - old) * half; i += kThreads) {
            const int r = old + i / half, d = i % half;
            const int64_t pos = p.tail_pos ? (int64_t)p.tail_pos[n0 + r] : p.p[it.b] + row0 + r - L;
            float co, si;
            turn_of(pos, p.turn[d], co, si);
            float* x = tile + r * D + d;
            float a = x[0] * co - x[half] * si, b = x[half] * co + x[0] * si;
            if (!isfinite(a)) { a = 0.f; bad = true; }         // two of the largest numbers together
            if (!isfinite(b)) { b = 0.f; bad = true; }
            x[0] = a;
            x[half] = b;
        }
        if (it.head == 0)
            for (int r = old + t; r < end; r += kThreads)
                p.pos[c.cap_off + row0 + r] = p.tail_pos ? p.tail_pos[n0 + r] : (int32_t)(p.p[it.b] + row0 + r - L);
        __syncthreads();
    }
    float m = 0.f;
#pragma unroll 4
    for (int i = t; i < end * (D / 4); i += kThreads) {
        const float4 x = reinterpret_cast<const float4*>(tile)[i];
        m = fmaxf(m, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(x.z), fabsf(x.w))));
    }
    m = block_max(m, red);
    store_block<D>(tile, m, dst, scale);
    if (bad) atomicOr(p.err, kErrValue);
}

// Sixteen numbers as bf16, times a block's scale.
__device__ __forceinline__ void widen16(const uint4& w, float scale, uint4& a, uint4& b) {
    const __nv_bfloat162 s = __float2bfloat162_rn(scale);
    auto pair = [&](uint32_t x) {
        const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), s);
        return *reinterpret_cast<const uint32_t*>(&r);
    };
    a = make_uint4(pair(e4m3_low(w.x)), pair(e4m3_high(w.x)), pair(e4m3_low(w.y)), pair(e4m3_high(w.y)));
    b = make_uint4(pair(e4m3_low(w.z)), pair(e4m3_high(w.z)), pair(e4m3_low(w.w)), pair(e4m3_high(w.w)));
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv8_widen_kernel(const __grid_constant__ Kv8WidenParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    Item it = item_of(p, blockIdx.x, p.V ? 2 : 1);
    const Kv8Char& c = p.ch[it.b];
    if (it.block - c.block0 >= p.sink[it.b]) it.block += p.gap[it.b];
    const int row0 = it.block * kKv8Rows;
    const int64_t slot = (int64_t)it.head * p.slab_rows + c.cap_off + row0;
    const uint4* src = reinterpret_cast<const uint4*>((it.is_v ? p.from.V : p.from.K) + slot * D);
    const float s = (it.is_v ? p.from.Vs : p.from.Ks)[slot / kKv8Rows];
    uint4* dst = reinterpret_cast<uint4*>((it.is_v ? p.V : p.K) + ((int64_t)it.head * p.dst_rows + c.row0 + row0) * D);
    const int n = min(c.rows - row0, kKv8Rows) * (D / 16);
    constexpr int kEach = kKv8Rows * D / 16 / kThreads;        // 1, 2 or 4 vectors a thread
    uint4 w[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kThreads;
        if (i < n) w[k] = src[i];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kThreads;
        uint4 a, b;
        if (i < n) {
            widen16(w[k], s, a, b);
            dst[2 * i] = a;
            dst[2 * i + 1] = b;
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv8_gather_kernel(const __grid_constant__ Kv8GatherParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    const Item it = item_of(p, blockIdx.x);
    const Kv8Char& c = p.ch[it.b];
    const int32_t* seg_start = p.seg_start + p.seg_off[it.b];
    const int32_t* seg_shift = p.seg_shift + p.seg_off[it.b];
    const int n_seg = p.n_seg[it.b];
    const uint8_t* from = it.is_v ? p.from.V : p.from.K;
    const float* scales = it.is_v ? p.from.Vs : p.from.Ks;
    __nv_bfloat16* to = it.is_v ? p.V : p.K;
    const int row0 = it.block * kKv8Rows, n = min(c.rows - row0, kKv8Rows) * (D / 16);
    const int64_t base = (int64_t)it.head * p.slab_rows + c.cap_off;
    constexpr int kEach = kKv8Rows * D / 16 / kThreads;
    uint4 w[kEach];
    float s[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kThreads;
        if (i >= n) continue;
        int row = row0 + i / (D / 16);
        if (row >= p.first[it.b]) {                            // the last segment that starts at or before it
            int lo = 0, hi = n_seg - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (seg_start[mid] <= row) lo = mid; else hi = mid - 1;
            }
            row += seg_shift[lo];
        }
        w[k] = *reinterpret_cast<const uint4*>(from + (base + row) * D + i % (D / 16) * 16);
        s[k] = scales[(base + row) / kKv8Rows];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kThreads;
        if (i >= n) continue;
        uint4* dst = reinterpret_cast<uint4*>(to + (base + row0) * D) + 2 * i;
        uint4 a, b;
        widen16(w[k], s[k], a, b);
        dst[0] = a;
        dst[1] = b;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv8_pack_kernel(const __grid_constant__ Kv8PackParams p) {
    __shared__ float red[kThreads / 32];
    grid_dependency_wait();
    grid_dependents_launch();
    const Item it = item_of(p, blockIdx.x);
    const Kv8Char& c = p.ch[it.b];
    const int row0 = it.block * kKv8Rows, n = min(c.rows - row0, kKv8Rows) * (D / 8);
    const uint4* src = reinterpret_cast<const uint4*>((it.is_v ? p.V : p.K) + ((int64_t)it.head * p.src_rows + c.row0 + row0) * D);
    const int64_t slot = (int64_t)it.head * p.slab_rows + c.cap_off + row0;
    constexpr int kEach = kKv8Rows * D / 8 / kThreads;         // 2, 4 or 8 vectors a thread
    uint4 w[kEach];
    float m = 0.f;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kThreads;
        w[k] = i < n ? src[i] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        bad = clear_not_finite(w[k]) || bad;
        const uint32_t* x = reinterpret_cast<const uint32_t*>(&w[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = bf2_f2(x[e]);
            m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    }
    m = block_max(m, red);
    const int e = kv8_exponent(m);
    const float inv = pow2(-e);
    uint2* dst = reinterpret_cast<uint2*>((it.is_v ? p.to.V : p.to.K) + slot * D);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const float2 a = bf2_f2(w[k].x), b = bf2_f2(w[k].y), f = bf2_f2(w[k].z), g = bf2_f2(w[k].w);
        dst[threadIdx.x + k * kThreads] = make_uint2(to_e4m3(a.x * inv, a.y * inv, b.x * inv, b.y * inv),
                                                     to_e4m3(f.x * inv, f.y * inv, g.x * inv, g.y * inv));
    }
    if (threadIdx.x == 0) (it.is_v ? p.to.Vs : p.to.Ks)[slot / kKv8Rows] = pow2(e);
    if (bad) atomicOr(p.err, kErrValue);
}

template <int D>
void launch_append(const Kv8AppendParams& p, cudaStream_t s) {
    constexpr int smem = kKv8Rows * D * (int)sizeof(float);
    static unsigned long long configured = 0;   // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(kv8_append_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        configured |= 1ull << (dev & 63);
    }
    launch_pdl(kv8_append_kernel<D>, dim3(p.n_items + p.total), dim3(kThreads), smem, s, p);
}

}  // namespace

void launch_kv8_append(const Kv8AppendParams& p, cudaStream_t s) {
    if (p.total <= 0) return;
    if (p.D == 64) launch_append<64>(p, s);
    else if (p.D == 128) launch_append<128>(p, s);
    else launch_append<256>(p, s);
}

void launch_kv8_widen(const Kv8WidenParams& p, cudaStream_t s) {
    if (p.n_items <= 0) return;
    launch_pdl(p.D == 64 ? kv8_widen_kernel<64> : p.D == 128 ? kv8_widen_kernel<128> : kv8_widen_kernel<256>, dim3(p.n_items),
               dim3(kThreads), 0, s, p);
}

void launch_kv8_gather(const Kv8GatherParams& p, cudaStream_t s) {
    if (p.n_items <= 0) return;
    launch_pdl(p.D == 64 ? kv8_gather_kernel<64> : p.D == 128 ? kv8_gather_kernel<128> : kv8_gather_kernel<256>, dim3(p.n_items),
               dim3(kThreads), 0, s, p);
}

void launch_kv8_pack(const Kv8PackParams& p, cudaStream_t s) {
    if (p.n_items <= 0) return;
    launch_pdl(p.D == 64 ? kv8_pack_kernel<64> : p.D == 128 ? kv8_pack_kernel<128> : kv8_pack_kernel<256>, dim3(p.n_items),
               dim3(kThreads), 0, s, p);
}

}  // namespace kvm
