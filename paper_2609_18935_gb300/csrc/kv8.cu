// Caches in 8 bits: into blocks and out of them (the numbers: kv8.cuh).
//
//  kv8_append : a tail's keys, rotated in fp32, and its values into the blocks behind
//               the live entries, each block formed whole (its older rows too, if the
//               new ones need a larger scale); the tail's rotated queries into q_rot; and
//               all blocks that it sees as bf16 rows (exact), which the tensor-core
//               attention reads.
//  kv8_widen  : blocks as bf16 rows for kvm_get_kv and the probe.
//  kv8_pack   : bf16 rows into blocks: kvm_set_kv.
// (Removals: kv_compact.)
//
// All are bound by memory.  No number in a cache is ever other than finite, those behind
// the last row in use too: what is not finite in a key or value goes in as 0 and is
// reported (kErrValue), as a draft's.
#include "draft_rows.cuh"
#include "kv8.cuh"
#include "kvm_internal.cuh"

namespace kvm {
namespace {

constexpr int kThreads = 256;
constexpr int kAppendThreads = 512;
constexpr int kPackThreads = 512;

// An item's character (the last whose first item is at or before it), head, K or V, and
// which of its items it is.
struct Item {
    int b, index, head;
    bool is_v;
};
template <int32_t Kv8AppendChar::*FIRST>
__device__ __forceinline__ Item item_of(const Kv8AppendParams& p, int item) {
    int lo = 0, hi = p.n_chars - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.ch[mid].*FIRST <= item) lo = mid; else hi = mid - 1;
    }
    const int local = item - p.ch[lo].*FIRST, per = 2 * p.Hkv;
    return {lo, local / per, local % per / 2, (bool)(local & 1)};
}

// Every block finds its place first: the constant cache's misses pass beside the grid before.
__device__ __forceinline__ void begin() {
    grid_dependency_wait();
    grid_dependents_launch();
}

template <int THREADS>
__device__ __forceinline__ float block_max(float m, float* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) m = fmaxf(m, red[w]);
    return m;
}

// A block's 64 x D numbers as bf16 rows, those below `rows`.
template <int D, int THREADS>
__device__ __forceinline__ void widen_block(const uint8_t* from, float scale, __nv_bfloat16* to, int rows) {
    constexpr int kEach = kKv8Rows * D / 8 / THREADS;
    const uint2* src = reinterpret_cast<const uint2*>(from);
    uint4* dst = reinterpret_cast<uint4*>(to);
    const __nv_bfloat162 s = __float2bfloat162_rn(scale);
    const int n = min(rows, kKv8Rows) * (D / 8);
    uint2 w[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * THREADS;
        if (i < n) w[k] = src[i];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * THREADS;
        if (i < n) dst[i] = widen8(w[k], s);
    }
}

// Some older blocks in sight of one head's K or V, all loads under way at once.
template <int D>
__device__ __forceinline__ void widen_old(const Kv8AppendParams& p, int item) {
    constexpr int kEach = 16, kVecs = kKv8Rows * D / 8;        // eights a thread, of a block
    static_assert(kEach * kAppendThreads == kv8_widen_blocks(D) * kVecs, "an item");
    const Item it = item_of<&Kv8AppendChar::old_off>(p, item);
    const Kv8AppendChar& c = p.ch[it.b];
    const int first = it.index * kv8_widen_blocks(D);
    begin();
    const int64_t slot0 = (int64_t)it.head * p.slab_rows + c.cap_off;
    const uint2* src = reinterpret_cast<const uint2*>((it.is_v ? p.to.V : p.to.K) + slot0 * D);
    uint4* dst = reinterpret_cast<uint4*>((it.is_v ? p.V : p.K) + slot0 * D);
    const float* scales = (it.is_v ? p.to.Vs : p.to.Ks) + slot0 / kKv8Rows;
    uint2 w[kEach];
    __nv_bfloat162 s[kEach];
    auto at = [&](int k, int& block) {                         // eight of the character's slab
        const int v = threadIdx.x + k * kAppendThreads, n = first + v / kVecs;
        block = n + (n >= c.sink ? c.gap : 0);
        return n < c.n_old ? (int64_t)block * kVecs + v % kVecs : (int64_t)-1;
    };
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        int block;
        const int64_t v = at(k, block);
        if (v < 0) continue;
        w[k] = src[v];
        s[k] = __float2bfloat162_rn(scales[block]);
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        int block;
        const int64_t v = at(k, block);
        if (v < 0) continue;
        dst[v] = widen8(w[k], s[k]);
    }
}

// A packed tail token's queries, rotated.
template <int D>
__device__ __forceinline__ void turn_queries(const Kv8AppendParams& p, int n, float* cs, float* sn) {
    const int t = threadIdx.x, half = p.R / 2;
    int lo = 0, hi = p.n_chars - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.ch[mid].tail_off <= n) lo = mid; else hi = mid - 1;
    }
    const int64_t tail0 = p.ch[lo].p - p.ch[lo].tail_off;
    begin();
    const int64_t pos = p.tail_pos ? (int64_t)p.tail_pos[n] : tail0 + n;
    const __nv_bfloat16* q = p.q + (int64_t)n * p.Hq * D;
    __nv_bfloat16* o = p.q_rot + (int64_t)n * p.Hq * D;
    if (half % 8 == 0) {
        const int per = half / 8 + (D - p.R) / 8;              // 16-byte pieces of a head: those turned in pairs first
        uint4 a, b;
        auto place = [&](int i) { return i / per * D + (i % per < half / 8 ? 8 * (i % per) : p.R + 8 * (i % per - half / 8)); };
        auto load = [&](int i) {
            if (i >= p.Hq * per) return;
            a = *reinterpret_cast<const uint4*>(q + place(i));
            if (i % per < half / 8) b = *reinterpret_cast<const uint4*>(q + place(i) + half);
        };
        load(t);                                               // under way during the angles
        for (int d = t; d < half; d += kAppendThreads) turn_of(pos, p.turn[d], cs[d], sn[d]);
        __syncthreads();
        for (int i = t; i < p.Hq * per; i += kAppendThreads) {
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
        return;
    }
    for (int d = t; d < half; d += kAppendThreads) turn_of(pos, p.turn[d], cs[d], sn[d]);
    __syncthreads();
    for (int i = t; i < p.Hq * D; i += kAppendThreads) {
        const int d = i % D;
        const float x = __bfloat162float(q[i]);
        o[i] = d >= p.R     ? q[i]
               : d < half   ? __float2bfloat16_rn(x * cs[d] - __bfloat162float(q[i + half]) * sn[d])
                            : __float2bfloat16_rn(x * cs[d - half] + __bfloat162float(q[i - half]) * sn[d - half]);
    }
}

// Eight numbers under a scale (its reciprocal inv, itself as bf16 in `to`): into the block and as bf16.
__device__ __forceinline__ void put8(const float (&x)[8], float inv, __nv_bfloat162 to, uint8_t* d8, __nv_bfloat16* d16) {
    const uint32_t a = to_e4m3(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), b = to_e4m3(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
    *reinterpret_cast<uint2*>(d8) = make_uint2(a, b);
    *reinterpret_cast<uint4*>(d16) = widen8(make_uint2(a, b), to);
}
__device__ __forceinline__ void get8(const uint4& w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = bf2_f2(v[e]);
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
    }
}

// A block behind the live entries, in registers from its loads to its stores: a thread has
// eight pairs that are turned (R up to 128, a multiple of 16), up to D / 64 eights that are
// not, and as many of older rows.  The angles are formed while the loads are under way.
template <int D>
__device__ __forceinline__ void form_block(const Kv8AppendParams& p, float* red) {
    constexpr int kOld = kKv8Rows * D / 8 / kAppendThreads, kFlat = kOld;
    const Item it = item_of<&Kv8AppendChar::blk_off>(p, blockIdx.x);
    const Kv8AppendChar& c = p.ch[it.b];
    const int t = threadIdx.x, L = c.L, row0 = (L / kKv8Rows + it.index) * kKv8Rows;
    const int old = min(max(L - row0, 0), kKv8Rows), end = min(L + c.M - row0, kKv8Rows);   // rows [old, end) are new, behind them 0
    const int64_t slot = (int64_t)it.head * p.slab_rows + c.cap_off + row0;
    uint8_t* dst = (it.is_v ? p.to.V : p.to.K) + slot * D;
    __nv_bfloat16* wide = (it.is_v ? p.V : p.K) + slot * D;
    float* scale = (it.is_v ? p.to.Vs : p.to.Ks) + slot / kKv8Rows;
    const int n0 = c.tail_off + row0 - L;                // packed token of the block's first row
    const int R = it.is_v ? 0 : p.R, half = R / 2, turned = half / 8, flat = (D - R) / 8;      // of a row: eights in pairs, and alone
    const __nv_bfloat16* x = (it.is_v ? p.v_new : p.k_new) + ((int64_t)n0 * p.Hkv + it.head) * D;
    const int64_t row = (int64_t)p.Hkv * D;
    const int tr = turned ? t / turned : kKv8Rows, td = turned ? t % turned * 8 : 0;           // the row and first dim of the pairs
    const bool has = tr >= old && tr < kKv8Rows;
    begin();
    const float s = old ? *scale : 0.f;
    uint2 was[kOld];
    uint4 is[kFlat], a = make_uint4(0, 0, 0, 0), b = a;
    if (has && tr < end) {
        a = *reinterpret_cast<const uint4*>(x + tr * row + td);
        b = *reinterpret_cast<const uint4*>(x + tr * row + td + half);
    }
#pragma unroll
    for (int k = 0; k < kFlat; ++k) {
        const int i = t + k * kAppendThreads, r = flat ? i / flat : kKv8Rows;
        is[k] = make_uint4(0, 0, 0, 0);
        if (r >= old && r < end) is[k] = *reinterpret_cast<const uint4*>(x + r * row + R + i % flat * 8);
    }
#pragma unroll
    for (int k = 0; k < kOld; ++k) {
        const int i = t + k * kAppendThreads;
        was[k] = make_uint2(0, 0);
        if (i < old * (D / 8)) was[k] = reinterpret_cast<const uint2*>(dst)[i];
    }
    float u[8], v[8], m = 0.f;
    bool bad = false;
    if (has) {
        float co[8], si[8];
        const int64_t pos = tr >= end ? 0 : p.tail_pos ? (int64_t)p.tail_pos[n0 + tr] : c.p + row0 + tr - L;
#pragma unroll
        for (int e = 0; e < 8; ++e) turn_of(pos, p.turn[td + e], co[e], si[e]);
        bad = clear_not_finite(a) || bad;
        bad = clear_not_finite(b) || bad;
        get8(a, u);
        get8(b, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = u[e];
            u[e] = y * co[e] - v[e] * si[e];
            v[e] = v[e] * co[e] + y * si[e];
            if (!isfinite(u[e])) { u[e] = 0.f; bad = true; }   // two of the largest numbers together
            if (!isfinite(v[e])) { v[e] = 0.f; bad = true; }
            m = fmaxf(m, fmaxf(fabsf(u[e]), fabsf(v[e])));
        }
    }
#pragma unroll
    for (int k = 0; k < kFlat; ++k) {
        bad = clear_not_finite(is[k]) || bad;
        float y[8];
        get8(is[k], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(y[e]));
    }
#pragma unroll
    for (int k = 0; k < kOld; ++k) m = fmaxf(m, e4m3_max(make_uint4(was[k].x, was[k].y, 0, 0)) * s);
    if (!it.is_v && it.head == 0)
        for (int r = old + t; r < end; r += kAppendThreads)
            p.pos[c.cap_off + row0 + r] = p.tail_pos ? p.tail_pos[n0 + r] : (int32_t)(c.p + row0 + r - L);
    m = block_max<kAppendThreads>(m, red);
    const int e = kv8_exponent(m);
    const float to = pow2(e), inv = pow2(-e);
    const __nv_bfloat162 to2 = __float2bfloat162_rn(to);
    if (has) {
        put8(u, inv, to2, dst + tr * D + td, wide + tr * D + td);
        put8(v, inv, to2, dst + tr * D + td + half, wide + tr * D + td + half);
    }
#pragma unroll
    for (int k = 0; k < kFlat; ++k) {
        const int i = t + k * kAppendThreads, r = flat ? i / flat : kKv8Rows;
        if (r < old || r >= kKv8Rows) continue;
        float y[8];
        get8(is[k], y);
        put8(y, inv, to2, dst + r * D + R + i % flat * 8, wide + r * D + R + i % flat * 8);
    }
#pragma unroll
    for (int k = 0; k < kOld; ++k) {
        const int i = t + k * kAppendThreads;
        if (i >= old * (D / 8)) continue;
        const uint2 w = s == to ? was[k] : requantised(was[k], s, inv);
        if (s != to) reinterpret_cast<uint2*>(dst)[i] = w;
        reinterpret_cast<uint4*>(wide)[i] = widen8(w, to2);
    }
    if (t == 0) *scale = to;
    if (bad) atomicOr(p.err, kErrValue);
}

// Blocks first (the longest way), then the blocks in sight that only need widening, then
// a thread block for each token's queries.  One launch for the three, bound by L2 (8 MB
// read and 17 written at 8192 entries, 256 tokens, 16 heads of 256): 9 us there, of which a
// new block takes 6, the widening 4 - 7; as two launches 11.1 and 8.5.
// IN_REGS: form_block; else, for the rotary dims that it does not take, by way of shared memory.
template <int D, bool IN_REGS>
__global__ void __launch_bounds__(kAppendThreads, 2) kv8_append_kernel(const __grid_constant__ Kv8AppendParams p) {
    extern __shared__ __align__(16) float tile[];              // [64][D]
    __shared__ float red[kAppendThreads / 32];
    __shared__ float cs[kMaxRotaryHalf], sn[kMaxRotaryHalf];
    const int t = threadIdx.x, half = p.R / 2;
    if ((int)blockIdx.x >= p.n_items + p.n_widen) {
        turn_queries<D>(p, blockIdx.x - p.n_items - p.n_widen, cs, sn);
        return;
    }
    if ((int)blockIdx.x >= p.n_items) {
        widen_old<D>(p, blockIdx.x - p.n_items);
        return;
    }
    if constexpr (IN_REGS) {
        form_block<D>(p, red);
        return;
    }
    const Item it = item_of<&Kv8AppendChar::blk_off>(p, blockIdx.x);
    const Kv8AppendChar& c = p.ch[it.b];
    const int L = c.L, row0 = (L / kKv8Rows + it.index) * kKv8Rows;
    const int old = min(max(L - row0, 0), kKv8Rows), end = min(L + c.M - row0, kKv8Rows);   // rows [old, end) are new
    const int64_t slot = (int64_t)it.head * p.slab_rows + c.cap_off + row0;
    uint8_t* dst = (it.is_v ? p.to.V : p.to.K) + slot * D;
    float* scale = (it.is_v ? p.to.Vs : p.to.Ks) + slot / kKv8Rows;
    const int n0 = c.tail_off + row0 - L;                // packed token of the block's first row
    bool bad = false;
    float m = 0.f;
    begin();
    {
        constexpr int kOld = (kKv8Rows * D / 16 + kAppendThreads - 1) / kAppendThreads, kNew = kKv8Rows * D / 8 / kAppendThreads;
        const float s = old ? *scale : 0.f;
        const uint4* src = reinterpret_cast<const uint4*>(dst);
        const __nv_bfloat16* x = it.is_v ? p.v_new : p.k_new;
        uint4 was[kOld], is[kNew];
#pragma unroll
        for (int k = 0; k < kOld; ++k) {
            const int i = t + k * kAppendThreads;
            if (i < old * (D / 16)) was[k] = src[i];
        }
#pragma unroll
        for (int k = 0; k < kNew; ++k) {
            const int i = t + k * kAppendThreads, r = i / (D / 8);
            is[k] = make_uint4(0, 0, 0, 0);
            if (r >= old && r < end) is[k] = *reinterpret_cast<const uint4*>(x + ((int64_t)(n0 + r) * p.Hkv + it.head) * D + i % (D / 8) * 8);
        }
#pragma unroll
        for (int k = 0; k < kOld; ++k) {
            const int i = t + k * kAppendThreads;
            if (i < old * (D / 16)) {
                m = fmaxf(m, e4m3_max(was[k]) * s);
                const uint32_t w[4] = {was[k].x, was[k].y, was[k].z, was[k].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float2 a = bf2_f2(e4m3_low(w[q])), b = bf2_f2(e4m3_high(w[q]));
                    reinterpret_cast<float4*>(tile)[4 * i + q] = make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
                }
            }
        }
        // the numbers that are not turned take part in the maximum here
        const int flat = it.is_v ? 0 : p.R;
#pragma unroll
        for (int k = 0; k < kNew; ++k) {
            const int i = t + k * kAppendThreads, d = i % (D / 8) * 8;
            if (i / (D / 8) < old) continue;
            bad = clear_not_finite(is[k]) || bad;
            const float2 f[4] = {bf2_f2(is[k].x), bf2_f2(is[k].y), bf2_f2(is[k].z), bf2_f2(is[k].w)};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (d + 2 * q >= flat) m = fmaxf(m, fmaxf(fabsf(f[q].x), fabsf(f[q].y)));
            }
            reinterpret_cast<float4*>(tile)[2 * i] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
            reinterpret_cast<float4*>(tile)[2 * i + 1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
        }
    }
    if (!it.is_v && half) {
        __syncthreads();
        for (int i = t; i < (end - old) * half; i += kAppendThreads) {
            const int r = old + i / half, d = i % half;
            const int64_t pos = p.tail_pos ? (int64_t)p.tail_pos[n0 + r] : c.p + row0 + r - L;
            float co, si;
            turn_of(pos, p.turn[d], co, si);
            float* x = tile + r * D + d;
            float a = x[0] * co - x[half] * si, b = x[half] * co + x[0] * si;
            if (!isfinite(a)) { a = 0.f; bad = true; }         // two of the largest numbers together
            if (!isfinite(b)) { b = 0.f; bad = true; }
            m = fmaxf(m, fmaxf(fabsf(a), fabsf(b)));
            x[0] = a;
            x[half] = b;
        }
    }
    if (!it.is_v && it.head == 0)
        for (int r = old + t; r < end; r += kAppendThreads)
            p.pos[c.cap_off + row0 + r] = p.tail_pos ? p.tail_pos[n0 + r] : (int32_t)(c.p + row0 + r - L);
    m = block_max<kAppendThreads>(m, red);
    const int e = kv8_exponent(m);
    const float to = pow2(e), inv = pow2(-e);
    uint32_t* d8 = reinterpret_cast<uint32_t*>(dst);
    uint2* d16 = reinterpret_cast<uint2*>((it.is_v ? p.V : p.K) + slot * D);
    const __nv_bfloat162 to2 = __float2bfloat162_rn(to);
    auto wide = [&](uint32_t x) {
        const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), to2);
        return *reinterpret_cast<const uint32_t*>(&r);
    };
#pragma unroll 4
    for (int i = t; i < kKv8Rows * D / 4; i += kAppendThreads) {
        const float4 x = reinterpret_cast<const float4*>(tile)[i];
        const uint32_t w = to_e4m3(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        d8[i] = w;
        d16[i] = make_uint2(wide(e4m3_low(w)), wide(e4m3_high(w)));
    }
    if (t == 0) *scale = to;
    if (bad) atomicOr(p.err, kErrValue);
}

// grid (blocks, heads, K and V)
template <int D>
__global__ void __launch_bounds__(kThreads) kv8_widen_kernel(const __grid_constant__ Kv8CopyParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    const bool is_v = blockIdx.z;
    const int row0 = blockIdx.x * kKv8Rows, head = blockIdx.y;
    const int64_t slot = head * p.slab_rows + p.cap_off + row0;
    widen_block<D, kThreads>((is_v ? p.cache.V : p.cache.K) + slot * D, (is_v ? p.cache.Vs : p.cache.Ks)[slot / kKv8Rows],
                             (is_v ? p.V : p.K) + (head * p.other_rows + p.row0 + row0) * D, p.rows - row0);
}

template <int D>
__global__ void __launch_bounds__(kPackThreads) kv8_pack_kernel(const __grid_constant__ Kv8CopyParams p) {
    __shared__ float red[kPackThreads / 32];
    grid_dependency_wait();
    grid_dependents_launch();
    const bool is_v = blockIdx.z;
    const int row0 = blockIdx.x * kKv8Rows, head = blockIdx.y, n = min(p.rows - row0, kKv8Rows) * (D / 8);
    const uint4* src = reinterpret_cast<const uint4*>((is_v ? p.V : p.K) + (head * p.other_rows + p.row0 + row0) * D);
    const int64_t slot = head * p.slab_rows + p.cap_off + row0;
    constexpr int kEach = kKv8Rows * D / 8 / kPackThreads;     // 1, 2 or 4 vectors a thread
    uint4 w[kEach];
    float m = 0.f;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = threadIdx.x + k * kPackThreads;
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
    m = block_max<kPackThreads>(m, red);
    const int e = kv8_exponent(m);
    const float inv = pow2(-e);
    uint2* dst = reinterpret_cast<uint2*>((is_v ? p.cache.V : p.cache.K) + slot * D);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const float2 a = bf2_f2(w[k].x), b = bf2_f2(w[k].y), f = bf2_f2(w[k].z), g = bf2_f2(w[k].w);
        dst[threadIdx.x + k * kPackThreads] = make_uint2(to_e4m3(a.x * inv, a.y * inv, b.x * inv, b.y * inv),
                                                     to_e4m3(f.x * inv, f.y * inv, g.x * inv, g.y * inv));
    }
    if (threadIdx.x == 0) (is_v ? p.cache.Vs : p.cache.Ks)[slot / kKv8Rows] = pow2(e);
    if (bad) atomicOr(p.err, kErrValue);
}

template <int D>
void launch_append(const Kv8AppendParams& p, cudaStream_t s) {
    const dim3 grid(p.n_items + p.n_widen + p.total);
    if (p.R % 16 == 0 && p.R <= 128) {
        launch_pdl(kv8_append_kernel<D, true>, grid, dim3(kAppendThreads), 0, s, p);
        return;
    }
    constexpr int smem = kKv8Rows * D * (int)sizeof(float);
    static unsigned long long configured = 0;   // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(kv8_append_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        configured |= 1ull << (dev & 63);
    }
    launch_pdl(kv8_append_kernel<D, false>, grid, dim3(kAppendThreads), smem, s, p);
}

}  // namespace

void launch_kv8_append(const Kv8AppendParams& p, cudaStream_t s) {
    if (p.total <= 0) return;
    if (p.D == 64) launch_append<64>(p, s);
    else if (p.D == 128) launch_append<128>(p, s);
    else launch_append<256>(p, s);
}

void launch_kv8_widen(const Kv8CopyParams& p, cudaStream_t s) {
    if (p.rows <= 0) return;
    launch_pdl(p.D == 64 ? kv8_widen_kernel<64> : p.D == 128 ? kv8_widen_kernel<128> : kv8_widen_kernel<256>,
               dim3((p.rows + kKv8Rows - 1) / kKv8Rows, p.Hkv, p.sides), dim3(kThreads), 0, s, p);
}

void launch_kv8_pack(const Kv8CopyParams& p, cudaStream_t s) {
    if (p.rows <= 0) return;
    launch_pdl(p.D == 64 ? kv8_pack_kernel<64> : p.D == 128 ? kv8_pack_kernel<128> : kv8_pack_kernel<256>,
               dim3((p.rows + kKv8Rows - 1) / kKv8Rows, p.Hkv, p.sides), dim3(kPackThreads), 0, s, p);
}

}  // namespace kvm
