// Attention of a few query rows a KV head (a decode step: one token, a group of heads)
// over a cache in 8 bits, or a windowed layer's in bf16.
//
// S^T = K Q^T and O^T = V^T P^T with mma.sync: the 16 keys of a step are the rows of the
// first product and the depth of the second, 8 query rows its columns.  The work is
// bound by the cache's bytes: 8 rows are a sixteenth of a tcgen05 tile, whose operands
// would have to pass through shared memory.
// 8-bit numbers become f16 (one instruction a pair), exactly; their blocks' scales stay
// outside, of K in the scores, of V as the sums are added up.  A query, rounded to bf16,
// is f16 times a power of two of its row (down to 2^-39 of the row's largest).  A weight is
// rounded to f16: off by up to 2^-11 of it, or 2^-32 of its warp's reference where it is small
// (f16 has steps of 2^-24 there, and weights are taken 2^7 higher).  The sum is of the weights
// before that rounding.  So a warp's part of a row is off by up to 2^-32 a key of its own largest
// weight, 2^-8 after 2^24 keys of one warp (a block's warps share a tile's keys, and a long tile's
// are shared by many blocks); a key at 2^-32 of the reference or below counts in the sum alone.
// As bf16 (a byte permute, a shift, a mask and a product a pair) 32 characters' step over 16K
// (284 MB) took 64.4 us, so 60.0, and 54.4 (5.2 TB/s) with longer ranges and what follows.
// bf16 caches: the words are the products' operands as they are.  Under a window of 4096
// the same characters take 46.5 us (259 MB, 5.6 TB/s), one over 512 entries 6.4; by way of
// rope_append and the tensor-core attention 49.5 and 9.4.
//
// One launch takes in the tail: a block turns its rows' queries itself, and the block
// whose range holds the end of a character's cache puts the new keys and values there
// (a character has one query tile a KV head, so no other block reads that end).  As a
// launch before this one that took 4 - 8 us of a step.
//
// The partition is the tensor-core attention's: 64-key units in contiguous ranges, a
// block an SM, partials of shared tiles for attn_combine.  A warp takes every WARPS-th
// 16 keys of a segment through a ring of its own in shared memory (cp.async, no barrier
// but the warp's), keeps its own softmax reference, sum and output in registers, and the
// block's warps meet at the segment's end.  Of 9 us for one character over 32K (7 units a
// block) 3.3 are the queries, beside which the rings' first stages are loaded, 3.5 the loop, 1
// the meeting.
//
// Layout.  The sum over d takes any order, the same for K and Q: lane (g, j) = (lane / 4,
// lane mod 4) reads 16 bytes of key g (and g + 8) at a time, and two words of them are its
// part of one product step.  For V it reads 16 bytes of its four keys 2j, 2j + 1, 2j + 8,
// 2j + 9, whose bytes meet in pairs of keys; a product's 16 rows are then two numbers of
// each lane g.  The rings' 16-byte pieces are turned by their row, so that each quarter
// of a warp reads all banks.
#include <cuda_fp16.h>

#include "attn_tiles.cuh"
#include "draft_rows.cuh"
#include "kv8.cuh"
#include "kvm_internal.cuh"
#include "sm100_ptx.cuh"

namespace kvm {
namespace {

using ptx::ex2;
using ptx::smem_u32;

constexpr int kStep = 16;                      // keys of a warp's step
constexpr int BM = kAttnRows;
constexpr float kUp = 7.f;                     // weights are taken 2^7 higher: up to 2^15, where f16 has room

// E: bytes of a cache's number, 1 (e4m3) or 2 (bf16).  Eight warps: twelve and sixteen (of
// fewer stages) took longer over 8 bits, 62.1 against 60.9 us for 32 characters over 16K,
// 8.1 against 7.3 for one over 512, more of them meet at the end.  Six where a key is 512 bytes:
// a warp's two stages are 32 KB, and eight warps' rings would be 256 of the 227 there are.
template <int D, int NT, int E>
struct Cfg {
    static constexpr int WARPS = D * E == 512 ? 6 : 8;
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int ROW = D * E;                          // bytes of a key, or value
    static constexpr int SIDE = kStep * ROW;                   // of a step's
    static constexpr int STAGE = 2 * SIDE + (E == 1 ? 16 : 0); // and its two scales
    static constexpr int STAGES = ROW == 512 ? 2 : ROW == 256 ? 3 : 6;
    static constexpr int RING = STAGES * STAGE;
    static constexpr int ROWS = 8 * NT;
    static constexpr int PITCH = D + 4;                        // floats of a merged row
    static constexpr int MERGE = WARPS * ROWS * PITCH * 4;
    // behind the rings: the warps' references and sums, a maximum of K and of V a warp,
    // the rows' turns, and their queries (bf16) or new keys (fp32)
    static constexpr int OFF_WM = WARPS * RING > MERGE ? WARPS * RING : MERGE;
    static constexpr int OFF_RED = OFF_WM + 2 * WARPS * ROWS * 4;
    static constexpr int OFF_TURN = OFF_RED + 2 * WARPS * 4;
    static constexpr int OFF_X = OFF_TURN + ROWS * D * 4;
    static constexpr int SMEM = OFF_X + ROWS * D * 4;
};
static_assert(Cfg<256, 2, 1>::SMEM <= 232448 && Cfg<128, 2, 1>::SMEM <= 232448 && Cfg<64, 2, 1>::SMEM <= 232448 &&
              Cfg<256, 2, 2>::SMEM <= 232448 && Cfg<128, 2, 2>::SMEM <= 232448 && Cfg<64, 2, 2>::SMEM <= 232448, "shared memory");

// Byte offset of 16-byte piece `col` of row `row` of a step's K or V, rows of ROW bytes.
template <int ROW>
__device__ __forceinline__ int piece(int row, int col) {
    if (ROW == 64) return (row >> 1) * 128 + (((((row & 1) << 2) | col) ^ ((row & 6))) << 4);
    return row * ROW + (((col & ~7) | ((col ^ row) & 7)) << 4);
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// c += scale * (A B)
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float scale) {
    float d[4] = {0.f, 0.f, 0.f, 0.f};
    mma16816(d, a0, a1, a2, a3, b0, b1);
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = fmaf(scale, d[e], c[e]);
}
// The low and the high two e4m3 numbers of a word as f16 (exactly).
__device__ __forceinline__ void e4m3_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t f2_h2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The new keys and values of one head that lie in key tile kt: into the cache's block, and
// the whole block under a larger (or smaller) scale where they need it.  By all threads;
// `load` may come long before `finish`, which lies between two barriers of the block.
template <int D, int NT>
struct FormedBlock {
    static constexpr int kWarps = Cfg<D, NT, 1>::WARPS, kThreads = Cfg<D, NT, 1>::THREADS;
    static constexpr int kOld = (kKv8Rows * D / 16 + kThreads - 1) / kThreads, kNew = (8 * NT * D / 8 + kThreads - 1) / kThreads;
    uint4 wk[kOld], wv[kOld], nv[kNew];
    float sk, sv;
    int64_t slot, src;
    int old, n, tok0;                                          // rows there, new rows, of them the first token

    __device__ __forceinline__ void load(const DecodeParams& pp, const AttnChar& ch, int kvh, int kt) {
        const AttnParams& p = pp.a;
        const int tid = threadIdx.x, row0 = kt * kAttnKeys;
        old = min(max(ch.L_prev - row0, 0), kKv8Rows);
        n = min(ch.L_prev + ch.M - row0, kKv8Rows) - old;
        tok0 = row0 + old - ch.L_prev;
        slot = (int64_t)kvh * p.slab_rows + ch.cap_off + row0;
        src = ((int64_t)(ch.tail_off + tok0) * p.Hkv + kvh) * D;
        const uint4* bk = reinterpret_cast<const uint4*>(pp.from.K + slot * D);
        const uint4* bv = reinterpret_cast<const uint4*>(pp.from.V + slot * D);
        sk = old ? pp.from.Ks[slot / kKv8Rows] : 0.f;
        sv = old ? pp.from.Vs[slot / kKv8Rows] : 0.f;
#pragma unroll
        for (int k = 0; k < kOld; ++k) {
            const int i = tid + k * kThreads;
            wk[k] = wv[k] = make_uint4(0, 0, 0, 0);
            if (i < old * (D / 16)) {
                wk[k] = bk[i];
                wv[k] = bv[i];
            }
        }
#pragma unroll
        for (int k = 0; k < kNew; ++k) {
            const int i = tid + k * kThreads;
            nv[k] = make_uint4(0, 0, 0, 0);
            if (i < n * (D / 8)) nv[k] = *reinterpret_cast<const uint4*>(p.v_new + src + (int64_t)(i / (D / 8)) * p.Hkv * D + i % (D / 8) * 8);
        }
    }
    __device__ __forceinline__ void finish(const DecodeParams& pp, const AttnChar& ch, int kvh, float* red, const float2* turn, float* keys);
};

template <int D, int NT>
__device__ __forceinline__ void FormedBlock<D, NT>::finish(const DecodeParams& pp, const AttnChar& ch, int kvh, float* red, const float2* turn,
                                                           float* keys) {
    const AttnParams& p = pp.a;
    const int tid = threadIdx.x, half = p.R / 2;
    const int64_t row = (int64_t)p.Hkv * D;
    uint4* bk = reinterpret_cast<uint4*>(pp.from.K + slot * D);
    uint4* bv = reinterpret_cast<uint4*>(pp.from.V + slot * D);
    float mk = 0.f, mv = 0.f;
    bool bad = false;
    auto key = [&](int r, int d) {
        __nv_bfloat16 x = p.k_new[src + r * row + d];
        bad = clear_not_finite(x) || bad;
        return __bfloat162float(x);
    };
    for (int i = tid; i < n * half; i += kThreads) {
        const int r = i / half, d = i % half;
        const float2 t = turn[(tok0 + r) * half + d];
        const float x = key(r, d), y = key(r, d + half);
        float a = x * t.x - y * t.y, b = y * t.x + x * t.y;
        if (!isfinite(a)) { a = 0.f; bad = true; }             // two of the largest numbers together
        if (!isfinite(b)) { b = 0.f; bad = true; }
        keys[r * D + d] = a;
        keys[r * D + d + half] = b;
        mk = fmaxf(mk, fmaxf(fabsf(a), fabsf(b)));
    }
    for (int i = tid; i < n * (D - p.R); i += kThreads) {
        const int r = i / (D - p.R), d = p.R + i % (D - p.R);
        const float x = key(r, d);
        keys[r * D + d] = x;
        mk = fmaxf(mk, fabsf(x));
    }
#pragma unroll
    for (int k = 0; k < kNew; ++k) {
        bad = clear_not_finite(nv[k]) || bad;
        const uint32_t w[4] = {nv[k].x, nv[k].y, nv[k].z, nv[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = bf2_f2(w[e]);
            mv = fmaxf(mv, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    }
#pragma unroll
    for (int k = 0; k < kOld; ++k) {
        mk = fmaxf(mk, e4m3_max(wk[k]) * sk);
        mv = fmaxf(mv, e4m3_max(wv[k]) * sv);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mk = fmaxf(mk, __shfl_xor_sync(0xffffffffu, mk, o));
        mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, o));
    }
    if ((tid & 31) == 0) {
        red[tid >> 5] = mk;
        red[kWarps + (tid >> 5)] = mv;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        mk = fmaxf(mk, red[w]);
        mv = fmaxf(mv, red[kWarps + w]);
    }
    const int ek = kv8_exponent(mk), ev = kv8_exponent(mv);
    const float tk = pow2(ek), tv = pow2(ev), ik = pow2(-ek), iv = pow2(-ev);
#pragma unroll
    for (int k = 0; k < kOld; ++k) {
        const int i = tid + k * kThreads;
        if (i < old * (D / 16)) {
            if (tk != sk) bk[i] = requantised(wk[k], sk, ik);
            if (tv != sv) bv[i] = requantised(wv[k], sv, iv);
        }
    }
    for (int i = tid; i < n * (D / 4); i += kThreads) {
        const float4 x = reinterpret_cast<const float4*>(keys)[i];
        reinterpret_cast<uint32_t*>(bk)[old * (D / 4) + i] = to_e4m3(x.x * ik, x.y * ik, x.z * ik, x.w * ik);
    }
#pragma unroll
    for (int k = 0; k < kNew; ++k) {
        const int i = tid + k * kThreads;
        const float2 a = bf2_f2(nv[k].x), b = bf2_f2(nv[k].y), c = bf2_f2(nv[k].z), d = bf2_f2(nv[k].w);
        if (i < n * (D / 8))
            reinterpret_cast<uint2*>(bv)[old * (D / 8) + i] =
                make_uint2(to_e4m3(a.x * iv, a.y * iv, b.x * iv, b.y * iv), to_e4m3(c.x * iv, c.y * iv, d.x * iv, d.y * iv));
    }
    if (tid == 0) {
        pp.from.Ks[slot / kKv8Rows] = tk;
        pp.from.Vs[slot / kKv8Rows] = tv;
    }
    if (kvh == 0 && tid < n) {
        const int t = tok0 + tid;
        p.pos[ch.cap_off + ch.L_prev + t] = p.tail_pos ? p.tail_pos[ch.tail_off + t] : (int32_t)(ch.p + t);
    }
    if (bad) atomicOr(p.err, kErrValue);
    __syncthreads();
}

// The same for a cache in bf16: tokens [t0, t1).
template <int D, int NT>
__device__ __forceinline__ void append_rows(const AttnParams& p, const AttnChar& ch, int kvh, int t0, int t1, const float2* turn) {
    constexpr int kThreads = Cfg<D, NT, 2>::THREADS;
    const int tid = threadIdx.x, half = p.R / 2, n = t1 - t0;
    const int64_t src = ((int64_t)(ch.tail_off + t0) * p.Hkv + kvh) * D, row = (int64_t)p.Hkv * D;
    const int64_t dst = ((int64_t)kvh * p.slab_rows + ch.cap_off + ch.L_prev + t0) * D;
    for (int i = tid; i < n * (D / 8); i += kThreads)
        *reinterpret_cast<uint4*>(p.V + dst + 8 * i) = *reinterpret_cast<const uint4*>(p.v_new + src + i / (D / 8) * row + i % (D / 8) * 8);
    for (int i = tid; i < n * half; i += kThreads) {
        const int r = i / half, d = i % half;
        const float2 t = turn[(t0 + r) * half + d];
        const float x = __bfloat162float(p.k_new[src + r * row + d]), y = __bfloat162float(p.k_new[src + r * row + d + half]);
        p.K[dst + r * D + d] = __float2bfloat16_rn(x * t.x - y * t.y);
        p.K[dst + r * D + d + half] = __float2bfloat16_rn(y * t.x + x * t.y);
    }
    for (int i = tid; i < n * (D - p.R); i += kThreads) {
        const int r = i / (D - p.R), d = p.R + i % (D - p.R);
        p.K[dst + r * D + d] = p.k_new[src + r * row + d];
    }
    if (kvh == 0 && tid < n) p.pos[ch.cap_off + ch.L_prev + t0 + tid] = p.tail_pos ? p.tail_pos[ch.tail_off + t0 + tid] : (int32_t)(ch.p + t0 + tid);
    __syncthreads();
}

template <int D, int NT, int E>
__global__ void __launch_bounds__(Cfg<D, NT, E>::THREADS, 1) decode_attention_kernel(const __grid_constant__ DecodeParams pp) {
    using C = Cfg<D, NT, E>;
    constexpr int kWarps = C::WARPS, kThreads = C::THREADS;
    constexpr int KS = D / 16;                                 // 16-row pieces of O^T
    constexpr bool SIXTEEN = E == 1 && D > 64;                 // a lane's dims that are neighbours
    extern __shared__ __align__(128) uint8_t smem[];
    const AttnParams& p = pp.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
    uint8_t* ring = smem + warp * C::RING;
    const uint32_t ring_at = smem_u32(ring);
    float* meet = reinterpret_cast<float*>(smem);              // [warp][row][PITCH], once the rings are done
    float* wm = reinterpret_cast<float*>(smem + C::OFF_WM);    // [warp][row]: reference, then sum
    float* wl = wm + kWarps * C::ROWS;
    float2* turn = reinterpret_cast<float2*>(smem + C::OFF_TURN);                      // [token][R / 2]
    __nv_bfloat16* q_s = reinterpret_cast<__nv_bfloat16*>(smem + C::OFF_X);            // [row][D]

    // the block's segments, as the tensor-core attention walks them
    const int cta = blockIdx.x, waves = p.waves;
    const int t_begin = p.cta_tile[cta], k_begin = p.cta_k[cta];
    const int t_end = p.cta_tile[cta + 1], k_end = p.cta_k[cta + 1];
    const int n_seg = waves + ((t_begin == t_end && k_begin == k_end) ? 0 : t_end - t_begin + (k_end > 0 ? 1 : 0));

    auto tile_of = [&](int seg) { return seg < waves ? seg * p.n_ctas + ((seg & 1) ? p.n_ctas - 1 - cta : cta) : t_begin + (seg - waves); };
    auto decode = [&](int t) { return p.window ? decode_tile<true, false>(p, t) : decode_tile<false, false>(p, t); };
    // the first segment's place, whose lines of the constant cache take 0.8 us, before the wait
    Tile T = {};
    if (n_seg > 0) T = decode(tile_of(0));

    // a removal, or the layer's last step, wrote the cache
    grid_dependency_wait();
    grid_dependents_launch();

    for (int seg = 0; seg < n_seg; ++seg) {
        const int t = tile_of(seg);
        if (seg > 0) T = decode(t);
        const AttnChar& ch = p.ch[T.b];
        const int k0 = seg == waves ? k_begin : 0, k1 = (seg >= waves && t == t_end) ? k_end : T.nk;
        const bool full = k0 == 0 && k1 == T.nk;
        const int steps = (k1 - k0) * (kAttnKeys / kStep);
        const int64_t slab = (int64_t)T.kvh * p.slab_rows + ch.cap_off;
        const int rows = (T.tok_end - T.tok0) * p.g;           // of them real

        // step s of the segment into ring place `at`
        auto load = [&](int s, int at) {
            if (s >= steps) return;
            const int64_t row = slab + (int64_t)key_tile<true>(T, k0 + s / 4) * kAttnKeys + s % 4 * kStep;
            const uint8_t* k = (E == 1 ? pp.from.K : reinterpret_cast<const uint8_t*>(p.K)) + row * C::ROW;
            const uint8_t* v = (E == 1 ? pp.from.V : reinterpret_cast<const uint8_t*>(p.V)) + row * C::ROW;
            const uint32_t to = ring_at + at * C::STAGE;
#pragma unroll
            for (int c = 0; c < C::ROW / 32; ++c) {
                const int id = c * 32 + lane, r = id / (C::ROW / 16), col = id % (C::ROW / 16);
                const uint32_t o = to + piece<C::ROW>(r, col);
                cp16(o, k + id * 16);
                cp16(o + C::SIDE, v + id * 16);
            }
            if (E == 1 && lane < 2) cp4(to + 2 * C::SIDE + 4 * lane, (lane ? pp.from.Vs : pp.from.Ks) + row / kKv8Rows);
        };
        // units from `fresh` on have new rows (a query tile holds all of its character's): this block
        // forms those of its range before anyone loads them, the others are under way meanwhile
        const int fresh = ch.L_prev / kAttnKeys - T.gap;
        const bool forms = fresh < k1;
        // what the queries and the block to form need goes first: behind the rings' 128 KB a load takes 2.5 us
        const int half = p.R / 2;
        const uint64_t word = tid < ch.M * half ? pp.turn[tid % half] : 0;
        auto row_of = [&](int r) { return p.q + ((int64_t)(ch.tail_off + r / p.g) * p.Hq + T.kvh * p.g + r % p.g) * D; };
        const bool eights = half % 8 == 0;
        const int per = half / 8 + (D - p.R) / 8;              // 16-byte pieces of a row: those turned in pairs first
        uint4 a, b;
        auto place = [&](int i) { return i % per < half / 8 ? 8 * (i % per) : p.R + 8 * (i % per - half / 8); };
        auto get = [&](int i) {
            if (i >= rows * per) return;
            const __nv_bfloat16* x = row_of(i / per) + place(i);
            a = *reinterpret_cast<const uint4*>(x);
            if (i % per < half / 8) b = *reinterpret_cast<const uint4*>(x + half);
        };
        if (eights) get(tid);
        FormedBlock<D, NT> block;
        if (E == 1 && NT == 1 && forms) block.load(pp, ch, T.kvh, key_tile<true>(T, max(k0, fresh)));
#pragma unroll
        for (int s = 0; s < C::STAGES - 1; ++s) {
            const int step = warp + s * kWarps;
            if (!forms || k0 + step / 4 < fresh) load(step, s);
            if (!forms) cp_commit();
        }
        {
            for (int i = tid; i < ch.M * half; i += kThreads) {
                const int t = i / half;
                const int64_t pos = p.tail_pos ? (int64_t)p.tail_pos[ch.tail_off + t] : ch.p + t;
                turn_of(pos, i == tid ? word : pp.turn[i % half], turn[i].x, turn[i].y);
            }
            if (eights) {
                __syncthreads();                               // the turns are there
                for (int i = tid; i < rows * per; i += kThreads) {
                    if (i > tid) get(i);
                    __nv_bfloat16* o = q_s + i / per * D + place(i);
                    if (i % per < half / 8) {
                        const float2* t = turn + i / per / p.g * half + place(i);
                        uint32_t* x = reinterpret_cast<uint32_t*>(&a);
                        uint32_t* y = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float2 u = bf2_f2(x[k]), v = bf2_f2(y[k]), t0 = t[2 * k], t1 = t[2 * k + 1];
                            x[k] = f2_bf2(u.x * t0.x - v.x * t0.y, u.y * t1.x - v.y * t1.y);
                            y[k] = f2_bf2(v.x * t0.x + u.x * t0.y, v.y * t1.x + u.y * t1.y);
                        }
                        *reinterpret_cast<uint4*>(o + half) = b;
                    }
                    *reinterpret_cast<uint4*>(o) = a;
                }
            } else {
                __syncthreads();
                for (int i = tid; i < rows * D; i += kThreads) {
                    const int r = i / D, d = i % D;
                    const __nv_bfloat16* x = row_of(r) + d;
                    const float2* t = turn + r / p.g * half;
                    q_s[i] = d >= p.R   ? *x
                             : d < half ? __float2bfloat16_rn(__bfloat162float(x[0]) * t[d].x - __bfloat162float(x[half]) * t[d].y)
                                        : __float2bfloat16_rn(__bfloat162float(x[0]) * t[d - half].x + __bfloat162float(x[-half]) * t[d - half].y);
                }
            }
            __syncthreads();
        }
        // Q: a lane's words of each step of the sum, rows g (and g + 8); over 8 bits as f16 times a power of two of the row
        uint32_t q[NT][KS][2];
        float row_scale[NT][2];                                // of rows 8 n + 2 j and the next
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = 8 * n + g;
            const __nv_bfloat16* src = q_s + r * D;
            if constexpr (E == 2) {
#pragma unroll
                for (int c = 0; c < KS / 2; ++c) {
                    const int col = 8 * (c >> 1) + 2 * j + (c & 1);
                    const uint4 x = r < rows ? *reinterpret_cast<const uint4*>(src + 8 * col) : make_uint4(0, 0, 0, 0);
                    q[n][2 * c][0] = x.x; q[n][2 * c][1] = x.y;
                    q[n][2 * c + 1][0] = x.z; q[n][2 * c + 1][1] = x.w;
                }
                row_scale[n][0] = row_scale[n][1] = p.scale_log2;
            } else {
                uint4 x[KS / 4][2];
                float top = 0.f;
#pragma unroll
                for (int c = 0; c < KS / 4; ++c) {
                    const int col = D == 64 ? j : 8 * (c >> 1) + 2 * j + (c & 1);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        x[c][h] = r < rows ? *reinterpret_cast<const uint4*>(src + 16 * col + 8 * h) : make_uint4(0, 0, 0, 0);
                        const uint32_t w[4] = {x[c][h].x, x[c][h].y, x[c][h].z, x[c][h].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) top = fmaxf(top, fmaxf(fabsf(bf2_f2(w[k]).x), fabsf(bf2_f2(w[k]).y)));
                    }
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // top < 2^ex: its row's numbers below 2^15
                const int ex = min(max((int)(__float_as_uint(top) >> 23) - 126, -110), 128);
                const float up = pow2(15 - ex), scale = pow2(ex - 15) * p.scale_log2;
#pragma unroll
                for (int c = 0; c < KS / 4; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t w[4] = {x[c][h].x, x[c][h].y, x[c][h].z, x[c][h].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float2 a = bf2_f2(w[k]);
                            q[n][4 * c + 2 * h + (k >> 1)][k & 1] = f2_h2(a.x * up, a.y * up);
                        }
                    }
                row_scale[n][0] = __shfl_sync(0xffffffffu, scale, 8 * j);
                row_scale[n][1] = __shfl_sync(0xffffffffu, scale, 8 * j + 4);
            }
        }
        if (forms) {
            __syncthreads();                                   // the queries' place takes the new keys
            if constexpr (E == 2) {
                const int t0 = max(key_tile<true>(T, max(k0, fresh)) * kAttnKeys - ch.L_prev, 0);
                append_rows<D, NT>(p, ch, T.kvh, t0, min((key_tile<true>(T, k1 - 1) + 1) * kAttnKeys - ch.L_prev, ch.M), turn);
            } else {
                for (int u = max(k0, fresh); u < k1; ++u) {
                    if (NT > 1 || u > max(k0, fresh)) block.load(pp, ch, T.kvh, key_tile<true>(T, u));
                    block.finish(pp, ch, T.kvh, reinterpret_cast<float*>(smem + C::OFF_RED), turn, reinterpret_cast<float*>(smem + C::OFF_X));
                }
            }
#pragma unroll
            for (int s = 0; s < C::STAGES - 1; ++s) {
                const int step = warp + s * kWarps;
                if (k0 + step / 4 >= fresh) load(step, s);
                cp_commit();
            }
        }
        // rows 8 n + 2 j and the next: their live indices, references, and this lane's share of the sums
        int at[NT][2];
        float m[NT][2], l[NT][2], o[NT][KS][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                at[n][e] = ch.L_prev + min(T.tok0 + (8 * n + 2 * j + e) / p.g, ch.M - 1);
                m[n][e] = -INFINITY;
                l[n][e] = 0.f;
            }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < KS; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][c][e] = 0.f;
        const int first_at = ch.L_prev + T.tok0, last_at = ch.L_prev + T.tok_end - 1;

        for (int s = warp, i = 0; s < steps; s += kWarps, ++i) {
            cp_wait<C::STAGES - 2>();
            __syncwarp();
            const uint8_t* kt = ring + (i % C::STAGES) * C::STAGE;
            const uint8_t* vt = kt + C::SIDE;
            const float ks = E == 1 ? *reinterpret_cast<const float*>(kt + 2 * C::SIDE) : 1.f;
            [[maybe_unused]] const float vs = E == 1 ? *reinterpret_cast<const float*>(kt + 2 * C::SIDE + 4) : 1.f;
            load(s + (C::STAGES - 1) * kWarps, (i + C::STAGES - 1) % C::STAGES);
            cp_commit();
            float sc[NT][2][4];                                // two chains of products
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[n][e >> 2][e & 3] = 0.f;
            if constexpr (E == 2) {
#pragma unroll
                for (int c = 0; c < KS / 2; ++c) {
                    const int col = 8 * (c >> 1) + 2 * j + (c & 1);
                    const uint4 x = *reinterpret_cast<const uint4*>(kt + piece<C::ROW>(g, col));
                    const uint4 y = *reinterpret_cast<const uint4*>(kt + piece<C::ROW>(g + 8, col));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma16816_bf16(sc[n][0], x.x, y.x, x.y, y.y, q[n][2 * c][0], q[n][2 * c][1]);
                        mma16816_bf16(sc[n][1], x.z, y.z, x.w, y.w, q[n][2 * c + 1][0], q[n][2 * c + 1][1]);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < KS / 4; ++c) {
                    const int col = D == 64 ? j : 8 * (c >> 1) + 2 * j + (c & 1);
                    const uint4 x = *reinterpret_cast<const uint4*>(kt + piece<C::ROW>(g, col));
                    const uint4 y = *reinterpret_cast<const uint4*>(kt + piece<C::ROW>(g + 8, col));
                    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t a0, a1, a2, a3;
                        e4m3_f16(xs[w], a0, a2);
                        e4m3_f16(ys[w], a1, a3);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816(sc[n][w & 1], a0, a1, a2, a3, q[n][4 * c + w][0], q[n][4 * c + w][1]);
                    }
                }
            }
            // keys g and g + 8 of the step for rows 2 j, 2 j + 1
            const int key0 = key_tile<true>(T, k0 + s / 4) * kAttnKeys + s % 4 * kStep;
            bool above = false;
            float x[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][e] = (sc[n][0][e] + sc[n][1][e]) * (ks * row_scale[n][e & 1]);
            if (key0 + kStep - 1 > first_at || (p.window && key0 <= last_at - p.window)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + g + 8 * (e >> 1), me = at[n][e & 1];
                        if (key > me || (p.window && key <= me - p.window && key >= p.n_sink)) x[n][e] = -INFINITY;
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) above = above || x[n][e] > m[n][e & 1] + 8.f;
            // the reference moves only when a score is 2^8 above it
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(x[n][e], x[n][e + 2]);
#pragma unroll
                        for (int b = 4; b < 32; b <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                        top = fmaxf(top, m[n][e]);
                        const float f = m[n][e] == top ? 1.f : ex2(m[n][e] - top);
                        m[n][e] = top;
                        l[n][e] *= f;
#pragma unroll
                        for (int c = 0; c < KS; ++c) {
                            o[n][c][e] *= f;
                            o[n][c][e + 2] *= f;
                        }
                    }
            }
            uint32_t b[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = ex2(x[n][e] - (m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1] - kUp));
                    l[n][e & 1] += w[e];
                }
                b[n][0] = transposed(E == 1 ? f2_h2(w[0], w[1]) : f2_bf2(w[0], w[1]));
                b[n][1] = transposed(E == 1 ? f2_h2(w[2], w[3]) : f2_bf2(w[2], w[3]));
            }
            if constexpr (E == 2) {
#pragma unroll
                for (int h = 0; h < D / 64; ++h) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const uint4*>(vt + piece<C::ROW>(2 * j + (k & 1) + 8 * (k >> 1), 8 * h + g));
                    const uint32_t* w[4] = {&v[0].x, &v[1].x, &v[2].x, &v[3].x};
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t a0 = __byte_perm(w[0][u], w[1][u], 0x5410), a1 = __byte_perm(w[0][u], w[1][u], 0x7632);
                        const uint32_t a2 = __byte_perm(w[2][u], w[3][u], 0x5410), a3 = __byte_perm(w[2][u], w[3][u], 0x7632);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816_bf16(o[n][4 * h + u], a0, a1, a2, a3, b[n][0], b[n][1]);
                    }
                }
            } else if constexpr (D == 64) {
                uint2 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const uint2*>(vt + piece<C::ROW>(2 * j + (k & 1) + 8 * (k >> 1), g >> 1) + 8 * (g & 1));
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t w0 = u < 2 ? v[0].x : v[0].y, w1 = u < 2 ? v[1].x : v[1].y, w2 = u < 2 ? v[2].x : v[2].y, w3 = u < 2 ? v[3].x : v[3].y;
                    const int pick = u & 1 ? 0x7362 : 0x5140;
                    uint32_t a0, a1, a2, a3;
                    e4m3_f16(__byte_perm(w0, w1, pick), a0, a1);
                    e4m3_f16(__byte_perm(w2, w3, pick), a2, a3);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816(o[n][u], a0, a1, a2, a3, b[n][0], b[n][1], vs);
                }
            } else {
#pragma unroll
                for (int h = 0; h < D / 128; ++h) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const uint4*>(vt + piece<C::ROW>(2 * j + (k & 1) + 8 * (k >> 1), 8 * h + g));
                    const uint32_t* w[4] = {&v[0].x, &v[1].x, &v[2].x, &v[3].x};
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int pick = u & 1 ? 0x7362 : 0x5140;
                        uint32_t a0, a1, a2, a3;
                        e4m3_f16(__byte_perm(w[0][u >> 1], w[1][u >> 1], pick), a0, a1);
                        e4m3_f16(__byte_perm(w[2][u >> 1], w[3][u >> 1], pick), a2, a3);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma16816(o[n][8 * h + u], a0, a1, a2, a3, b[n][0], b[n][1], vs);
                    }
                }
            }
            __syncwarp();                                      // the ring's place is read before it is filled again
        }
        cp_wait<0>();
        // ------------------------------------------------------------ the warps meet
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int b = 4; b < 32; b <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], b);
                if (g == 0) {
                    wm[warp * C::ROWS + 8 * n + 2 * j + e] = m[n][e] - kUp;
                    wl[warp * C::ROWS + 8 * n + 2 * j + e] = l[n][e];
                }
            }
        __syncthreads();                                       // every ring is done
        // a lane's numbers of a row are neighbours, 8 of them a piece (16 over 8 bits, but for D 64); every
        // other lane's 16-byte words change places, so that a quarter warp meets all banks
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float* row = meet + (warp * C::ROWS + 8 * n + 2 * j + e) * C::PITCH;
#pragma unroll
                for (int c = 0; c < KS; c += 2) {
                    const int d4 = SIXTEEN ? 32 * (c >> 3) + 4 * g + (c & 7) / 2 : 16 * (c >> 2) + 2 * g + (c & 3) / 2;
                    *reinterpret_cast<float4*>(row + 4 * (d4 ^ (g & 1))) =
                        make_float4(o[n][c][e], o[n][c][e + 2], o[n][c + 1][e], o[n][c + 1][e + 2]);
                }
            }
        __syncthreads();
        const int64_t slot = 2 * cta + (seg == waves ? 0 : 1);
        for (int it = tid; it < rows * (D / 4); it += kThreads) {
            const int r = it % rows, d4 = it / rows;           // rows fastest, as in the partials
            float top = -INFINITY, lt = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, wm[w * C::ROWS + r]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            const int gw = SIXTEEN ? d4 >> 2 : d4 >> 1;        // the lane that wrote it
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float mw = wm[w * C::ROWS + r];
                const float f = mw == -INFINITY ? 0.f : ex2(mw - top);
                const float4 v = *reinterpret_cast<const float4*>(meet + (w * C::ROWS + r) * C::PITCH + 4 * (d4 ^ (gw & 1)));
                lt += f * wl[w * C::ROWS + r];
                acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            }
            if (full) {
                const float inv = 1.f / lt;                    // a row sees itself
                __nv_bfloat16* dst = p.out + ((int64_t)(ch.tail_off + T.tok0 + r / p.g) * p.Hq + T.kvh * p.g + r % p.g) * D + 4 * d4;
                *reinterpret_cast<uint2*>(dst) = make_uint2(f2_bf2(acc.x * inv, acc.y * inv), f2_bf2(acc.z * inv, acc.w * inv));
            } else {
                reinterpret_cast<float4*>(p.part_o + (slot * (D / 32) + d4 / 8) * 8 * BM * 4)[d4 % 8 * BM + r] = acc;
                if (d4 == 0) {
                    p.part_ml[(slot * BM + r) * 2] = lt == lt ? top : 0.f;   // a query that is not finite: NaN, not nothing
                    p.part_ml[(slot * BM + r) * 2 + 1] = lt;
                }
            }
        }
        __syncthreads();                                       // before the next segment fills the rings
    }
}

template <int D, int NT, int E>
void launch(const DecodeParams& p, cudaStream_t s) {
    using C = Cfg<D, NT, E>;
    static unsigned long long configured = 0;   // one bit per device
    int dev = 0;
    cudaGetDevice(&dev);
    if (!(configured >> (dev & 63) & 1ull)) {
        cudaFuncSetAttribute(decode_attention_kernel<D, NT, E>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        configured |= 1ull << (dev & 63);
    }
    launch_pdl(decode_attention_kernel<D, NT, E>, dim3(p.a.n_ctas), dim3(C::THREADS), C::SMEM, s, p);
}

template <int D>
void launch_d(const DecodeParams& p, cudaStream_t s) {
    if (p.from.K) p.rows <= 8 ? launch<D, 1, 1>(p, s) : launch<D, 2, 1>(p, s);
    else p.rows <= 8 ? launch<D, 1, 2>(p, s) : launch<D, 2, 2>(p, s);
}

}  // namespace

void launch_decode_attention(const DecodeParams& p, cudaStream_t s) {
    if (p.a.n_ctas <= 0) return;
    if (p.a.D == 64) launch_d<64>(p, s);
    else if (p.a.D == 128) launch_d<128>(p, s);
    else launch_d<256>(p, s);
}

}  // namespace kvm
