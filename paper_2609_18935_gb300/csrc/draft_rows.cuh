// A drafted node's key and value on their way into the caches.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

namespace kvm {

// bf16 elements that are not finite become 0; true if there was one.  A tile's weight
// of 0 for a value out of sight would turn it into a NaN of every row, in later calls
// too while the slot lies in their last tile.
__device__ __forceinline__ bool clear_not_finite(uint4& v) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
        w[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
        bad = bad || lo || hi;
    }
    return bad;
}

__device__ __forceinline__ bool clear_not_finite(__nv_bfloat16& v) {
    const bool bad = (__bfloat16_as_ushort(v) & 0x7f80) == 0x7f80;
    if (bad) v = __ushort_as_bfloat16(0);
    return bad;
}

// Eight elements of a key and those `half` further on, rotated by the (cos, sin) of
// their pairs.  store: true if one was not finite (and went in as 0).
struct TurnedNode {
    uint4 a, y;
    float4 t[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* src, int half, const float2* turn) {
        a = *reinterpret_cast<const uint4*>(src);
        y = *reinterpret_cast<const uint4*>(src + half);
#pragma unroll
        for (int q = 0; q < 4; ++q) t[q] = reinterpret_cast<const float4*>(turn)[q];
    }
    __device__ __forceinline__ bool store(__nv_bfloat16* dst, int half) {
        const bool first = clear_not_finite(a), bad = clear_not_finite(y) || first;
        __nv_bfloat162* u = reinterpret_cast<__nv_bfloat162*>(&a);
        __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(&y);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 f = __bfloat1622float2(u[q]), s = __bfloat1622float2(w[q]);
            u[q] = __floats2bfloat162_rn(f.x * t[q].x - s.x * t[q].y, f.y * t[q].z - s.y * t[q].w);
            w[q] = __floats2bfloat162_rn(s.x * t[q].x + f.x * t[q].y, s.y * t[q].z + f.y * t[q].w);
        }
        *reinterpret_cast<uint4*>(dst) = a;
        *reinterpret_cast<uint4*>(dst + half) = y;
        return bad;
    }
};

}  // namespace kvm
