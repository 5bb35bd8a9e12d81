// Numbers of a cache in 8 bits.
//
// A block is 64 slots of one KV head, of K or of V.  Its numbers are e4m3 times 2^e, e
// the smallest integer (and at least -117, so that 2^(e-9) is a normal float) with
// max |x| <= 448 * 2^e (and at most 119: what is beyond 448 * 2^119, a bf16 number,
// becomes that); x becomes the nearest multiple of the grid, ties to even.  The
// scale is a power of two so that numbers of one block carry over into another (a
// removal, a token appended to a half-filled block) as they are: with a larger scale
// only what falls below 2^-6 of it is rounded again, by at most 2^-10 of the scale
// where the block's largest number is over 224 of it.  A scale of max / 448 would use the
// last bit of range better (at most a factor 2 of 2^17) and round every survivor of a
// removal again, to 2^-4 of its value.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

namespace kvm {

// The exponent e of a block whose largest magnitude is amax (finite).
__device__ __forceinline__ int kv8_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    // amax = m 2^E with m in [1/2, 1): 448 = 7/8 2^9
    const int E = (int)(b >> 23) - 126;
    return min(max(E - 9 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), -117), 119);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Four floats as e4m3, in order from the lowest byte (to the nearest, ties to even).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}

// Two e4m3 numbers as bf16, exactly: bytes n and m of the eight of (lo, hi), each beside
// eight copies of its sign (a selector's bit 3), move up four bits into sign, exponent
// and mantissa: the number times 2^-120, a subnormal one as a subnormal.  The product
// undoes that.
__device__ __forceinline__ constexpr uint32_t e4m3_pick(int n, int m) { return n | (8 + n) << 4 | m << 8 | (8 + m) << 12; }
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t lo, uint32_t hi, uint32_t pick) {
    uint32_t x;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(x) : "r"(lo), "r"(hi), "r"(pick));
    x = x << 4 & 0x87f087f0u;
    const uint32_t k = 0x7b807b80u;                          // 2^120
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&k));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// The low and the high two numbers of a word.
__device__ __forceinline__ uint32_t e4m3_low(uint32_t w) { return e4m3_pair(w, w, e4m3_pick(0, 1)); }
__device__ __forceinline__ uint32_t e4m3_high(uint32_t w) { return e4m3_pair(w, w, e4m3_pick(2, 3)); }

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

// Eight numbers as bf16, times a block's scale (exactly: see the least exponent above).
// Eight, not sixteen: 32 bytes a thread, in two stores, filled every sector by halves (the
// widening of a round's two layers took 35.0 us against 30.4).
__device__ __forceinline__ uint4 widen8(const uint2& w, __nv_bfloat162 scale) {
    auto pair = [&](uint32_t x) {
        const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&x), scale);
        return *reinterpret_cast<const uint32_t*>(&r);
    };
    return make_uint4(pair(e4m3_low(w.x)), pair(e4m3_high(w.x)), pair(e4m3_low(w.y)), pair(e4m3_high(w.y)));
}

// Largest magnitude of sixteen numbers, as their bytes' order has it.
__device__ __forceinline__ float e4m3_max(const uint4& w) {
    const uint32_t k = 0x007f007fu;
    const uint32_t m = __vmaxu2(__vmaxu2(__vmaxu2(w.x & k, w.y & k), __vmaxu2(w.z & k, w.w & k)),
                                __vmaxu2(__vmaxu2(w.x >> 8 & k, w.y >> 8 & k), __vmaxu2(w.z >> 8 & k, w.w >> 8 & k)));
    return __uint_as_float(e4m3_low(max(m & 0xffffu, m >> 16)) << 16);
}

// Eight (sixteen) numbers of scale `from` under the scale whose reciprocal is `inv`.
__device__ __forceinline__ uint2 requantised(const uint2& w, float from, float inv) {
    auto word = [&](uint32_t x) {
        const uint32_t lo = e4m3_low(x), hi = e4m3_high(x);
        auto f = [&](uint32_t bits) { return __uint_as_float(bits) * from * inv; };
        return to_e4m3(f(lo << 16), f(lo & 0xffff0000u), f(hi << 16), f(hi & 0xffff0000u));
    };
    return make_uint2(word(w.x), word(w.y));
}
__device__ __forceinline__ uint4 requantised(const uint4& w, float from, float inv) {
    const uint2 a = requantised(make_uint2(w.x, w.y), from, inv), b = requantised(make_uint2(w.z, w.w), from, inv);
    return make_uint4(a.x, a.y, b.x, b.y);
}

}  // namespace kvm
