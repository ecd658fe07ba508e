// Codes of the paged cache to fp16, two at a time.  A field of b bits at bit s of a 16-bit half, or-ed into the pattern of
// 1024 (0x6400), is the fp16 number 1024 + u 2^s as long as s + b <= 10; one fused multiply-add by 2^-s brings it to u minus
// the code's offset, exactly.  Fields further up come down with one shift per word first.
#pragma once

#include <cuda_fp16.h>

#include "paged.cuh"

namespace a48p {

// the 32-bit word (x & mask) | 0x64006400 in one instruction
__device__ __forceinline__ uint32_t magic(uint32_t x, uint32_t mask) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "n"(0x64006400));
    return r;
}
template <int S>
__device__ __forceinline__ uint32_t fields(uint32_t word, uint32_t mask, int offset) {
    const uint32_t x = magic(word, mask << S);
    const __half2 mul = __half2half2(__float2half(1.f / (1 << S))), add = __half2half2(__float2half(-(1024.f / (1 << S)) - offset));
    const __half2 r = S == 0 ? __hadd2(*reinterpret_cast<const __half2*>(&x), add)
                             : __hfma2(*reinterpret_cast<const __half2*>(&x), mul, add);
    return *reinterpret_cast<const uint32_t*>(&r);
}
// the four 4-bit fields of both halves of a word, lowest first
__device__ __forceinline__ void nibbles(uint32_t w, uint32_t* out) {
    out[0] = fields<0>(w, 0x000f000fu, 8);
    out[1] = fields<4>(w, 0x000f000fu, 8);
    w >>= 8;
    out[2] = fields<0>(w, 0x000f000fu, 8);
    out[3] = fields<4>(w, 0x000f000fu, 8);
}
// the two bytes of both halves
__device__ __forceinline__ void bytes(uint32_t w, uint32_t* out) {
    out[0] = fields<0>(w, 0x00ff00ffu, 128);
    out[1] = fields<0>(w >> 8, 0x00ff00ffu, 128);
}
// the five 3-bit fields of both halves of three words, and the sixteenth from their top bits
__device__ __forceinline__ void triples(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t* out) {
    const uint32_t w[3] = {w0, w1, w2};
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        out[5 * j] = fields<0>(w[j], 0x00070007u, 4);
        out[5 * j + 1] = fields<3>(w[j], 0x00070007u, 4);
        out[5 * j + 2] = fields<6>(w[j], 0x00070007u, 4);
        const uint32_t up = w[j] >> 9;
        out[5 * j + 3] = fields<0>(up, 0x00070007u, 4);
        out[5 * j + 4] = fields<3>(up, 0x00070007u, 4);
    }
    const uint32_t top = ((w0 >> 15) & 0x00010001u) | ((w1 >> 14) & 0x00020002u) | ((w2 >> 13) & 0x00040004u);
    out[15] = fields<0>(top, 0x00070007u, 4);
}

// The same fields as they are: u 2^s in the mantissa of a subnormal fp16 number, u 2^(s-24).  One mask per pair; the offset and
// the 2^(s-24) are the other operand's.
__device__ __forceinline__ void raw_nibbles(uint32_t w, uint32_t* out) {
    out[0] = w & 0x000f000fu;
    out[1] = w & 0x00f000f0u;
    w >>= 8;
    out[2] = w & 0x000f000fu;
    out[3] = w & 0x00f000f0u;
}
__device__ __forceinline__ void raw_bytes(uint32_t w, uint32_t* out) {
    out[0] = w & 0x00ff00ffu;
    out[1] = (w >> 8) & 0x00ff00ffu;
}
__device__ __forceinline__ void raw_triples(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t* out) {
    const uint32_t w[3] = {w0, w1, w2};
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        out[5 * j] = w[j] & 0x00070007u;
        out[5 * j + 1] = w[j] & 0x00380038u;
        out[5 * j + 2] = w[j] & 0x01c001c0u;
        const uint32_t up = w[j] >> 9;
        out[5 * j + 3] = up & 0x00070007u;
        out[5 * j + 4] = up & 0x00380038u;
    }
    out[15] = ((w0 >> 15) & 0x00010001u) | ((w1 >> 14) & 0x00020002u) | ((w2 >> 13) & 0x00040004u);
}
// s of the i-th word that they give
template <int BITS>
__device__ __forceinline__ constexpr int raw_shift(int i) {
    return BITS == 8 ? 0 : BITS == 4 ? 4 * (i & 1) : i == 15 ? 0 : i % 5 < 3 ? 3 * (i % 5) : 3 * (i % 5 - 3);
}

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// The e that brings the largest of some query entries (finite, as bits) to [2^14, 2^15), fp16's top; entries below fp32's
// normal numbers go as far as they go (their scores are nothing).
__device__ __forceinline__ int query_exponent(uint32_t top) { return top ? 14 + 127 - (int)(top >> 23) : 0; }
// A kernel argument kept in a register: read in a loop it would come from the constant bank again and again, which the
// loop's own code keeps pushing out of the cache (measured: 0.5k clocks a tile of the tile kernel).
__device__ __forceinline__ int in_register(int x) {
    asm volatile("" : "+r"(x));
    return x;
}

// 2^x, two units in the last place at most; 2^-inf = 0
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace a48p
