// The 8-bit activation checkpoint: int8 codes and one scale byte per block of 32 consecutive channels of a pixel.
//   amax = largest |x| of the block, e = the smallest integer in [-127, 121] with rint(amax / 2^e) <= 127, 121 if there is none (the largest
//   bf16 is 127.5 * 2^121), code = rint(x / 2^e) (ties to even) within [-127, 127], scale byte = e + 127. A block that holds an infinity or a NaN: scale byte 255, codes 0; it stands for NaN.
// The scale is a power of two, so that the division is exact and a code is one rounding of x, the same wherever it is computed; a value
// code * 2^e has 7 significant bits, so that it is exact in bf16. (A scale of amax / 127 would make the steps 1.4 times finer on average,
// and codes would depend on how the quotient is rounded.)
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace act8 {

constexpr int kBlock = 32;                   // channels of a block
constexpr uint32_t kBad = 255;               // scale byte of a block that stands for NaN
constexpr uint32_t kTop = 248;               // largest scale byte of any other

__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = __bfloat1622float2(h[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    uint4 v;
    __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    return v;
}

// The bits to keep of the vector of channels c0 .. c0 + 7 of C: pad lanes come out as zeros.
__device__ __forceinline__ uint4 keep_bits(int c0, int C)
{
    uint32_t k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = (c0 + 2 * j < C ? 0xffffu : 0u) | (c0 + 2 * j + 1 < C ? 0xffff0000u : 0u);
    return make_uint4(k[0], k[1], k[2], k[3]);
}

__device__ __forceinline__ uint4 and4(const uint4 &a, const uint4 &b) { return make_uint4(a.x & b.x, a.y & b.y, a.z & b.z, a.w & b.w); }

// Largest magnitude of eight bf16 values, as the bits of a positive bf16 (a NaN's bits are above infinity's).
__device__ __forceinline__ uint32_t amax8(const uint4 &v)
{
    const uint32_t m = 0x7fff7fffu;
    const uint32_t t = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
    const uint32_t lo = t & 0xffffu, hi = t >> 16;
    return lo > hi ? lo : hi;
}

// Scale byte from those bits: the exponent field of amax less 6, one more where the significand is 255/128 (which would round to 128).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax)
{
    if (amax >= 0x7f80u) return kBad;
    const int b = (int)((amax + 1u) >> 7) - 6;
    return b <= 0 ? 0u : b > (int)kTop ? kTop : (uint32_t)b;
}

// Eight codes. 1.5 * 2^23 added: the low byte of the sum is x / 2^e rounded to the nearest even integer (the product is exact).
__device__ __forceinline__ uint2 encode8(const uint4 &v, uint32_t byte)
{
    if (byte == kBad) return make_uint2(0u, 0u);
    const float inv = __uint_as_float((254u - byte) << 23);
    float f[8];
    unpack8(v, f);
    uint32_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(fmaf(f[j], inv, 12582912.f));
    if (byte == kTop)                                            // (only here may a value be as large as 127.5 steps)
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(fminf(fmaxf(__uint_as_float(r[j]), 12582912.f - 127.f), 12582912.f + 127.f));
    uint2 q;
    q.x = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
    q.y = __byte_perm(__byte_perm(r[4], r[5], 0x0040), __byte_perm(r[6], r[7], 0x0040), 0x5410);
    return q;
}

__device__ __forceinline__ float scale_of(uint32_t byte)
{
    return __uint_as_float(byte == 0u ? 0x00400000u : byte == kBad ? 0x7fc00000u : byte << 23);
}

// The eight values. A code's byte, its sign bit flipped, behind the exponent of 2^23 is the number 2^23 + 128 + code.
__device__ __forceinline__ void decode8(const uint2 &q, uint32_t byte, float (&f)[8])
{
    const float s = scale_of(byte);
    const uint32_t a = q.x ^ 0x80808080u, b = q.y ^ 0x80808080u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[j] = (__uint_as_float(__byte_perm(a, 0x4b000000u, 0x7440 + j)) - 8388736.f) * s;
        f[4 + j] = (__uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440 + j)) - 8388736.f) * s;
    }
}

// Largest of `w` neighbouring lanes (1, 2 or 4, aligned): the lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t a, int w)
{
    if (w > 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    if (w > 2) a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
    return a;
}

}  // namespace act8
