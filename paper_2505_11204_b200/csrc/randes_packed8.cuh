// Eight-bit blocks on the device: the scale of a block, codes of its elements, and where they lie.
#pragma once

#include <cuda_fp16.h>

#include "randes_device.cuh"

namespace randes {
namespace device {

constexpr uint32_t kNotFinite = 0x7F800000u;      // a greatest magnitude (as bits) from here on: the block holds a NaN or an infinity

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Exponent + 127 of the least power of two, 2^-100 at least, that takes the block's greatest magnitude to 448 = 1.75 * 2^8 or below:
// the carry out of the mantissa says whether that lies above 1.75. A block that holds a NaN or an infinity: 1 (its codes are NaN).
__device__ __forceinline__ uint32_t block_scale(uint32_t amax)
{
    const uint32_t e = ((amax + 0x1FFFFFu) >> 23) - 8;
    return amax >= kNotFinite ? 127u : (amax < (27u + 8u) << 23 ? 27u : e);
}
// what elements are multiplied by, exactly, before they are rounded to a code (254 - e is in 7 .. 227), and what a code counts
__device__ __forceinline__ float block_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }
__device__ __forceinline__ float block_unit(uint32_t e) { return __uint_as_float(e << 23); }

// Four codes (e4m3, nearest even), the first in the low byte.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
constexpr uint32_t kNanCodes = 0x7F7F7F7Fu;
__device__ __forceinline__ uint2 codes8(const float (&v)[8], uint32_t amax, uint32_t e)
{
    const float s = block_inverse(e);
    if (amax >= kNotFinite) return make_uint2(kNanCodes, kNanCodes);
    return make_uint2(codes4(v[0] * s, v[1] * s, v[2] * s, v[3] * s), codes4(v[4] * s, v[5] * s, v[6] * s, v[7] * s));
}
// The four values behind a word of codes, exact (an e4m3 value is a half), times the block's unit.
__device__ __forceinline__ void values4(uint32_t w, float unit, float* v)
{
    uint32_t lo, hi;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"(static_cast<uint16_t>(w)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"(static_cast<uint16_t>(w >> 16)));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    v[0] = a.x * unit; v[1] = a.y * unit; v[2] = b.x * unit; v[3] = b.y * unit;
}

// Byte offset of column c (a multiple of 8) of a row inside its tile: 16-byte pieces in the order that the tensor core's
// 128-byte swizzle wants, so that a tile goes into shared memory by a plain copy.
__device__ __forceinline__ uint32_t code_at(uint32_t r, uint32_t c) { return (r & 127) * 128 + ((((c >> 4) & 7) ^ (r & 7)) << 4) + (c & 8); }

// Element access of rows in memory, eight neighbouring columns to a lane.
template <typename T> struct Octet { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ void widen(const Octet<T>& o, float (&v)[8])
{
#pragma unroll
    for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) {
        float u[Store<T>::CPL];
        Store<T>::widen(o.w[h], u);
#pragma unroll
        for (int e = 0; e < Store<T>::CPL; ++e) v[h * Store<T>::CPL + e] = u[e];
    }
}
template <typename T> __device__ __forceinline__ Octet<T> narrow(const float (&v)[8]);
template <> __device__ __forceinline__ Octet<float> narrow<float>(const float (&v)[8])
{
    Octet<float> o;
    o.w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    o.w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    return o;
}
template <> __device__ __forceinline__ Octet<bf16> narrow<bf16>(const float (&v)[8])
{
    Octet<bf16> o;
    o.w[0] = make_uint4(Out<bf16>::pack(v[0], v[1]), Out<bf16>::pack(v[2], v[3]), Out<bf16>::pack(v[4], v[5]), Out<bf16>::pack(v[6], v[7]));
    return o;
}
// columns c .. c + 7 of a row on a 16-byte boundary; zero beyond the row's end
template <typename T> __device__ __forceinline__ Octet<T> load_octet(const T* row, uint32_t c, uint32_t cols)
{
    Octet<T> o;
    if (c + 8 <= cols) {
#pragma unroll
        for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) o.w[h] = __ldcs(reinterpret_cast<const uint4*>(row + c) + h);
    } else {
        float v[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) v[e] = c + e < cols ? Store<T>::load1(row + c + e) : 0.f;
        o = narrow<T>(v);
    }
    return o;
}
template <typename T> __device__ __forceinline__ void store_octet(T* row, uint32_t c, uint32_t cols, const float (&v)[8])
{
    if (c + 8 <= cols) {
        const Octet<T> o = narrow<T>(v);
#pragma unroll
        for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) reinterpret_cast<uint4*>(row + c)[h] = o.w[h];
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            if (c + e < cols) Out<T>::store1(row + c + e, v[e]);
    }
}
// Rows that start anywhere: a warp's run of 256 columns, lane l holding columns l, l + 32 .. l + 224, so that memory is read and
// written by neighbours together, one element to a lane and instruction.
template <typename T> __device__ __forceinline__ void load_strided(const T* row, uint32_t first, uint32_t cols, int lane, float (&v)[8])
{
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        const uint32_t at = first + 32 * k + lane;
        v[k] = at < cols ? Store<T>::load1(row + at) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void store_strided(T* row, uint32_t first, uint32_t cols, int lane, const float (&v)[8])
{
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
        const uint32_t at = first + 32 * k + lane;
        if (at < cols) Out<T>::store1(row + at, v[k]);
    }
}

// A warp's 256 columns of row r, from column `first` on, into eight bits; returns the scales of its two blocks (the second in bits 8-15).
// OCTETS: lane l holds columns 8 l .. 8 l + 7; otherwise l, l + 32 ...
template <bool OCTETS> __device__ __forceinline__ uint32_t pack_run(char* dst, const Packed8Layout& lay, uint32_t r, uint32_t first, const float (&v)[8], int lane)
{
    if (OCTETS) {
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_bits(amax, magnitude(v[e]));
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) amax = max_bits(amax, __shfl_xor_sync(~0u, amax, o));
        const uint32_t c = first + 8 * lane, kb = c >> 7, e = block_scale(amax);
        if (kb < lay.col_blocks) *reinterpret_cast<uint2*>(dst + lay.tile(r >> 7, kb) + code_at(r, c)) = codes8(v, amax, e);
        return __shfl_sync(~0u, e, 0) | (__shfl_sync(~0u, e, 16) << 8);
    }
    uint32_t scales = 0;
#pragma unroll
    for (uint32_t b = 0; b < 2; ++b) {
        const uint32_t kb = (first >> 7) + b;
        if (kb >= lay.col_blocks) break;
        uint32_t amax = 0;
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) amax = max_bits(amax, magnitude(v[4 * b + e]));
        amax = __reduce_max_sync(~0u, amax);
        const uint32_t s = block_scale(amax);
        const float inv = block_inverse(s);
        const uint32_t w = amax >= kNotFinite ? kNanCodes : codes4(v[4 * b] * inv, v[4 * b + 1] * inv, v[4 * b + 2] * inv, v[4 * b + 3] * inv);
        char* to = dst + lay.tile(r >> 7, kb) + (r & 127) * 128 + (lane & 15);
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) to[((2 * e + (lane >> 4)) ^ (r & 7)) << 4] = static_cast<char>(w >> (8 * e));
        scales |= s << (8 * b);
    }
    return scales;
}
// and its scales, where no word of four blocks is at hand
__device__ __forceinline__ void store_scales(char* dst, const Packed8Layout& lay, uint32_t r, uint32_t first, uint32_t scales, int lane)
{
    const uint32_t kb = (first >> 7) + lane;
    if (lane < 2 && kb < lay.col_blocks) dst[lay.scales(r >> 7, kb >> 2) + Packed8Layout::scale_word(r) + (kb & 3)] = static_cast<char>(scales >> (8 * lane));
}

}  // namespace device
}  // namespace randes
