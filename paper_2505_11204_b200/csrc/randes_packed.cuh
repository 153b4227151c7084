// Device helpers shared by the kernels that read packed weights: the decoding of codes, activations, bulk copies and
// bounded waits. The layout of a packed matrix is described in randes_packed.cu.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "randes_device.cuh"
#include "randes_internal.h"

namespace randes {
namespace device {

// The four operand registers of one word of codes, as q / 64. A code left in the low byte of a bf16 is a number too: bf16
// counts in steps of 2^-133 through its whole first two binades, so bits 0-3 read u 2^-133 and bits 4-7 read 16 u 2^-133
// (u = q + 8). One exact multiply-add brings either to u / 64 - 1/8. So a word takes one shift instead of three, and no
// bias has to be put in. Parts of 1/64, not units: a product with an activation cannot overflow where the weight itself
// (q s, with s << 1) would not; the factor comes back with the partial sums.
constexpr float kCodeUnit = 64.f;
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ void decode(uint32_t word, uint32_t (&a)[4])
{
    constexpr uint32_t k127 = 0x7F007F00u, k123 = 0x7D007D00u, kOff = 0xBE00BE00u;    // 2^127, 2^123, -1/8, twice each
    const uint32_t high = word >> 8;
    a[0] = fma_bf16x2(word & 0x000F000Fu, k127, kOff);
    a[1] = fma_bf16x2(word & 0x00F000F0u, k123, kOff);
    a[2] = fma_bf16x2(high & 0x000F000Fu, k127, kOff);
    a[3] = fma_bf16x2(high & 0x00F000F0u, k123, kOff);
}

// Activations: a lane's eight neighbouring columns of one token, as loaded and as four words of bf16 pairs. An fp32
// activation becomes three bf16 terms by truncation (8 + 8 + 8 bits: their sum is the fp32 value exactly, down to where the
// last term underflows), so that products and sums keep fp32's accuracy on the bf16 tensor core.
template <typename XT> struct Acts;
template <> struct Acts<bf16> {
    static constexpr int kTerms = 1;
    struct Raw { uint4 r[1]; };
    static __device__ __forceinline__ Raw words(const bf16* p) { return Raw{{__ldg(reinterpret_cast<const uint4*>(p))}}; }
    static __device__ __noinline__ Raw gather(const bf16* p, uint32_t c, uint32_t cols)      // element by element
    {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = c + 2 * e < cols ? __ldg(q + c + 2 * e) : 0u, hi = c + 2 * e + 1 < cols ? __ldg(q + c + 2 * e + 1) : 0u;
            w[e] = lo | (hi << 16);
        }
        return Raw{{make_uint4(w[0], w[1], w[2], w[3])}};
    }
    static __device__ __forceinline__ Raw zero() { return Raw{{make_uint4(0, 0, 0, 0)}}; }
    static __device__ __forceinline__ void terms(const Raw& v, uint32_t (&w)[1][4])
    {
        w[0][0] = v.r[0].x; w[0][1] = v.r[0].y; w[0][2] = v.r[0].z; w[0][3] = v.r[0].w;
    }
};
template <> struct Acts<float> {
    static constexpr int kTerms = 3;
    struct Raw { uint4 r[2]; };
    static __device__ __forceinline__ Raw words(const float* p)
    {
        return Raw{{__ldg(reinterpret_cast<const uint4*>(p)), __ldg(reinterpret_cast<const uint4*>(p) + 1)}};
    }
    static __device__ __noinline__ Raw gather(const float* p, uint32_t c, uint32_t cols)
    {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = c + e < cols ? __float_as_uint(__ldg(p + c + e)) : 0u;
        return Raw{{make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7])}};
    }
    static __device__ __forceinline__ Raw zero() { return Raw{{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)}}; }
    static __device__ __forceinline__ void terms(const Raw& v, uint32_t (&w)[3][4])
    {
        float f[8] = {__uint_as_float(v.r[0].x), __uint_as_float(v.r[0].y), __uint_as_float(v.r[0].z), __uint_as_float(v.r[0].w),
                      __uint_as_float(v.r[1].x), __uint_as_float(v.r[1].y), __uint_as_float(v.r[1].z), __uint_as_float(v.r[1].w)};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = f[2 * e], b = f[2 * e + 1];
                w[k][e] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
                const float ta = __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), tb = __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
                f[2 * e] = a == ta ? 0.f : a - ta;           // the comparison keeps an infinity out of the lower terms
                f[2 * e + 1] = b == tb ? 0.f : b - tb;
            }
        }
    }
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Tries of a wait. One that is not answered sleeps for 4 us (measured on a barrier that nothing completes), so a wait gives up
// after about a second, far beyond any copy; 2^22 of them would be 17.
constexpr uint32_t kWaitLimit = 1u << 18;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i)
        if (bar_try(bar, parity)) return true;
    return false;
}

}  // namespace device
}  // namespace randes
