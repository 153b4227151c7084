// Weights in four bits with group scales: written from a weight (or straight from base and superposition), read
// back, and applied to a few tokens.
//
// Per group of g = 32, 64 or 128 columns of a row (the last group of a row may be shorter), with a = max |w|:
//     s = bf16( fl(a / 7) )      0 where that is below 2^-100;  NaN where the group holds a NaN or an infinity
//     q = rint( fl(w / s) )      in [-7, 7]: s is at most 2^-9 (relative) below a / 7, so |w / s| <= 7.02
//     the four bits stand for q * s.
// The scale is bf16 because it then has fp32's range (no group can overflow or needs a global factor) at two bytes,
// and q is taken against the rounded scale, so the rounding costs no accuracy of its own. The clamp of the definition
// never acts for the reason given above.
//
// Layout: records of 64 rows x 64 columns (128 columns for groups of 128), [row block][column block], each
//     codes   [tile of 64 columns][row tile of 16][lane] 16 bytes
//     scales  [group][row tile][lane / 4] one word: rows g (low half) and g + 8 (high half) of the row tile
// so that the columns one warp works through are one contiguous run of memory -- one bulk copy per stage -- and one
// 16-byte load per lane brings the A operands of four m16n8k16 products in the order the tensor core wants them.
// Lane (g = lane / 4, t = lane % 4) holds rows g and g + 8. Its 32-bit word j holds the four columns
//     c(j, e) = 32 (j / 2) + 8 t + 4 (j % 2) + e,    e = 0 .. 3
// of both rows, code + 8 in nibble order (g,0) (g+8,0) (g,2) (g+8,2) (g,1) (g+8,1) (g,3) (g+8,3): shifting the word by
// 4 i and masking with 0x000F000F leaves operand register i. The columns a lane owns are 8 neighbours in each half of
// the tile, so that the activations it multiplies are two 16-byte loads.
#include <cuda_bf16.h>
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>

#include "randes_packed.cuh"

namespace cg = cooperative_groups;

namespace randes {

static __device__ unsigned int g_packed_giveups;   // warps that gave up waiting for a copy (0 in a healthy run)

namespace {

using namespace device;

constexpr int kPackWarps = 4;                 // warps per CTA of the pack and unpack kernels (8: up to a tenth slower)
constexpr float kMinScale = 0x1p-100f;        // far enough from the subnormals for the quotient below to be exact

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// w / s correctly rounded, given inv = fl(1 / s): one Newton step on the quotient (Markstein 1990). No operand or
// residual leaves the normal range: s >= 2^-100 and |w| <= 7.02 s.
__device__ __forceinline__ float quotient(float w, float s, float inv)
{
    const float q = w * inv;
    return __fmaf_rn(__fmaf_rn(-q, s, w), inv, q);
}
__device__ __forceinline__ f32x2 quotient2(f32x2 w, f32x2 neg_s, f32x2 inv)
{
    const f32x2 q = mul2(w, inv);
    return fma2(fma2(q, neg_s, w), inv, q);
}
__device__ __forceinline__ f32x2 twice(float x) { return pack2(__float_as_uint(x), __float_as_uint(x)); }

// Eight neighbouring columns of one row as they lie in memory.
template <typename T> struct Eight { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Eight<T> load8(const T* p)
{
    Eight<T> v;
#pragma unroll
    for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) v.w[h] = __ldcs(reinterpret_cast<const uint4*>(p) + h);
    return v;
}
template <typename T> __device__ __noinline__ Eight<T> gather8(const T* row, uint32_t c, uint32_t cols)      // zero beyond the row's end
{
    Eight<T> v;
    T e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = c + k < cols ? row[c + k] : T(0.f);
    memcpy(&v, e, sizeof v);
    return v;
}
template <typename T> __device__ __forceinline__ void widen8(const Eight<T>& r, float (&v)[8])
{
#pragma unroll
    for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) {
        float u[Store<T>::CPL];
        Store<T>::widen(r.w[h], u);
#pragma unroll
        for (int e = 0; e < Store<T>::CPL; ++e) v[h * Store<T>::CPL + e] = u[e];
    }
}

// Rows that do not start on 16-byte boundaries go through shared memory, element by element but neighbours together: a warp's
// 16 x 128 tile, rows a little apart so that the lanes' 16-byte accesses fall into different banks. (Each lane touching its
// own eight columns in memory took 71 us instead of 12 to unpack 4001 x 4001 bf16, retrieve-and-pack 43 instead of 25.)
template <typename T> struct Tile {
    static constexpr uint32_t kPitch = 128 * sizeof(T) + 16;
    static constexpr uint32_t kBytes = 16 * kPitch;
};
template <typename T>
__device__ __forceinline__ void tile_in(unsigned char* tile, const T* m, uint64_t stride, uint32_t rt, uint32_t ku, uint32_t rows, uint32_t cols, int lane)
{
#pragma unroll 4
    for (uint32_t i = 0; i < 16; ++i) {
        const uint32_t r = rt * 16 + i;
        const T* from = m + r * stride;
        T* to = reinterpret_cast<T*>(tile + i * Tile<T>::kPitch);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t c = ku * 128 + j * 32 + lane;
            to[j * 32 + lane] = r < rows && c < cols ? from[c] : T(0.f);
        }
    }
    __syncwarp();
}
template <typename T>
__device__ __forceinline__ void tile_out(const unsigned char* tile, T* m, uint64_t stride, uint32_t rt, uint32_t ku, uint32_t rows, uint32_t cols, int lane)
{
    __syncwarp();
#pragma unroll 4
    for (uint32_t i = 0; i < 16; ++i) {
        const uint32_t r = rt * 16 + i;
        if (r >= rows) break;
        T* to = m + r * stride;
        const T* from = reinterpret_cast<const T*>(tile + i * Tile<T>::kPitch);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const uint32_t c = ku * 128 + j * 32 + lane;
            if (c < cols) to[c] = from[j * 32 + lane];
        }
    }
}
template <typename T> __device__ __forceinline__ Eight<T> from_tile(const unsigned char* tile, uint32_t row, uint32_t c)
{
    Eight<T> v;
#pragma unroll
    for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) v.w[h] = *reinterpret_cast<const uint4*>(tile + row * Tile<T>::kPitch + c * sizeof(T) + h * 16);
    return v;
}

template <typename T> __device__ __forceinline__ void to_tile(unsigned char* tile, uint32_t row, uint32_t c, const Eight<T>& v)
{
#pragma unroll
    for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h) *reinterpret_cast<uint4*>(tile + row * Tile<T>::kPitch + c * sizeof(T) + h * 16) = v.w[h];
}

// Which matrix of the launch a CTA works on, and the warp's 16-row x 128-column unit in it.
template <typename Args> __device__ __forceinline__ bool find_unit(const Args& a, uint32_t& which, uint32_t& rt, uint32_t& ku)
{
    uint32_t m = 0;
    while (m + 1 < a.n && blockIdx.x >= a.mat[m + 1].first_cta) ++m;
    which = m;
    const uint32_t kus = (a.mat[m].cols + 127) / 128, tiles = (a.mat[m].rows + 63) / 64 * 4;     // fewer than 2^32 units: a matrix has fewer elements
    const uint32_t u = (blockIdx.x - a.mat[m].first_cta) * kPackWarps + (threadIdx.x >> 5);
    rt = u / kus;
    ku = u - rt * kus;
    return rt < tiles;
}

__device__ __forceinline__ float max3_abs_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Bits of the greatest magnitude of eight columns and of those of the neighbouring lanes (32 columns): compared as whole
// numbers between lanes, so that a NaN is the greatest.
__device__ __forceinline__ uint32_t top_of_lanes(uint32_t x)
{
    x = umax(x, __shfl_xor_sync(~0u, x, 1));
    return umax(x, __shfl_xor_sync(~0u, x, 2));
}
__device__ __forceinline__ uint32_t top_of(const float (&v)[8])
{
    const float m = max3_abs_nan(max3_abs_nan(v[0], v[1], v[2]), max3_abs_nan(v[3], v[4], v[5]), max3_abs_nan(v[6], v[7], 0.f));
    return top_of_lanes(__float_as_uint(m) & 0x7FFFFFFFu);
}
__device__ __forceinline__ uint32_t top_of(const uint4& w)        // bf16 pairs
{
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    const uint32_t m = max2_nan(max2_nan(w.x & kAbs, w.y & kAbs), max2_nan(w.z & kAbs, w.w & kAbs));
    return top_of_lanes(umax(m << 16, m & 0xFFFF0000u));
}

// One warp turns 16 rows x 128 columns into two tiles. RETRIEVE: the weight is fma(lambda, s * M, W_0) with the sign bits of the
// unit's 128 columns out of one Philox block -- the value retrieve writes in fp32, never stored. Bound by HBM for fp32 (16384 x
// 4096: 42 us, the rate of a copy) and by instruction issue for bf16, with half the bytes per code (50257 x 768: 21.1 us, 4.6
// TB/s; both rows' loads at once change nothing).
//
// Warps per SM, measured at 16384 x 4096 fp32 and 50257 x 768 bf16: a plain pack wants 32 of them (64 registers) and to keep its
// 16-byte loads coming (fp32 41.7 us at 32 warps, 44.1 at 24; bf16 22.4 and 24.3). A retrieve holds two tensors' words: with
// fp32 on either side 16 warps and no spills (80 us; 24 warps 98, 32 warps 118), with bf16 on both 24 (36.2 us, 38.8 at 32; 33.1 since two
// elements share their instructions).
template <typename WT, typename MT, bool RETRIEVE>
__global__ void __launch_bounds__(kPackWarps * 32, !RETRIEVE ? 8 : (sizeof(WT) + sizeof(MT) == 4 ? 6 : 4)) pack_kernel(const __grid_constant__ PackArgs a)
{
    uint32_t which, rt, ku;
    if (!find_unit(a, which, rt, ku)) return;
    const PackMatrix& m = a.mat[which];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t cols = m.cols, c0 = ku * 128 + 8 * t;
    const bool whole = ku * 128 + 128 <= cols && rt * 16 + 16 <= m.rows;       // the unit lies inside the matrix
    const int per = a.group >> 5;     // 32-column quarters per group: 1, 2 or 4

    extern __shared__ __align__(16) unsigned char tiles[];        // only where a matrix of the launch needs it
    unsigned char* tile = tiles + (threadIdx.x >> 5) * a.tile_bytes;

    uint4 blk = make_uint4(0, 0, 0, 0);
    if (RETRIEVE && m.flip) blk = philox4x32_10(ku, m.slot, kTagSign, a.task.id, a.task.key0, a.task.key1);
    uint32_t scale_bits[2];           // of quarter t
    // A word of codes is sum_i (q_i + 8) 16^i. Adding 1.5 * 2^23 to a quotient rounds it to the nearest integer (ties to
    // even) and leaves kRound + q in its bits, so one integer multiply-add per code puts it in place; what the constants
    // add up to is known beforehand.
    constexpr uint32_t kRound = 0x4B400000u;
    uint32_t word[4][2];              // [quarter][word of the quarter]
#pragma unroll
    for (int p = 0; p < 4; ++p) word[p][0] = word[p][1] = 0x88888888u - kRound * 0x11111111u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {     // row g, row g + 8
        const uint32_t r = rt * 16 + h * 8 + g;
        const WT* w = static_cast<const WT*>(m.src) + r * m.stride;
        const MT* sup = static_cast<const MT*>(m.m) + static_cast<size_t>(r) * cols;
        Eight<WT> raw[4];
        Eight<MT> add[4];
        if (whole && (m.vec & 1u)) {
#pragma unroll
            for (int p = 0; p < 4; ++p) raw[p] = load8<WT>(w + c0 + 32 * p);
        } else if (!(m.vec & 1u)) {
            if (h == 0) tile_in<WT>(tile, static_cast<const WT*>(m.src), m.stride, rt, ku, m.rows, cols, lane);
#pragma unroll
            for (int p = 0; p < 4; ++p) raw[p] = from_tile<WT>(tile, h * 8 + g, 32 * p + 8 * t);
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) raw[p] = gather8<WT>(w, c0 + 32 * p, r < m.rows ? cols : 0u);
        }
        if (RETRIEVE) {
            if (whole && (m.vec & 2u)) {
#pragma unroll
                for (int p = 0; p < 4; ++p) add[p] = load8<MT>(sup + c0 + 32 * p);
            } else if (!(m.vec & 2u)) {
                unsigned char* second = tile + Tile<WT>::kBytes;
                if (h == 0) tile_in<MT>(second, static_cast<const MT*>(m.m), cols, rt, ku, m.rows, cols, lane);
#pragma unroll
                for (int p = 0; p < 4; ++p) add[p] = from_tile<MT>(second, h * 8 + g, 32 * p + 8 * t);
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p) add[p] = gather8<MT>(sup, c0 + 32 * p, r < m.rows ? cols : 0u);
            }
        }
        float v[4][8];
        uint32_t top[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (sizeof(WT) == 2 && !RETRIEVE) {
                top[p] = top_of(raw[p].w[0]);            // widened below, where it is divided
            } else {
                widen8<WT>(raw[p], v[p]);
                if (RETRIEVE) {
                    // this lane's eight signs; in a pair of bf16 bit 2 e goes to bit 15, bit 2 e + 1 to bit 31 (the two copies of the
                    // byte do not overlap)
                    const uint32_t byte = ((p == 0 ? blk.x : (p == 1 ? blk.y : (p == 2 ? blk.z : blk.w))) >> (8 * t)) & 0xFFu;
                    auto pair = [&](int e) { return (byte * ((1u << (15 - 2 * e)) + (1u << (30 - 2 * e)))) & 0x80008000u; };
                    if (sizeof(MT) == 2) {
                        uint4& x = add[p].w[0];
                        x = make_uint4(x.x ^ pair(0), x.y ^ pair(1), x.z ^ pair(2), x.w ^ pair(3));
                    }
                    float d[8];
                    widen8<MT>(add[p], d);
                    const f32x2 lambda2 = twice(a.lambda);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        if (sizeof(MT) == 4) {
                            d[e] = flip(d[e], (byte << (31 - e)) & 0x80000000u);
                            d[e + 1] = flip(d[e + 1], (byte << (30 - e)) & 0x80000000u);
                        }
                        unpack2(fma2(lambda2, pack2(__float_as_uint(d[e]), __float_as_uint(d[e + 1])), pack2(__float_as_uint(v[p][e]), __float_as_uint(v[p][e + 1]))), v[p][e], v[p][e + 1]);
                    }
                }
                top[p] = top_of(v[p]);
            }
        }
        if (per >= 2) {
            top[0] = top[1] = umax(top[0], top[1]);
            top[2] = top[3] = umax(top[2], top[3]);
        }
        if (per == 4) top[0] = top[1] = top[2] = top[3] = umax(top[0], top[2]);
        // The four lanes of a row share the divisions: lane t makes the scale of quarter t.
        const uint32_t mine = t == 0 ? top[0] : (t == 1 ? top[1] : (t == 2 ? top[2] : top[3]));
        const bool finite = mine < 0x7F800000u;
        float s = __bfloat162float(__float2bfloat16_rn(quotient(__uint_as_float(mine), 7.f, 1.f / 7.f)));       // (of use from 2^-100 on)
        if (!(finite && s >= kMinScale)) s = 0.f;             // too small for a scale (or not a number): code 0
        const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
        scale_bits[h] = finite ? __float_as_uint(s) >> 16 : 0x7FC0u;
        const bool spoilt = __any_sync(~0u, !finite);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const float sp = __shfl_sync(~0u, s, (lane & ~3) | p), ip = __shfl_sync(~0u, inv, (lane & ~3) | p);
            if (sizeof(WT) == 2 && !RETRIEVE) widen8<WT>(raw[p], v[p]);
            if (spoilt && sp == 0.f) {                        // a NaN would reach the other row's codes
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] = 0.f;
            }
            if (sizeof(WT) == 4 && !RETRIEVE) {               // two at a time is no faster where HBM bounds it (42.0 us, 43.1)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int pos = ((e >> 1) & 1) * 2 + h + (e & 1) * 4;      // nibble of (row half, column): see the layout above
                    word[p][e >> 2] += __float_as_uint(quotient(v[p][e], sp, ip) + __uint_as_float(kRound)) * (1u << (4 * pos));
                }
                continue;
            }
            const f32x2 neg_s = twice(-sp), inv2 = twice(ip), round2 = twice(__uint_as_float(kRound));
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const f32x2 q = add2(quotient2(pack2(__float_as_uint(v[p][e]), __float_as_uint(v[p][e + 1])), neg_s, inv2), round2);
                const int pos = ((e >> 1) & 1) * 2 + h;      // and the next column's nibble four further
                word[p][e >> 2] += static_cast<uint32_t>(q) * (1u << (4 * pos)) + static_cast<uint32_t>(q >> 32) * (1u << (4 * pos + 16));
            }
        }
    }
    const PackedLayout lay(m.rows, cols, a.group);
    char* dst = static_cast<char*>(m.dst);
    *reinterpret_cast<uint4*>(dst + lay.codes(rt, 2 * ku) + lane * 16) = make_uint4(word[0][0], word[0][1], word[1][0], word[1][1]);
    if (lay.has_tile(2 * ku + 1))
        *reinterpret_cast<uint4*>(dst + lay.codes(rt, 2 * ku + 1) + lane * 16) = make_uint4(word[2][0], word[2][1], word[3][0], word[3][1]);
    if ((t & (per - 1)) == 0 && lay.has_tile(2 * ku + t / 2))
        *reinterpret_cast<uint32_t*>(dst + lay.scales(rt, 4 * ku + t) + g * 4) = scale_bits[0] | (scale_bits[1] << 16);
}

// `vec`: 1 in words of 16 bytes, 2 (fp32) in words of 32 bytes: a lane's eight columns in one store, so
// that every store fills whole sectors (16384 x 4096: 53 us against 69).
template <typename OT> __device__ __forceinline__ void store8(OT* row, uint32_t c, uint32_t cols, uint32_t vec, const Eight<OT>& v)
{
    constexpr int W = sizeof(OT) / 2;
    if (W == 2 && vec == 2 && c + 8 <= cols) {
        asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(row + c), "r"(v.w[0].x), "r"(v.w[0].y), "r"(v.w[0].z), "r"(v.w[0].w), "r"(v.w[W - 1].x), "r"(v.w[W - 1].y), "r"(v.w[W - 1].z), "r"(v.w[W - 1].w) : "memory");
    } else if (c + 8 <= cols) {
#pragma unroll
        for (int h = 0; h < W; ++h) __stcs(reinterpret_cast<uint4*>(row + c) + h, v.w[h]);
    } else {
        OT e[8];
        memcpy(e, &v, sizeof e);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c + k < cols) row[c + k] = e[k];
    }
}

// Eight values out of the operand registers (q / 64) of two words, for row half h: see the layout above. Both products by 64 and
// the fp32 ones by the scale are exact; a bf16 value is rounded once, in the second product.
template <typename OT> __device__ __forceinline__ Eight<OT> values8(const uint32_t (&q)[2][4], int h, uint32_t scale);      // scale: bf16 bits
template <> __device__ __forceinline__ Eight<bf16> values8(const uint32_t (&q)[2][4], int h, uint32_t scale)
{
    const uint32_t s2 = __byte_perm(scale, scale, 0x1010), unit = __float_as_uint(kCodeUnit) | (__float_as_uint(kCodeUnit) >> 16);
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = mul_bf16x2(mul_bf16x2(q[e >> 1][(e & 1) * 2 + h], unit), s2);
    return Eight<bf16>{{make_uint4(v[0], v[1], v[2], v[3])}};
}
template <> __device__ __forceinline__ Eight<float> values8(const uint32_t (&q)[2][4], int h, uint32_t scale)
{
    const f32x2 s2 = twice(__uint_as_float(scale << 16)), unit = twice(kCodeUnit);
    f32x2 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t pair = q[e >> 1][(e & 1) * 2 + h];
        v[e] = mul2(mul2(pack2(pair << 16, pair & 0xFFFF0000u), unit), s2);
    }
    Eight<float> r;
    memcpy(&r, v, sizeof r);
    return r;
}

// The values that the four bits stand for. Bound by its stores (16384 x 4096 fp32: 53 us, 5.7 TB/s; 50257 x 768 bf16: 15.9 us, 6.1
// TB/s).
template <typename OT> __global__ void __launch_bounds__(kPackWarps * 32) unpack_kernel(const __grid_constant__ UnpackArgs a)
{
    uint32_t which, rt, ku;
    if (!find_unit(a, which, rt, ku)) return;
    const UnpackMatrix& m = a.mat[which];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t cols = m.cols;
    const PackedLayout lay(m.rows, cols, a.group);
    const char* src = static_cast<const char*>(m.src);
    extern __shared__ __align__(16) unsigned char tiles[];
    unsigned char* tile = tiles + (threadIdx.x >> 5) * a.tile_bytes;
    uint4 w[2];
    w[0] = __ldcs(reinterpret_cast<const uint4*>(src + lay.codes(rt, 2 * ku) + lane * 16));
    w[1] = lay.has_tile(2 * ku + 1) ? __ldcs(reinterpret_cast<const uint4*>(src + lay.codes(rt, 2 * ku + 1) + lane * 16)) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t c = ku * 128 + 32 * p + 8 * t;
        if (c >= cols) continue;
        const uint32_t sb = __ldg(reinterpret_cast<const uint32_t*>(src + lay.scales(rt, 4 * ku + p) + g * 4));
        const uint32_t words[2] = {p & 1 ? w[p >> 1].z : w[p >> 1].x, p & 1 ? w[p >> 1].w : w[p >> 1].y};
        uint32_t q[2][4];                // operand registers of the two words: [i] holds row half i % 2, column pair i / 2
        decode(words[0], q[0]);
        decode(words[1], q[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t r = rt * 16 + h * 8 + g;
            if (m.vec && r >= m.rows) continue;
            const Eight<OT> v = values8<OT>(q, h, h ? sb >> 16 : sb & 0xFFFFu);
            if (m.vec) store8<OT>(static_cast<OT*>(m.dst) + r * m.stride, c, cols, m.vec, v);
            else to_tile<OT>(tile, h * 8 + g, 32 * p + 8 * t, v);
        }
    }
    if (!m.vec) tile_out<OT>(tile, static_cast<OT*>(m.dst), m.stride, rt, ku, m.rows, cols, lane);
}

// ---- products with a few tokens -----------------------------------------------------------------
constexpr int kMulWarps = 8;
constexpr int kDevices = 64;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

constexpr int kTiles = 2;                        // column tiles per stage
constexpr int kDepth = 2;                        // stages of a warp's ring
constexpr int kRowTiles = 4;                     // row tiles a warp takes along: one row block
constexpr int kRows = 16 * kRowTiles;

// A segment is one packed matrix with the tokens that go through it: the base with every token, then each slot of the
// superposition with the tokens whose task keeps this layer there.
//
// The column blocks of all segments, one after the other, are dealt in equal contiguous runs to 2^log_split warps of a CTA
// times the CTAs of a cluster; the other warps of the CTA do the same for other row blocks. A warp takes 64 rows along:
// what it does per tile of activations (three-way split, signs) is paid once for four tiles of codes. Each warp feeds
// itself: codes and scales through a ring of two stages, one bulk copy per stage, activations one tile ahead in registers;
// no warp waits for another until the end. Its sums of one segment stay in registers until its run leaves the segment. All
// partial sums meet in shared memory, those of a cluster's CTAs through distributed shared memory, and are added in a fixed
// order: results do not depend on timing.
//
// What bounds it: some 6 us that do not depend on the columns (start, first loads, the join), then 5.2 TB/s, where the ring
// alone streams 6.05: 16384 rows and 4096, 8192, 16384, 32768 columns take 11.3, 18.8, 32.9, 60.1 us with one bf16 token (eight: at most
// 1.1 more). At 16384 x 8192 no unit is full (issue 0.54 of the slots, about 80 instructions per tile of 16 x 64 codes; HBM 0.40,
// tensor pipe 0.24): below that size the 6 us are the larger part. 768 x 768: 3.9 us.
template <typename XT, int GROUP>
__global__ void __launch_bounds__(kMulWarps * 32, 2) packed_linear_kernel(const __grid_constant__ PackedLinearArgs<kNarrowTokens> a)
{
    typedef Acts<XT> Act;
    constexpr bool HALF = GROUP == 32;
    constexpr uint32_t kBlockTiles = GROUP == 128 ? 2 : 1;                       // column tiles per record
    constexpr uint32_t kCodeBytes = kBlockTiles * kRowTiles * 512, kRecord = kCodeBytes + (HALF ? 2 : 1) * kRowTiles * 32;
    constexpr uint32_t kBlocks = kTiles / kBlockTiles;                           // records per stage
    constexpr uint32_t kStage = kBlocks * kRecord;
    extern __shared__ float part[];      // [row block of the CTA][part][position in the token lists][kRows]
    cg::cluster_group cluster = cg::this_cluster();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ls = a.log_split, kp = warp & ((1u << ls) - 1), wr = warp >> ls, split = 1u << ls, blocks_cta = kMulWarps >> ls;
    const uint32_t lr = a.log_ranks, ranks = 1u << lr, rank = blockIdx.x & (ranks - 1);
    const uint32_t first_block = (blockIdx.x >> lr) * blocks_cta, rb = first_block + wr;
    const uint32_t kbs = (a.cols + 64 * kBlockTiles - 1) / (64 * kBlockTiles), rbs = (a.rows + kRows - 1) / kRows;
    const uint32_t n_pos = a.seg[a.n_seg - 1].first + a.seg[a.n_seg - 1].count;
    const uint64_t total = static_cast<uint64_t>(kbs) * a.n_seg;
    const XT* x = static_cast<const XT*>(a.x);
    float* mine = part + static_cast<size_t>(wr * split + kp) * n_pos * kRows;

    const uint32_t lo = static_cast<uint32_t>(total * (rank * split + kp) >> (ls + lr));
    const uint32_t hi = rb < rbs ? static_cast<uint32_t>(total * (rank * split + kp + 1) >> (ls + lr)) : lo;

    const uint32_t smem = static_cast<uint32_t>(__cvta_generic_to_shared(part));
    const uint32_t bars = smem + a.ring_at + warp * kDepth * 8;
    const uint32_t ring = smem + a.ring_at + kMulWarps * kDepth * 8 + warp * kDepth * kStage;
    if (lane == 0) {
        for (uint32_t d = 0; d < kDepth; ++d) bar_init(bars + d * 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();

    uint32_t left = hi - lo, fseg = lo / max(kbs, 1u), fkb = lo - fseg * kbs, fstage = 0;      // what is fetched next
    auto fetch = [&]() {
        if (!left) return;
        const uint32_t n = min(min(kBlocks, kbs - fkb), left);
        if (lane == 0) {
            const uint32_t bar = bars + fstage * 8;
            bar_expect(bar, n * kRecord);
            bulk_copy(ring + fstage * kStage, static_cast<const char*>(a.seg[fseg].packed) + (static_cast<size_t>(rb) * kbs + fkb) * kRecord, n * kRecord, bar);
        }
        fstage ^= 1u;
        left -= n;
        fkb += n;
        if (fkb == kbs) { fkb = 0; ++fseg; }
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d) fetch();
    for (uint32_t i = lane; i < n_pos * (kRows / 4); i += 32) reinterpret_cast<float4*>(mine)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncwarp();

    uint32_t u = lo, useg = lo / max(kbs, 1u), ukb = lo - useg * kbs, stage = 0, parity = 0;
    bool ok = true;
    while (u < hi && ok) {
        const uint32_t k0 = ukb, k1 = min(kbs, k0 + (hi - u));
        const PackedSegment& sg = a.seg[useg++];
        u += k1 - k0;
        ukb = 0;
        const uint32_t count = sg.count, tok = min(static_cast<uint32_t>(g), count - 1);
        const bool signs = sg.flip != 0;
        // Columns n of a product do not meet: what the lanes without a token hold (the last token's activations) goes nowhere.
        const XT* xt = x + a.token[sg.first + tok] * a.x_stride;
        const uint32_t whole = a.x_vec ? a.cols / 64 : 0u;        // column tiles whose activations are whole 16-byte words
        typename Act::Raw raw[2];
        auto load = [&](uint32_t kt) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const uint32_t c = kt * 64 + 32 * p + 8 * t;
                if (kt < whole) raw[p] = Act::words(xt + c);
                else raw[p] = c < a.cols ? Act::gather(xt, c, a.cols) : Act::zero();
            }
        };
        const uint32_t kt1 = min(k1 * kBlockTiles, (a.cols + 63) / 64);
        load(k0 * kBlockTiles);
        DevTask task = {0, 0, 0, 0};
        if (signs) task = a.task[a.token_task[sg.first + tok]];
        float tot[kRowTiles][4];
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) tot[r][0] = tot[r][1] = tot[r][2] = tot[r][3] = 0.f;
        uint4 blk = make_uint4(0, 0, 0, 0);
        uint32_t blk0 = ~0u;         // first of the four sign blocks that the lanes of a token hold
        for (uint32_t kb = k0; kb < k1; kb += kBlocks) {
            const uint32_t st = ring + stage * kStage;
            ok = bar_wait(bars + stage * 8, parity);
            if (!ok) break;
            const uint32_t kt0 = kb * kBlockTiles, nt = min(static_cast<uint32_t>(kTiles), kt1 - kt0);
#pragma unroll
            for (uint32_t i = 0; i < static_cast<uint32_t>(kTiles); ++i) {
                if (i >= nt) break;
                const uint32_t kt = kt0 + i;
                uint32_t xa[2][Act::kTerms][4];
                Act::terms(raw[0], xa[0]);
                Act::terms(raw[1], xa[1]);
                if (kt + 1 < kt1) load(kt + 1);
                if (signs) {
                    if (blk0 == ~0u || (kt >> 1) - blk0 >= 4) {
                        blk0 = kt >> 1;      // lane t of a token makes the block of columns 128 (blk0 + t) ..
                        blk = philox4x32_10(blk0 + t, sg.slot, kTagSign, task.id, task.key0, task.key1);
                    }
                    const int src = (lane & ~3) | static_cast<int>((kt >> 1) - blk0);
                    const uint32_t w0 = __shfl_sync(~0u, kt & 1 ? blk.z : blk.x, src), w1 = __shfl_sync(~0u, kt & 1 ? blk.w : blk.y, src);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const uint32_t bits = ((p ? w1 : w0) >> (8 * t)) & 0xFFu;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            // bit 2e of the byte lands on bit 15, bit 2e + 1 on bit 31; the two copies do not overlap
                            const uint32_t mask = (bits * ((1u << (15 - 2 * e)) + (1u << (30 - 2 * e)))) & 0x80008000u;
#pragma unroll
                            for (int k = 0; k < Act::kTerms; ++k) xa[p][k][e] ^= mask;
                        }
                    }
                }
                // word by word across the row tiles, so that a product does not wait for the one before it
                const uint32_t rec = st + (kBlockTiles == 1 ? i * kRecord : 0u);
                const uint32_t cat = rec + (kBlockTiles == 2 ? i * (kRowTiles * 512) : 0u) + lane * 16, sat = rec + kCodeBytes + g * 4;
                uint4 cw[kRowTiles];
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) cw[r] = lds128(cat + r * 512);
                float acc[kRowTiles][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int r = 0; r < kRowTiles; ++r) {
                        uint32_t am[4];
                        decode(j == 0 ? cw[r].x : (j == 1 ? cw[r].y : (j == 2 ? cw[r].z : cw[r].w)), am);
#pragma unroll
                        for (int k = 0; k < Act::kTerms; ++k) {
                            const uint32_t b0 = xa[j >> 1][k][2 * (j & 1)], b1 = xa[j >> 1][k][2 * (j & 1) + 1];
                            if (k == 0 && (j == 0 || (HALF && j == 2))) mma_16816_first(acc[r], am, b0, b1);
                            else mma_16816(acc[r], am, b0, b1);
                        }
                    }
                    if ((HALF && j == 1) || j == 3) {
#pragma unroll
                        for (int r = 0; r < kRowTiles; ++r) {
                            const uint32_t s2 = lds_u32(sat + r * 32 + (HALF && j == 3 ? kRowTiles * 32 : 0));
                            const float s_lo = __uint_as_float(s2 << 16), s_hi = __uint_as_float(s2 & 0xFFFF0000u);
                            tot[r][0] = __fmaf_rn(s_lo, acc[r][0], tot[r][0]);
                            tot[r][1] = __fmaf_rn(s_lo, acc[r][1], tot[r][1]);
                            tot[r][2] = __fmaf_rn(s_hi, acc[r][2], tot[r][2]);
                            tot[r][3] = __fmaf_rn(s_hi, acc[r][3], tot[r][3]);
                        }
                    }
                }
            }
            __syncwarp();                // every lane has read the stage: it may be filled again
            fetch();
            stage ^= 1u;
            parity ^= stage ^ 1u;
        }
        {
            const uint32_t i = 2 * t;
            float* to = mine + (sg.first + i) * kRows + g;
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r) {
                if (i < count) { to[r * 16] = kCodeUnit * tot[r][0]; to[r * 16 + 8] = kCodeUnit * tot[r][2]; }
                if (i + 1 < count) { to[kRows + r * 16] = kCodeUnit * tot[r][1]; to[kRows + r * 16 + 8] = kCodeUnit * tot[r][3]; }
            }
        }
    }
    if (!ok) {                           // a copy that never arrived: count it, give the others time, spoil the sums
        if (lane == 0) atomicAdd(&g_packed_giveups, 1u);
        for (uint32_t d = 0; d < kDepth; ++d) (void)bar_wait(bars + d * 8, d < stage ? parity ^ 1u : parity);
        for (uint32_t i = lane; i < n_pos * kRows; i += 32) mine[i] = NAN;
    }
    __syncthreads();
    // the CTA's y = (sum of the base's parts) + lambda * (sum of the slot's parts), each sum in part order
    const uint32_t rows_cta = blocks_cta * kRows, n_out = rows_cta * a.n_tokens;
    float* sums = part + static_cast<size_t>(kMulWarps) * n_pos * kRows;      // [token][row of the CTA], only with a cluster
    const uint64_t row0 = static_cast<uint64_t>(first_block) * kRows;
    auto store = [&](uint32_t tok, uint32_t r, float y) {
        if (row0 + r >= a.rows) return;
        const size_t at = tok * a.y_stride + row0 + r;
        if (a.y_bf16) static_cast<bf16*>(a.y)[at] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.y)[at] = y;
    };
    for (uint32_t o = threadIdx.x; o < n_out; o += kMulWarps * 32) {
        const uint32_t r = o % rows_cta, tok = o / rows_cta;
        const float* p = part + static_cast<size_t>(r / kRows) * split * n_pos * kRows + r % kRows;
        float y = 0.f, d = 0.f;
        for (uint32_t k = 0; k < split; ++k) y += p[(k * n_pos + tok) * kRows];
        if (a.n_seg > 1) {
            const uint32_t pos = a.pos_of_token[tok];
            for (uint32_t k = 0; k < split; ++k) d += p[(k * n_pos + pos) * kRows];
            y = __fmaf_rn(a.lambda, d, y);
        }
        if (ranks == 1) store(tok, r, y);
        else sums[o] = y;
    }
    if (ranks > 1) {
        cluster.sync();
        for (uint32_t o = rank * (kMulWarps * 32) + threadIdx.x; o < n_out; o += ranks * kMulWarps * 32) {
            float y = 0.f;
            for (uint32_t k = 0; k < ranks; ++k) y += cluster.map_shared_rank(sums, k)[o];
            store(o / rows_cta, o % rows_cta, y);
        }
        cluster.sync();          // nobody leaves while its sums may still be read
    }
}

template <typename XT, int GROUP> cudaError_t launch_mul(PackedLinearArgs<kNarrowTokens>& a, int sm_count, int device, cudaStream_t s)
{
    const PackedLayout lay(a.rows, a.cols, a.group);
    const uint64_t total = static_cast<uint64_t>(lay.col_blocks) * a.n_seg, blocks = (a.rows + kRows - 1) / kRows;
    // As many warps to a row block as still fit the SMs at once (two CTAs each), as long as every warp has a record: first the
    // warps of a CTA share rows, then the CTAs of a cluster do. (One and a third rounds of CTAs instead of one: no faster.)
    const uint64_t slots = static_cast<uint64_t>(sm_count) * 2;
    a.log_split = a.log_ranks = 0;
    while (a.log_split < 3 && ((blocks << (a.log_split + 1)) + kMulWarps - 1) / kMulWarps <= slots && (2u << a.log_split) <= total) ++a.log_split;
    while (a.log_split == 3 && a.log_ranks < 3 && (blocks << (a.log_ranks + 1)) <= slots && (16ull << a.log_ranks) <= total) ++a.log_ranks;
    const uint32_t blocks_cta = kMulWarps >> a.log_split, ranks = 1u << a.log_ranks;
    const uint32_t n_pos = a.seg[a.n_seg - 1].first + a.seg[a.n_seg - 1].count;
    a.ring_at = (kMulWarps * n_pos + (ranks > 1 ? blocks_cta * a.n_tokens : 0)) * kRows * static_cast<uint32_t>(sizeof(float));
    const size_t smem = a.ring_at + static_cast<size_t>(kMulWarps) * kDepth * ((kTiles >> lay.log_tiles) * lay.record + 8);
    // A kernel has to opt in beyond 48 KiB, per device: once, to the most that any call can want (every token a slot of its own, a
    // cluster; a limit of each call's own size could be lowered again by another thread before the launch).
    constexpr uint32_t kRecords = GROUP == 128 ? kTiles / 2 : kTiles, kRecord = GROUP == 128 ? 4224 : (GROUP == 32 ? 2304 : 2176);
    constexpr size_t kMost = (kMulWarps * 2 * kNarrowTokens + kNarrowTokens) * kRows * sizeof(float) + kMulWarps * kDepth * (kRecords * kRecord + 8);
    static_assert(kMost <= 113 * 1024, "two CTAs per SM");
    if (smem > kMost) return cudaErrorInvalidValue;
    static std::atomic<bool> granted[kDevices];
    if (device >= kDevices || !granted[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(packed_linear_kernel<XT, GROUP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMost));
        if (e != cudaSuccess) return e;
        if (device < kDevices) granted[device].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((blocks + blocks_cta - 1) / blocks_cta * ranks));
    cfg.blockDim = dim3(kMulWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = ranks > 1;
    return cudaLaunchKernelEx(&cfg, packed_linear_kernel<XT, GROUP>, a);
}

template <typename XT> cudaError_t launch_group(PackedLinearArgs<kNarrowTokens>& a, int sm_count, int device, cudaStream_t s)
{
    if (a.group == 32) return launch_mul<XT, 32>(a, sm_count, device, s);
    if (a.group == 64) return launch_mul<XT, 64>(a, sm_count, device, s);
    return launch_mul<XT, 128>(a, sm_count, device, s);
}

}  // namespace

int launch_packed_linear(PackedLinearArgs<kNarrowTokens>& a, bool x_bf16, int sm_count, int device, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return static_cast<int>(x_bf16 ? launch_group<bf16>(a, sm_count, device, s) : launch_group<float>(a, sm_count, device, s));
}

int packed_giveups(unsigned int* count)
{
    return static_cast<int>(cudaMemcpyFromSymbol(count, g_packed_giveups, sizeof(unsigned int)));
}

namespace {
template <typename M> unsigned deal_ctas(M* mat, uint32_t n)
{
    uint64_t at = 0;
    for (uint32_t i = 0; i < n; ++i) {
        mat[i].first_cta = static_cast<uint32_t>(at);
        at += (static_cast<uint64_t>((mat[i].rows + 63) / 64) * 4 * ((mat[i].cols + 127) / 128) + kPackWarps - 1) / kPackWarps;
    }
    return static_cast<unsigned>(at);
}
}  // namespace

int launch_pack(int w_dtype, int m_dtype, bool retrieve, PackArgs& a, void* stream)
{
    const unsigned grid = deal_ctas(a.mat, a.n);
    if (!grid) return 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    constexpr int kThreads = kPackWarps * 32;
    const uint32_t all = retrieve ? 3u : 1u;
    a.tile_bytes = 0;
    for (uint32_t i = 0; i < a.n; ++i)
        if ((a.mat[i].vec & all) != all)
            a.tile_bytes = (w_dtype == 1 ? Tile<bf16>::kBytes : Tile<float>::kBytes) + (retrieve ? (m_dtype == 1 ? Tile<bf16>::kBytes : Tile<float>::kBytes) : 0u);
    const size_t smem = static_cast<size_t>(kPackWarps) * a.tile_bytes;
    auto run = [&](auto kernel) {
        if (smem > 48 * 1024) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
            if (e != cudaSuccess) return static_cast<int>(e);
        }
        kernel<<<grid, kThreads, smem, s>>>(a);
        return static_cast<int>(cudaGetLastError());
    };
    if (!retrieve) return w_dtype == 1 ? run(pack_kernel<bf16, bf16, false>) : run(pack_kernel<float, float, false>);
    if (w_dtype == 1) return m_dtype == 1 ? run(pack_kernel<bf16, bf16, true>) : run(pack_kernel<bf16, float, true>);
    return m_dtype == 1 ? run(pack_kernel<float, bf16, true>) : run(pack_kernel<float, float, true>);
}

int launch_unpack(int out_dtype, UnpackArgs& a, void* stream)
{
    const unsigned grid = deal_ctas(a.mat, a.n);
    if (!grid) return 0;
    a.tile_bytes = 0;
    for (uint32_t i = 0; i < a.n; ++i)
        if (!a.mat[i].vec) a.tile_bytes = out_dtype == 1 ? Tile<bf16>::kBytes : Tile<float>::kBytes;
    const size_t smem = static_cast<size_t>(kPackWarps) * a.tile_bytes;
    if (out_dtype == 1) unpack_kernel<bf16><<<grid, kPackWarps * 32, smem, static_cast<cudaStream_t>(stream)>>>(a);
    else unpack_kernel<float><<<grid, kPackWarps * 32, smem, static_cast<cudaStream_t>(stream)>>>(a);
    return static_cast<int>(cudaGetLastError());
}

}  // namespace randes
