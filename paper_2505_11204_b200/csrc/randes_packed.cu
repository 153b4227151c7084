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
// Layout: tiles of 16 rows x 64 columns, 512 bytes = 16 bytes per lane, ordered [row tile][column tile][lane], so that
// one 16-byte load per lane brings the A operands of four m16n8k16 products in the order the tensor core wants them.
// Lane (g = lane / 4, t = lane % 4) holds rows g and g + 8. Its 32-bit word j holds the four columns
//     c(j, e) = 32 (j / 2) + 8 t + 4 (j % 2) + e,    e = 0 .. 3
// of both rows, code + 8 in nibble order (g,0) (g+8,0) (g,2) (g+8,2) (g,1) (g+8,1) (g,3) (g+8,3): shifting the word by
// 4 i and masking with 0x000F000F leaves operand register i. The columns a lane owns are 8 neighbours in each half of
// the tile, so that the activations it multiplies are two 16-byte loads. After the codes come the scales,
// [row tile][group][g], one word per lane row: rows g (low half) and g + 8 (high half).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "randes_device.cuh"
#include "randes_internal.h"

namespace randes {
namespace {

using namespace device;

constexpr int kPackWarps = 8;                 // warps per CTA of the pack and unpack kernels
constexpr float kMinScale = 0x1p-100f;        // far enough from the subnormals for the quotient below to be exact

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// w / s correctly rounded, given inv = fl(1 / s): one Newton step on the quotient (Markstein 1990). No operand or
// residual leaves the normal range: s >= 2^-100 and |w| <= 7.02 s.
__device__ __forceinline__ float quotient(float w, float s, float inv)
{
    const float q = w * inv;
    return __fmaf_rn(__fmaf_rn(-q, s, w), inv, q);
}

// eight neighbouring columns of one row, zero beyond the row's end
template <typename T>
__device__ __forceinline__ void load8(const T* row, uint32_t c, uint32_t cols, bool vec, float (&v)[8])
{
    if (vec && c + 8 <= cols) {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 r = __ldcs(reinterpret_cast<const uint4*>(row + c) + h);
                v[4 * h] = __uint_as_float(r.x); v[4 * h + 1] = __uint_as_float(r.y);
                v[4 * h + 2] = __uint_as_float(r.z); v[4 * h + 3] = __uint_as_float(r.w);
            }
        } else {
            float u[Store<T>::CPL];
            Store<T>::widen(__ldcs(reinterpret_cast<const uint4*>(row + c)), u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = u[e % Store<T>::CPL];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? Store<T>::load1(row + c + e) : 0.f;
    }
}

// Which matrix of the launch a CTA works on, and the warp's 16-row x 128-column unit in it.
template <typename Args> __device__ __forceinline__ bool find_unit(const Args& a, uint32_t& which, uint32_t& rt, uint32_t& ku)
{
    uint32_t m = 0;
    while (m + 1 < a.n && blockIdx.x >= a.mat[m + 1].first_cta) ++m;
    which = m;
    const uint32_t kus = (a.mat[m].cols + 127) / 128;
    const uint64_t u = static_cast<uint64_t>(blockIdx.x - a.mat[m].first_cta) * kPackWarps + (threadIdx.x >> 5);
    if (u >= static_cast<uint64_t>((a.mat[m].rows + 15) / 16) * kus) return false;
    rt = static_cast<uint32_t>(u / kus);
    ku = static_cast<uint32_t>(u % kus);
    return true;
}

// One warp turns 16 rows x 128 columns into two tiles. RETRIEVE: the weight is fma(lambda, s * M, W_0) with the sign
// bits of the unit's 128 columns out of one Philox block -- the value retrieve writes in fp32, never stored.
template <typename WT, typename MT, bool RETRIEVE>
__global__ void __launch_bounds__(kPackWarps * 32) pack_kernel(const __grid_constant__ PackArgs a)
{
    uint32_t which, rt, ku;
    if (!find_unit(a, which, rt, ku)) return;
    const PackMatrix& m = a.mat[which];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const WT* w = static_cast<const WT*>(m.src);
    const MT* sup = static_cast<const MT*>(m.m);
    const bool vec_w = m.vec & 1u, vec_m = m.vec & 2u;
    const uint32_t cols = m.cols, c0 = ku * 128 + 8 * t;

    uint4 blk = make_uint4(0, 0, 0, 0);
    if (RETRIEVE && m.flip) blk = philox4x32_10(ku, m.slot, kTagSign, a.task.id, a.task.key0, a.task.key1);
    float v[2][4][8];      // [row g / g + 8][32-column quarter][column]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t r = rt * 16 + h * 8 + g;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (r < m.rows) {
                load8<WT>(w + r * m.stride, c0 + 32 * p, cols, vec_w, v[h][p]);
                if (RETRIEVE) {
                    float d[8];
                    load8<MT>(sup + static_cast<size_t>(r) * cols, c0 + 32 * p, cols, vec_m, d);
                    const uint32_t word = p == 0 ? blk.x : (p == 1 ? blk.y : (p == 2 ? blk.z : blk.w));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[h][p][e] = __fmaf_rn(a.lambda, flip(d[e], (word >> (8 * t + e)) << 31), v[h][p][e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[h][p][e] = 0.f;
            }
        }
    }
    uint32_t top[2][4];    // bits of the greatest magnitude per quarter: as integers, so that a NaN is the greatest
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            uint32_t x = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) x = umax(x, __float_as_uint(v[h][p][e]) & 0x7FFFFFFFu);
            x = umax(x, __shfl_xor_sync(~0u, x, 1));
            top[h][p] = umax(x, __shfl_xor_sync(~0u, x, 2));
        }
    const int per = a.group >> 5;     // quarters per group: 1, 2 or 4
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (per >= 2) {
            top[h][0] = top[h][1] = umax(top[h][0], top[h][1]);
            top[h][2] = top[h][3] = umax(top[h][2], top[h][3]);
        }
        if (per == 4) top[h][0] = top[h][1] = top[h][2] = top[h][3] = umax(top[h][0], top[h][2]);
    }
    uint32_t scale_bits[2][4];
    uint32_t word[4][2];              // [quarter][word of the quarter]
#pragma unroll
    for (int p = 0; p < 4; ++p) word[p][0] = word[p][1] = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const bool finite = top[h][p] < 0x7F800000u;
            const float s7 = __fdiv_rn(__uint_as_float(top[h][p]), 7.f);
            const uint32_t sb = __bfloat16_as_ushort(__float2bfloat16_rn(s7));
            float s = __uint_as_float(sb << 16);
            if (!(s >= kMinScale)) s = 0.f;
            scale_bits[h][p] = finite ? __float_as_uint(s) >> 16 : 0x7FC0u;
            const float inv = finite && s > 0.f ? __frcp_rn(s) : 0.f;
            // a group that is all NaN or all zero keeps code 0: its values are cleared here, not in the quotient
            const bool live = inv != 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = live ? quotient(v[h][p][e], s, inv) : 0.f;
                // adding 1.5 * 2^23 rounds to the nearest integer (ties to even) and leaves it in the low bits
                const uint32_t code = __float_as_uint(q + (12582912.f + 8.f)) & 15u;
                // nibble of (row half h, column e % 4) in word e / 4: see the layout above
                const int pos = ((e >> 1) & 1) * 2 + h + (e & 1) * 4;
                word[p][e >> 2] |= code << (4 * pos);
            }
        }
    const uint32_t kts = (cols + 63) / 64, n_groups = packed_groups(cols, a.group);
    uint4* codes = static_cast<uint4*>(m.dst) + (static_cast<size_t>(rt) * kts + 2 * ku) * 32 + lane;
    codes[0] = make_uint4(word[0][0], word[0][1], word[1][0], word[1][1]);
    if (2 * ku + 1 < kts) codes[32] = make_uint4(word[2][0], word[2][1], word[3][0], word[3][1]);
    uint32_t* scales = reinterpret_cast<uint32_t*>(static_cast<char*>(m.dst) + packed_codes_bytes(m.rows, cols)) +
                       static_cast<size_t>(rt) * n_groups * 8;
    if (t == 0) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t grp = ku * (4 / per) + p / per;
            if (p % per == 0 && grp < n_groups) scales[static_cast<size_t>(grp) * 8 + g] = scale_bits[0][p] | (scale_bits[1][p] << 16);
        }
    }
}

template <typename OT> __device__ __forceinline__ void store8(OT* row, uint32_t c, uint32_t cols, bool vec, const float (&v)[8])
{
    if (vec && c + 8 <= cols) {
        Out<OT>::template store<8>(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) Out<OT>::store1(row + c + e, v[e]);
    }
}

// The values that the four bits stand for: q * s is exact in fp32 (3 + 8 bits), rounded once for bf16.
template <typename OT> __global__ void __launch_bounds__(kPackWarps * 32) unpack_kernel(const __grid_constant__ UnpackArgs a)
{
    uint32_t which, rt, ku;
    if (!find_unit(a, which, rt, ku)) return;
    const UnpackMatrix& m = a.mat[which];
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t cols = m.cols, kts = (cols + 63) / 64, n_groups = packed_groups(cols, a.group);
    const uint4* codes = static_cast<const uint4*>(m.src) + (static_cast<size_t>(rt) * kts + 2 * ku) * 32 + lane;
    uint4 w[2];
    w[0] = __ldcs(codes);
    w[1] = 2 * ku + 1 < kts ? __ldcs(codes + 32) : make_uint4(0, 0, 0, 0);
    const uint32_t* scales = reinterpret_cast<const uint32_t*>(static_cast<const char*>(m.src) + packed_codes_bytes(m.rows, cols)) +
                             static_cast<size_t>(rt) * n_groups * 8;
    const int per = a.group >> 5;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t grp = ku * (4 / per) + p / per;
        const uint32_t c = ku * 128 + 32 * p + 8 * t;
        if (grp >= n_groups || c >= cols) continue;
        const uint32_t sb = __ldg(scales + static_cast<size_t>(grp) * 8 + g);
        const uint32_t words[2] = {p & 1 ? w[p >> 1].z : w[p >> 1].x, p & 1 ? w[p >> 1].w : w[p >> 1].y};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t r = rt * 16 + h * 8 + g;
            if (r >= m.rows) continue;
            const float s = __uint_as_float(h ? sb & 0xFFFF0000u : sb << 16);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pos = ((e >> 1) & 1) * 2 + h + (e & 1) * 4;
                v[e] = (static_cast<float>((words[e >> 2] >> (4 * pos)) & 15u) - 8.f) * s;
            }
            store8<OT>(static_cast<OT*>(m.dst) + r * m.stride, c, cols, m.vec, v);
        }
    }
}

// ---- products with a few tokens -----------------------------------------------------------------
constexpr int kMulWarps = 8;

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Operand register i of one word of codes, as q / 16. 0x4100 is 8 in bf16 with a last place of 1/16, so the nibble dropped
// into its mantissa reads 8 + (q + 8) / 16; taking 8.5 away is exact. Sixteenths, not units: a product with an activation
// then cannot overflow where the weight itself (q * s, s << 1) would not; the factor comes back with the partial sums.
constexpr float kCodeUnit = 16.f;
__device__ __forceinline__ uint32_t decode2(uint32_t word, int i)
{
    const uint32_t biased = ((word >> (4 * i)) & 0x000F000Fu) | 0x41004100u;
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(biased), "r"(0x41084108u));
    return r;
}

// Activations: a lane's eight neighbouring columns of one token as four words of bf16 pairs. An fp32 activation becomes
// three bf16 terms by truncation (8 + 8 + 8 bits: their sum is the fp32 value exactly, down to where the last term
// underflows), so that products and sums keep fp32's accuracy on the bf16 tensor core.
template <typename XT> struct Acts;
template <> struct Acts<bf16> {
    static constexpr int kTerms = 1;
    uint32_t w[1][4];
    __device__ __forceinline__ void load(const bf16* p, uint32_t c, uint32_t cols, bool vec)
    {
        if (vec && c + 8 <= cols) {
            const uint4 r = __ldg(reinterpret_cast<const uint4*>(p + c));
            w[0][0] = r.x; w[0][1] = r.y; w[0][2] = r.z; w[0][3] = r.w;
        } else {
            const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = c + 2 * e < cols ? __ldg(q + c + 2 * e) : 0u, hi = c + 2 * e + 1 < cols ? __ldg(q + c + 2 * e + 1) : 0u;
                w[0][e] = lo | (hi << 16);
            }
        }
    }
};
template <> struct Acts<float> {
    static constexpr int kTerms = 3;
    uint32_t w[3][4];
    __device__ __forceinline__ void load(const float* p, uint32_t c, uint32_t cols, bool vec)
    {
        float v[8];
        if (vec && c + 8 <= cols) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 r = __ldg(reinterpret_cast<const float4*>(p + c) + h);
                v[4 * h] = r.x; v[4 * h + 1] = r.y; v[4 * h + 2] = r.z; v[4 * h + 3] = r.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? __ldg(p + c + e) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = v[2 * e], b = v[2 * e + 1];
                w[k][e] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
                const float ta = __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), tb = __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
                v[2 * e] = a == ta ? 0.f : a - ta;           // the comparison keeps an infinity out of the lower terms
                v[2 * e + 1] = b == tb ? 0.f : b - tb;
            }
        }
    }
};

// NB blocks of 8 tokens per pass. HALF: groups of 32 columns (two scales per tile and row) instead of 64 or 128.
//
// A CTA's eight warps are `split` parts of the columns x (8 / split) tiles of 16 rows. A segment is one packed matrix with
// the tokens that go through it: the base with every token, then each slot of the superposition with the tokens whose
// task keeps this layer there. Partial sums of all parts and segments meet in shared memory and are added in a fixed
// order, so results do not depend on timing.
template <int NB, typename XT, bool HALF>
__global__ void __launch_bounds__(kMulWarps * 32) packed_linear_kernel(const __grid_constant__ PackedLinearArgs a)
{
    extern __shared__ float part[];      // [row tile of the CTA][part][position in the token lists][16 rows]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t split = a.split, kp = warp % split, wr = warp / split, tiles_cta = kMulWarps / split;
    const uint32_t rt = blockIdx.x * tiles_cta + wr;
    const uint32_t kts = (a.cols + 63) / 64, rts = (a.rows + 15) / 16;
    const uint32_t k0 = static_cast<uint32_t>(static_cast<uint64_t>(kts) * kp / split), k1 = static_cast<uint32_t>(static_cast<uint64_t>(kts) * (kp + 1) / split);
    const uint32_t n_pos = a.seg[a.n_seg - 1].first + a.seg[a.n_seg - 1].count;
    const XT* x = static_cast<const XT*>(a.x);
    const uint32_t n_groups = packed_groups(a.cols, a.group);
    if (rt < rts) {
        for (uint32_t sgi = 0; sgi < a.n_seg; ++sgi) {
            const PackedSegment& sg = a.seg[sgi];
            const uint4* codes = static_cast<const uint4*>(sg.packed) + static_cast<size_t>(rt) * kts * 32 + lane;
            const uint32_t* scales = reinterpret_cast<const uint32_t*>(static_cast<const char*>(sg.packed) + packed_codes_bytes(a.rows, a.cols)) +
                                     static_cast<size_t>(rt) * n_groups * 8 + g;
            const XT* xr[NB];
            float tot[NB][4];
            uint4 blk[NB];
            DevTask task[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t i = b * 8 + g;
                const bool on = i < sg.count;
                const uint32_t pos = sg.first + (on ? i : 0);
                xr[b] = on ? x + a.token[pos] * a.x_stride : nullptr;
                if (sg.flip) task[b] = a.task[a.token_task[pos]];
                tot[b][0] = tot[b][1] = tot[b][2] = tot[b][3] = 0.f;
                blk[b] = make_uint4(0, 0, 0, 0);
            }
            uint32_t blk0 = ~0u;         // first of the four sign blocks that the lanes of a token hold
            for (uint32_t kt = k0; kt < k1; ++kt) {
                const uint4 cw = __ldg(codes + static_cast<size_t>(kt) * 32);
                const uint32_t sc0 = __ldg(scales + static_cast<size_t>(HALF ? 2 * kt : kt * 64 / a.group) * 8);
                const uint32_t sc1 = HALF && 2 * kt + 1 < n_groups ? __ldg(scales + static_cast<size_t>(2 * kt + 1) * 8) : 0u;
                if (sg.flip && (blk0 == ~0u || (kt >> 1) - blk0 >= 4)) {
                    blk0 = kt >> 1;      // lane t of a token makes the block of columns 128 (blk0 + t) ..
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        blk[b] = philox4x32_10(blk0 + t, sg.slot, kTagSign, task[b].id, task[b].key0, task[b].key1);
                }
                uint32_t am[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    am[0][i] = decode2(cw.x, i); am[1][i] = decode2(cw.y, i);
                    am[2][i] = decode2(cw.z, i); am[3][i] = decode2(cw.w, i);
                }
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if (static_cast<uint32_t>(b * 8) >= sg.count) break;
                    Acts<XT> xa[2];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        if (xr[b]) {
                            xa[p].load(xr[b], kt * 64 + 32 * p + 8 * t, a.cols, a.x_vec);
                        } else {
#pragma unroll
                            for (int k = 0; k < Acts<XT>::kTerms; ++k)
#pragma unroll
                                for (int e = 0; e < 4; ++e) xa[p].w[k][e] = 0u;
                        }
                    }
                    if (sg.flip) {
                        const int src = (lane & ~3) | static_cast<int>((kt >> 1) - blk0);
                        const uint32_t w0 = __shfl_sync(~0u, kt & 1 ? blk[b].z : blk[b].x, src), w1 = __shfl_sync(~0u, kt & 1 ? blk[b].w : blk[b].y, src);
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const uint32_t bits = ((p ? w1 : w0) >> (8 * t)) & 0xFFu;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                // bit 2e of the byte lands on bit 15, bit 2e + 1 on bit 31; the two copies do not overlap
                                const uint32_t mask = (bits * ((1u << (15 - 2 * e)) + (1u << (30 - 2 * e)))) & 0x80008000u;
#pragma unroll
                                for (int k = 0; k < Acts<XT>::kTerms; ++k) xa[p].w[k][e] ^= mask;
                            }
                        }
                    }
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
#pragma unroll
                        for (int k = 0; k < Acts<XT>::kTerms; ++k)
                            mma_16816(acc, am[j], xa[j >> 1].w[k][2 * (j & 1)], xa[j >> 1].w[k][2 * (j & 1) + 1]);
                        if ((HALF && j == 1) || j == 3) {
                            const uint32_t sc = HALF && j == 3 ? sc1 : sc0;
                            const float lo = __uint_as_float(sc << 16), hi = __uint_as_float(sc & 0xFFFF0000u);
                            tot[b][0] = __fmaf_rn(lo, acc[0], tot[b][0]);
                            tot[b][1] = __fmaf_rn(lo, acc[1], tot[b][1]);
                            tot[b][2] = __fmaf_rn(hi, acc[2], tot[b][2]);
                            tot[b][3] = __fmaf_rn(hi, acc[3], tot[b][3]);
                            acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
                        }
                    }
                }
            }
            float* mine = part + (static_cast<size_t>(wr * split + kp) * n_pos + sg.first) * 16;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t i = b * 8 + 2 * t;
                if (i < sg.count) { mine[i * 16 + g] = kCodeUnit * tot[b][0]; mine[i * 16 + g + 8] = kCodeUnit * tot[b][2]; }
                if (i + 1 < sg.count) { mine[(i + 1) * 16 + g] = kCodeUnit * tot[b][1]; mine[(i + 1) * 16 + g + 8] = kCodeUnit * tot[b][3]; }
            }
        }
    }
    __syncthreads();
    // y = (sum of the base's parts) + lambda * (sum of the slot's parts), each sum in part order
    const uint32_t n_out = tiles_cta * 16 * a.n_tokens;
    for (uint32_t o = threadIdx.x; o < n_out; o += kMulWarps * 32) {
        const uint32_t r = o % (tiles_cta * 16), tok = o / (tiles_cta * 16);
        const uint64_t row = static_cast<uint64_t>(blockIdx.x) * tiles_cta * 16 + r;
        if (row >= a.rows) continue;
        const float* p = part + static_cast<size_t>(r >> 4) * split * n_pos * 16 + (r & 15);
        float y = 0.f, d = 0.f;
        for (uint32_t k = 0; k < split; ++k) y += p[(k * n_pos + tok) * 16];
        if (a.n_seg > 1) {
            const uint32_t pos = a.pos_of_token[tok];
            for (uint32_t k = 0; k < split; ++k) d += p[(k * n_pos + pos) * 16];
            y = __fmaf_rn(a.lambda, d, y);
        }
        const size_t at = tok * a.y_stride + row;
        if (a.y_bf16) static_cast<bf16*>(a.y)[at] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.y)[at] = y;
    }
}

template <int NB, typename XT, bool HALF> cudaError_t launch_mul(const PackedLinearArgs& a, unsigned grid, size_t smem, cudaStream_t s)
{
    if (smem > 48 * 1024) {   // beyond this a kernel has to opt in, per device
        const cudaError_t e = cudaFuncSetAttribute(packed_linear_kernel<NB, XT, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    packed_linear_kernel<NB, XT, HALF><<<grid, kMulWarps * 32, smem, s>>>(a);
    return cudaGetLastError();
}

template <typename XT, bool HALF> cudaError_t launch_nb(const PackedLinearArgs& a, unsigned grid, size_t smem, cudaStream_t s)
{
    if (a.n_tokens <= 8) return launch_mul<1, XT, HALF>(a, grid, smem, s);
    if (a.n_tokens <= 16) return launch_mul<2, XT, HALF>(a, grid, smem, s);
    if (a.n_tokens <= 32) return launch_mul<4, XT, HALF>(a, grid, smem, s);
    return launch_mul<8, XT, HALF>(a, grid, smem, s);
}

}  // namespace

int launch_packed_linear(PackedLinearArgs& a, bool x_bf16, int sm_count, void* stream)
{
    const uint32_t rts = (a.rows + 15) / 16, kts = (a.cols + 63) / 64;
    uint32_t split = 1;
    // enough warps to keep about sixteen per SM loading, as long as every part has a tile
    while (split < kMulWarps && static_cast<uint64_t>(rts) * split < static_cast<uint64_t>(sm_count) * 16 && split * 2 <= kts) split *= 2;
    a.split = split;
    const uint32_t tiles_cta = kMulWarps / split;
    const uint32_t n_pos = a.seg[a.n_seg - 1].first + a.seg[a.n_seg - 1].count;
    const size_t smem = static_cast<size_t>(kMulWarps) * n_pos * 16 * sizeof(float);
    const unsigned grid = (rts + tiles_cta - 1) / tiles_cta;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool half = a.group == 32;
    cudaError_t e;
    if (x_bf16) e = half ? launch_nb<bf16, true>(a, grid, smem, s) : launch_nb<bf16, false>(a, grid, smem, s);
    else e = half ? launch_nb<float, true>(a, grid, smem, s) : launch_nb<float, false>(a, grid, smem, s);
    return static_cast<int>(e);
}

namespace {
template <typename M> unsigned deal_ctas(M* mat, uint32_t n)
{
    uint64_t at = 0;
    for (uint32_t i = 0; i < n; ++i) {
        mat[i].first_cta = static_cast<uint32_t>(at);
        at += (static_cast<uint64_t>((mat[i].rows + 15) / 16) * ((mat[i].cols + 127) / 128) + kPackWarps - 1) / kPackWarps;
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
    if (!retrieve) {
        if (w_dtype == 1) pack_kernel<bf16, bf16, false><<<grid, kThreads, 0, s>>>(a);
        else pack_kernel<float, float, false><<<grid, kThreads, 0, s>>>(a);
    } else if (w_dtype == 1) {
        if (m_dtype == 1) pack_kernel<bf16, bf16, true><<<grid, kThreads, 0, s>>>(a);
        else pack_kernel<bf16, float, true><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (m_dtype == 1) pack_kernel<float, bf16, true><<<grid, kThreads, 0, s>>>(a);
        else pack_kernel<float, float, true><<<grid, kThreads, 0, s>>>(a);
    }
    return static_cast<int>(cudaGetLastError());
}

int launch_unpack(int out_dtype, UnpackArgs& a, void* stream)
{
    const unsigned grid = deal_ctas(a.mat, a.n);
    if (!grid) return 0;
    if (out_dtype == 1) unpack_kernel<bf16><<<grid, kPackWarps * 32, 0, static_cast<cudaStream_t>(stream)>>>(a);
    else unpack_kernel<float><<<grid, kPackWarps * 32, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return static_cast<int>(cudaGetLastError());
}

}  // namespace randes
