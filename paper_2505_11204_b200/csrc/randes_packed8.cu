// Weights and activations in eight bits: written row by row (or straight from base and superposition), written turned, and
// read back.
//
// Per block of 128 columns of a row (the last may be shorter), with a = max |w|:
//     e = the least integer, -100 at least, with a <= 448 * 2^e        code = e4m3( w * 2^-e )        the code stands for code * 2^e
// A block that holds a NaN or an infinity gets NaN in every code. The scale is a power of two for three reasons: the tensor
// core multiplies such scales itself, so a product needs no pass over its partial sums; w * 2^-e is exact, so there is one
// rounding, of at most 2^-4 of the value (down to 2^-6 of the block's unit 2^e; 2^-10 units below that); and a matrix cut into
// blocks along its other axis keeps its values, but for those that are subnormal in their new block.
//
// Layout: tiles of 128 rows x 128 columns of codes, [row tile][column block], 16 KiB each: row r at 128 r, its 16-byte piece p at
// place p ^ (r % 8) -- the image that the tensor core's 128-byte swizzle expects in shared memory, so that one plain bulk copy
// brings an operand. Behind the codes the scales, exponents + 127 as bytes, [row tile][group of four column blocks] 512 bytes: the
// word of row r (its four blocks) at 16 (r % 32) + 4 (r / 32 % 4), as the tensor core wants them in tensor memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "randes_packed8.cuh"

namespace randes {
namespace {

using namespace device;

constexpr int kWarps8 = 4;                    // warps per CTA of pack and unpack
constexpr uint32_t kRows8 = 4;                // rows per warp
constexpr uint32_t kCtaRows8 = kWarps8 * kRows8;

template <typename Args> __device__ __forceinline__ uint32_t matrix_of(const Args& a, uint32_t cta)
{
    uint32_t i = 0;
    while (i + 1 < a.n && cta >= a.mat[i + 1].first_cta) ++i;
    return i;
}

// A warp takes rows r0 .. r0 + 3 of 512 columns: two runs of 256, lane l holding columns 8 l .. 8 l + 7 of either.
template <typename T, typename M, bool RETRIEVE, uint32_t BATCH>
__global__ void __launch_bounds__(kWarps8 * 32) pack8_kernel(const __grid_constant__ Pack8Batch<BATCH> a)
{
    __shared__ __align__(16) float s_scratch[kWarps8][256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Pack8Matrix& m = a.mat[BATCH == 1 ? 0 : matrix_of(a, blockIdx.x)];
    const Packed8Layout lay(m.rows, m.cols);
    const uint32_t cta = blockIdx.x - m.first_cta, rb = cta / lay.groups, g = cta - rb * lay.groups;
    const uint32_t r0 = rb * kCtaRows8 + warp * kRows8, cols = m.cols;
    if (r0 >= m.rows) return;
    const uint32_t n = min(kRows8, m.rows - r0);
    char* dst = static_cast<char*>(m.dst);
    uint32_t word[kRows8] = {};
#pragma unroll
    for (uint32_t half = 0; half < 2; ++half) {
        const uint32_t c = g * 512 + half * 256 + lane * 8, kb = c >> 7;
        if (g * 512 + half * 256 >= cols) break;
        float v[kRows8][8];
        auto read = [&](const auto* p, uint64_t stride, bool vec, float (&to)[kRows8][8]) {
            typedef typename std::remove_const<typename std::remove_pointer<decltype(p)>::type>::type E;
            if (vec) {
                Octet<E> o[kRows8];
#pragma unroll
                for (uint32_t i = 0; i < kRows8; ++i)
                    if (i < n) o[i] = load_octet(p + (r0 + i) * stride, c, cols);
#pragma unroll
                for (uint32_t i = 0; i < kRows8; ++i)
                    if (i < n) widen(o[i], to[i]);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < kRows8; ++i)
                    if (i < n) load_loose(p + (r0 + i) * stride, c, cols, lane, to[i]);
#pragma unroll
                for (uint32_t i = 0; i < kRows8; ++i)
                    if (i < n) turn_in(to[i], s_scratch[warp], lane);
            }
        };
        read(static_cast<const T*>(m.src), m.stride, m.vec & 1u, v);
        if (RETRIEVE) {
            float d[kRows8][8];
            read(static_cast<const M*>(m.m), cols, m.vec & 2u, d);
            uint32_t bits = 0;
            if (m.flip) {
                const uint4 blk = philox4x32_10(kb, m.slot, kTagSign, a.task.id, a.task.key0, a.task.key1);
                const uint32_t q = (c >> 5) & 3;
                bits = (q == 0 ? blk.x : (q == 1 ? blk.y : (q == 2 ? blk.z : blk.w))) >> (c & 31);
            }
#pragma unroll
            for (uint32_t i = 0; i < kRows8; ++i)
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) v[i][e] = __fmaf_rn(a.lambda, flip(d[i][e], (bits >> e) << 31), v[i][e]);
        }
#pragma unroll
        for (uint32_t i = 0; i < kRows8; ++i) {
            if (i >= n) break;
            uint32_t amax = 0;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) amax = max_bits(amax, magnitude(v[i][e]));
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) amax = max_bits(amax, __shfl_xor_sync(~0u, amax, o));
            const uint32_t e = block_scale(amax), r = r0 + i;
            if (kb < lay.col_blocks) *reinterpret_cast<uint2*>(dst + lay.tile(r >> 7, kb) + code_at(r, c)) = codes8(v[i], amax, e);
            word[i] |= (__shfl_sync(~0u, e, 0) | (__shfl_sync(~0u, e, 16) << 8)) << (16 * half);
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < kRows8; ++i)
        if (i < n && lane == static_cast<int>(i))
            *reinterpret_cast<uint32_t*>(dst + lay.scales(r0 >> 7, g) + Packed8Layout::scale_word(r0 + i)) = word[i];
}

template <typename T, uint32_t BATCH> __global__ void __launch_bounds__(kWarps8 * 32) unpack8_kernel(const __grid_constant__ Unpack8Batch<BATCH> a)
{
    __shared__ __align__(16) float s_scratch[kWarps8][256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Unpack8Matrix& m = a.mat[BATCH == 1 ? 0 : matrix_of(a, blockIdx.x)];
    const Packed8Layout lay(m.rows, m.cols);
    const uint32_t cta = blockIdx.x - m.first_cta, rb = cta / lay.groups, g = cta - rb * lay.groups;
    const uint32_t r0 = rb * kCtaRows8 + warp * kRows8, cols = m.cols;
    if (r0 >= m.rows) return;
    const uint32_t n = min(kRows8, m.rows - r0);
    const char* src = static_cast<const char*>(m.src);
    uint2 codes[2][kRows8];
    uint32_t word[kRows8];
#pragma unroll
    for (uint32_t i = 0; i < kRows8; ++i) {
        if (i >= n) break;
        const uint32_t r = r0 + i;
        word[i] = __ldg(reinterpret_cast<const uint32_t*>(src + lay.scales(r >> 7, g) + Packed8Layout::scale_word(r)));
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half) {
            const uint32_t c = g * 512 + half * 256 + lane * 8;
            if (c >> 7 < lay.col_blocks) codes[half][i] = __ldcs(reinterpret_cast<const uint2*>(src + lay.tile(r >> 7, c >> 7) + code_at(r, c)));
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < kRows8; ++i) {
        if (i >= n) break;
        T* row = static_cast<T*>(m.dst) + (r0 + i) * m.stride;
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half) {
            const uint32_t c = g * 512 + half * 256 + lane * 8;
            if (g * 512 + half * 256 >= cols) break;
            float v[8];
            const float unit = block_unit((word[i] >> (8 * ((c >> 7) & 3))) & 0xFFu);
            values4(codes[half][i].x, unit, v);
            values4(codes[half][i].y, unit, v + 4);
            if (m.vec) store_octet(row, c, cols, v);
            else store_loose(row, c, cols, v, s_scratch[warp], lane);
        }
    }
}

// A tile of 128 x 128 in blocks along its columns, and with BOTH in blocks along its rows too, out of one read. A thread holds 8 rows
// x 8 columns; the greatest magnitudes of the columns meet in shared memory; the codes of a column are turned there, 8-byte pieces
// exchanged by the column's octet so that neither the writes nor the reads meet in a bank.
template <typename T> __device__ __forceinline__ void load_sub(const Turn8Args& a, uint32_t r0, uint32_t c, float* scratch, int lane, float (&v)[8][8])
{
    const T* src = static_cast<const T*>(a.src);
    if (a.vec) {
        Octet<T> o[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (r0 + i < a.rows) o[i] = load_octet(src + (r0 + i) * a.stride, c, a.cols);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (r0 + i < a.rows) widen(o[i], v[i]);
            else
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    } else {
        // half a warp reads a row's 128 columns: 16 neighbours at a time
        const uint32_t l = lane & 15, first = c - 8 * l;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
                const uint32_t at = first + 16 * k + l;
                v[i][k] = r0 + i < a.rows && at < a.cols ? Store<T>::load1(src + (r0 + i) * a.stride + at) : 0.f;
            }
        float* mine = scratch + (lane >> 4) * 128;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) mine[16 * k + l] = v[i][k];
            __syncwarp();
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) v[i][e] = mine[8 * l + e];
            __syncwarp();
        }
    }
}
template <> __device__ __forceinline__ void load_sub<uint8_t>(const Turn8Args& a, uint32_t r0, uint32_t c, float*, int, float (&v)[8][8])
{
    const Packed8Layout lay(a.rows, a.cols);
    const char* src = static_cast<const char*>(a.src);
    const uint32_t rt = r0 >> 7, kb = c >> 7;
    uint2 w[8];
    uint32_t e[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        w[i] = make_uint2(0, 0);
        e[i] = 0;
        if (r0 + i < a.rows) {
            w[i] = __ldcs(reinterpret_cast<const uint2*>(src + lay.tile(rt, kb) + code_at(r0 + i, c)));
            e[i] = __ldg(reinterpret_cast<const unsigned char*>(src + lay.scales(rt, kb >> 2) + Packed8Layout::scale_word(r0 + i) + (kb & 3)));
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        values4(w[i].x, block_unit(e[i]), v[i]);
        values4(w[i].y, block_unit(e[i]), v[i] + 4);
    }
}

constexpr int kTurnThreads = 256;

template <typename T, bool BOTH> __global__ void __launch_bounds__(kTurnThreads, 2) turn8_kernel(const Turn8Args a)
{
    __shared__ __align__(16) float s_scratch[kTurnThreads / 32][256];
    __shared__ __align__(16) uint32_t s_max[kTurnThreads / 32][128];
    __shared__ __align__(16) unsigned char s_tile[128 * 128];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t blocks = (a.cols + 127) / 128, rt = blockIdx.x / blocks, kb = blockIdx.x - rt * blocks;
    const uint32_t l = tid & 15, rg = tid >> 4;
    const uint32_t r0 = rt * 128 + rg * 8, c = kb * 128 + l * 8;
    float v[8][8];
    load_sub<T>(a, r0, c, s_scratch[warp], lane, v);

    uint32_t top[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) top[e] = max_bits(top[e], magnitude(v[i][e]));
#pragma unroll
    for (int e = 0; e < 8; ++e) top[e] = max_bits(top[e], __shfl_xor_sync(~0u, top[e], 16));
    if (lane < 16) {
        reinterpret_cast<uint4*>(s_max[warp])[2 * l] = make_uint4(top[0], top[1], top[2], top[3]);
        reinterpret_cast<uint4*>(s_max[warp])[2 * l + 1] = make_uint4(top[4], top[5], top[6], top[7]);
    }
    if (BOTH) {
        const Packed8Layout lay(a.rows, a.cols);
        char* dst = static_cast<char*>(a.dst);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t amax = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = max_bits(amax, magnitude(v[i][e]));
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) amax = max_bits(amax, __shfl_xor_sync(~0u, amax, o));
            const uint32_t e = block_scale(amax), r = r0 + i;
            if (r < a.rows) {
                *reinterpret_cast<uint2*>(dst + lay.tile(rt, kb) + code_at(r, c)) = codes8(v[i], amax, e);
                if (l == 0) dst[lay.scales(rt, kb >> 2) + Packed8Layout::scale_word(r) + (kb & 3)] = static_cast<char>(e);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTurnThreads / 32; ++w) {
        const uint4 p = reinterpret_cast<const uint4*>(s_max[w])[2 * l], q = reinterpret_cast<const uint4*>(s_max[w])[2 * l + 1];
        top[0] = max_bits(top[0], p.x); top[1] = max_bits(top[1], p.y); top[2] = max_bits(top[2], p.z); top[3] = max_bits(top[3], p.w);
        top[4] = max_bits(top[4], q.x); top[5] = max_bits(top[5], q.y); top[6] = max_bits(top[6], q.z); top[7] = max_bits(top[7], q.w);
    }
    const Packed8Layout lay(a.cols, a.rows);
    char* turned = static_cast<char*>(a.turned);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t s = block_scale(top[e]);
        const float col[8] = {v[0][e], v[1][e], v[2][e], v[3][e], v[4][e], v[5][e], v[6][e], v[7][e]};
        *reinterpret_cast<uint2*>(s_tile + (l * 8 + e) * 128 + ((rg ^ l) << 3)) = codes8(col, top[e], s);
        if (rg == 0 && c + e < a.cols) turned[lay.scales(kb, rt >> 2) + Packed8Layout::scale_word(l * 8 + e) + (rt & 3)] = static_cast<char>(s);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t at = k * kTurnThreads + tid, row = at >> 3, piece = at & 7, f = row >> 3;      // f: what the row's pieces were exchanged by
        if (kb * 128 + row >= a.cols) break;
        const uint4 w = *reinterpret_cast<const uint4*>(s_tile + row * 128 + ((piece ^ (f >> 1)) << 4));
        const uint4 o = f & 1 ? make_uint4(w.z, w.w, w.x, w.y) : w;
        *reinterpret_cast<uint4*>(turned + lay.tile(kb, rt) + row * 128 + ((piece ^ (row & 7)) << 4)) = o;
    }
}

template <typename Args> uint32_t count_ctas(Args& a)
{
    uint32_t ctas = 0;
    for (uint32_t i = 0; i < a.n; ++i) {
        a.mat[i].first_cta = ctas;
        ctas += (a.mat[i].rows / kCtaRows8 + (a.mat[i].rows % kCtaRows8 != 0)) * Packed8Layout(a.mat[i].rows, a.mat[i].cols).groups;
    }
    return ctas;
}

template <typename T, typename M, bool RETRIEVE> int run_pack8(Pack8Args& a, void* stream)
{
    const uint32_t ctas = count_ctas(a);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.n == 1) pack8_kernel<T, M, RETRIEVE, 1><<<ctas, kWarps8 * 32, 0, s>>>(Pack8Batch<1>{{a.mat[0]}, 1, a.lambda, a.task});
    else pack8_kernel<T, M, RETRIEVE, kPackBatch><<<ctas, kWarps8 * 32, 0, s>>>(a);
    return static_cast<int>(cudaGetLastError());
}
template <typename T> int run_unpack8(Unpack8Args& a, void* stream)
{
    const uint32_t ctas = count_ctas(a);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.n == 1) unpack8_kernel<T, 1><<<ctas, kWarps8 * 32, 0, s>>>(Unpack8Batch<1>{{a.mat[0]}, 1});
    else unpack8_kernel<T, kPackBatch><<<ctas, kWarps8 * 32, 0, s>>>(a);
    return static_cast<int>(cudaGetLastError());
}
template <typename T> int run_turn8(const Turn8Args& a, void* stream)
{
    const uint32_t ctas = ((a.rows + 127) / 128) * ((a.cols + 127) / 128);
    if constexpr (sizeof(T) > 1) {      // (a checkpoint has its blocks along the rows already)
        if (a.dst) {
            turn8_kernel<T, true><<<ctas, kTurnThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
            return static_cast<int>(cudaGetLastError());
        }
    }
    turn8_kernel<T, false><<<ctas, kTurnThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return static_cast<int>(cudaGetLastError());
}

}  // namespace

int launch_pack8(int w_dtype, int m_dtype, bool retrieve, Pack8Args& a, void* stream)
{
    if (!retrieve) return w_dtype ? run_pack8<bf16, bf16, false>(a, stream) : run_pack8<float, float, false>(a, stream);
    if (w_dtype) return m_dtype ? run_pack8<bf16, bf16, true>(a, stream) : run_pack8<bf16, float, true>(a, stream);
    return m_dtype ? run_pack8<float, bf16, true>(a, stream) : run_pack8<float, float, true>(a, stream);
}

int launch_unpack8(int out_dtype, Unpack8Args& a, void* stream)
{
    return out_dtype ? run_unpack8<bf16>(a, stream) : run_unpack8<float>(a, stream);
}

int launch_turn8(int src_dtype, const Turn8Args& a, void* stream)
{
    if (src_dtype < 0) return run_turn8<uint8_t>(a, stream);
    return src_dtype ? run_turn8<bf16>(a, stream) : run_turn8<float>(a, stream);
}

}  // namespace randes
