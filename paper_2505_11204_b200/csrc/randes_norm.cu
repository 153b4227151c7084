// Root-mean-square norm of rows with the residual's addition in front and eight bits behind, and its gradient.
//
//     h = x + r, rounded to the activations' type        s = 1 / sqrt( mean h^2 + eps )        y = (h s) gain
//     n = h s,  g = dy gain:     dx = s ( g - n mean(g n) ) + dh        dgain = sum over rows of dy n
// The norm is taken of h as it is stored, so that the backward pass, which reads h, sees what the forward pass saw; dx is the
// gradient of x and of r alike, dh what reaches h past the norm. Sums run in fp32; a sum of squares that leaves fp32 is taken
// again in fp64.
//
// One pass: a row stays in registers, eight neighbouring columns to a thread and step, between the loads and the sum's return,
// so 16 neighbouring lanes hold a block of 128 columns and its scale in eight bits is four shuffles away.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "randes_packed8.cuh"

namespace randes {
namespace {

using namespace device;

// Threads to a row, columns of a row per thread (8 CHUNKS), rows to a CTA: warps take rows of their own up to 1024 columns.
template <int THREADS> constexpr int kRowsPerCta = THREADS == 32 ? 4 : 1;

__device__ __forceinline__ float gain_at(const void* gain, bool bf, uint32_t c)
{
    return bf ? Store<bf16>::load1(static_cast<const bf16*>(gain) + c) : __ldg(static_cast<const float*>(gain) + c);
}
__device__ __forceinline__ void load_gain(const void* gain, bool bf, uint32_t c, uint32_t cols, float (&v)[8])
{
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) v[e] = gain && c + e < cols ? gain_at(gain, bf, c + e) : 1.f;
}

template <typename V> __device__ __forceinline__ V warp_sum(V v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// The sum over the threads of a row, in every one of them, always in the same order. `part`: a word per warp, not touched again
// before the row's threads have met once more.
template <int THREADS, typename V> __device__ __forceinline__ V row_sum(V v, V* part, int tid)
{
    v = warp_sum(v);
    if (THREADS == 32) return v;
    if ((tid & 31) == 0) part[tid >> 5] = v;
    __syncthreads();
    V all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) all += part[w];
    return all;
}

// A row's columns 8 (k THREADS + t) .. + 7, k < CHUNKS, all loads before the first use.
template <typename T, int THREADS, int CHUNKS>
__device__ __forceinline__ void load_row(const T* row, bool vec, uint32_t cols, int t, float* scratch, float (&v)[CHUNKS][8])
{
    const int lane = t & 31;
    if (vec) {
        Octet<T> o[CHUNKS];
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) o[k] = load_octet(row, (k * THREADS + t) * 8, cols);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) widen(o[k], v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) load_loose(row, (k * THREADS + t) * 8, cols, lane, v[k]);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) turn_in(v[k], scratch, lane);
    }
}
template <typename T> __device__ __forceinline__ void store_chunk(T* row, bool vec, uint32_t c, uint32_t cols, const float (&v)[8], float* scratch, int lane)
{
    if (vec) store_octet(row, c, cols, v);
    else store_loose(row, c, cols, v, scratch, lane);
}
// Eight columns into eight bits: the block's scale from its 16 lanes.
__device__ __forceinline__ void store8(char* dst, const Packed8Layout& lay, uint32_t r, uint32_t c, const float (&v)[8], int lane)
{
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max_bits(amax, magnitude(v[e]));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) amax = max_bits(amax, __shfl_xor_sync(~0u, amax, o));
    const uint32_t kb = c >> 7, e = block_scale(amax);
    if (kb >= lay.col_blocks) return;
    *reinterpret_cast<uint2*>(dst + lay.tile(r >> 7, kb) + code_at(r, c)) = codes8(v, amax, e);
    if ((lane & 15) == 0) dst[lay.scales(r >> 7, kb >> 2) + Packed8Layout::scale_word(r) + (kb & 3)] = static_cast<char>(e);
}

template <typename T, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS* kRowsPerCta<THREADS>) norm_kernel(const NormArgs a)
{
    constexpr int kWarps = THREADS * kRowsPerCta<THREADS> / 32;
    __shared__ __align__(16) float s_scratch[kWarps][256];
    __shared__ float s_part[THREADS == 32 ? 1 : kWarps];
    __shared__ double s_part64[THREADS == 32 ? 1 : kWarps];
    const int t = THREADS == 32 ? threadIdx.x & 31 : threadIdx.x, lane = t & 31;
    const uint32_t r = THREADS == 32 ? blockIdx.x * kRowsPerCta<THREADS> + (threadIdx.x >> 5) : blockIdx.x;
    if (THREADS == 32 && r >= a.rows) return;
    float* scratch = s_scratch[threadIdx.x >> 5];
    const uint32_t cols = a.cols;
    const Packed8Layout lay(a.rows, cols);

    float v[CHUNKS][8];
    load_row<T, THREADS, CHUNKS>(static_cast<const T*>(a.x) + r * a.x_stride, a.vec, cols, t, scratch, v);
    if (a.residual) {
        float d[CHUNKS][8];
        load_row<T, THREADS, CHUNKS>(static_cast<const T*>(a.residual) + r * a.residual_stride, a.vec, cols, t, scratch, d);
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] += d[k][e];
            widen(narrow<T>(v[k]), v[k]);                   // what is stored is what is normed
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const uint32_t c = (k * THREADS + t) * 8;
        if (a.h && c - 8 * lane < cols) store_chunk(static_cast<T*>(a.h) + r * a.h_stride, a.vec, c, cols, v[k], scratch, lane);
        if (a.kept8) store8(static_cast<char*>(a.kept8), lay, r, c, v[k], lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __fmaf_rn(v[k][e], v[k][e], ss);
    }
    ss = row_sum<THREADS>(ss, s_part, t);
    float s;
    if (ss == INFINITY) {                                   // the same for all threads of the row
        double wide = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) wide += static_cast<double>(v[k][e]) * v[k][e];
        s = static_cast<float>(1.0 / sqrt(row_sum<THREADS>(wide, s_part64, t) / cols + a.eps));
    } else {
        s = __frsqrt_rn(ss / cols + a.eps);
    }
    if (a.rstd && t == 0) a.rstd[r] = s;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const uint32_t c = (k * THREADS + t) * 8;
        if (c - 8 * lane >= cols) break;                    // the same for a warp
        float w[8];
        load_gain(a.gain, a.gain_bf16, c, cols, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = c + e < cols ? v[k][e] * s * w[e] : 0.f;      // (0 * NaN behind the row's end would spoil the block)
        if (a.y) store_chunk(static_cast<T*>(a.y) + r * a.y_stride, a.vec, c, cols, w, scratch, lane);
        if (a.y8) store8(static_cast<char*>(a.y8), lay, r, c, w, lane);
    }
}

// A CTA walks rows and keeps its share of dgain in registers; the shares of all CTAs are added in a fixed order by a second kernel.
template <typename T, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS* kRowsPerCta<THREADS>) norm_grad_kernel(const NormGradArgs a)
{
    constexpr int kWarps = THREADS * kRowsPerCta<THREADS> / 32;
    constexpr int kSum = THREADS == 32 ? 256 * CHUNKS : 1;
    __shared__ __align__(16) float s_scratch[kWarps][256];
    __shared__ float s_part[2][THREADS == 32 ? 1 : kWarps];
    __shared__ float s_sum[kSum];
    const int t = THREADS == 32 ? threadIdx.x & 31 : threadIdx.x, lane = t & 31;
    float* scratch = s_scratch[threadIdx.x >> 5];
    const uint32_t cols = a.cols;
    const Packed8Layout lay(a.rows, cols);
    const uint32_t step = gridDim.x * kRowsPerCta<THREADS>;
    float sum[CHUNKS][8] = {};
    uint32_t turn = 0;
    for (uint32_t r = blockIdx.x * kRowsPerCta<THREADS> + (THREADS == 32 ? threadIdx.x >> 5 : 0); r < a.rows; r += step, turn ^= 1) {
        float n[CHUNKS][8], g[CHUNKS][8];
        const float s = __ldg(a.rstd + r);
        if (a.kept8) {
            const char* src = static_cast<const char*>(a.kept8);
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                const uint32_t c = (k * THREADS + t) * 8, kb = c >> 7;
                uint2 w = make_uint2(0, 0);
                uint32_t e = 0;
                if (kb < lay.col_blocks) {
                    w = __ldcs(reinterpret_cast<const uint2*>(src + lay.tile(r >> 7, kb) + code_at(r, c)));
                    e = __ldg(reinterpret_cast<const unsigned char*>(src + lay.scales(r >> 7, kb >> 2) + Packed8Layout::scale_word(r) + (kb & 3)));
                }
                values4(w.x, block_unit(e), n[k]);
                values4(w.y, block_unit(e), n[k] + 4);
                if (c + 8 > cols)
#pragma unroll
                    for (int j = 0; j < 8; ++j) n[k][j] = c + j < cols ? n[k][j] : 0.f;      // (codes behind the row's end may be NaN)
            }
        } else {
            load_row<T, THREADS, CHUNKS>(static_cast<const T*>(a.h) + r * a.h_stride, a.vec, cols, t, scratch, n);
        }
        load_row<T, THREADS, CHUNKS>(static_cast<const T*>(a.dy) + r * a.dy_stride, a.vec, cols, t, scratch, g);
        float inner = 0.f;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            float w[8];
            load_gain(a.gain, a.gain_bf16, (k * THREADS + t) * 8, cols, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[k][e] *= s;
                sum[k][e] = __fmaf_rn(g[k][e], n[k][e], sum[k][e]);
                g[k][e] *= w[e];
                inner = __fmaf_rn(g[k][e], n[k][e], inner);
            }
        }
        inner = row_sum<THREADS>(inner, s_part[turn], t) / cols;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const uint32_t c = (k * THREADS + t) * 8;
            if (c - 8 * lane >= cols) break;
            float d[8];
            if (a.dh) {
                const T* row = static_cast<const T*>(a.dh) + r * a.dh_stride;
                if (a.vec) {
                    widen(load_octet(row, c, cols), d);
                } else {
                    load_loose(row, c, cols, lane, d);
                    turn_in(d, scratch, lane);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = s * __fmaf_rn(-n[k][e], inner, g[k][e]);
                d[e] = a.dh ? v + d[e] : v;
            }
            store_chunk(static_cast<T*>(a.dx) + r * a.dx_stride, a.vec, c, cols, d, scratch, lane);
        }
    }
    if (!a.dgain) return;
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * cols;
    if (THREADS == 32) {                                    // the warps of a CTA, one after the other
        for (int w = 0; w < kWarps; ++w) {
            __syncthreads();
            if (static_cast<int>(threadIdx.x >> 5) != w) continue;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float& to = s_sum[e * 32 * CHUNKS + k * 32 + lane];
                    to = w ? to + sum[k][e] : sum[k][e];
                }
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < cols; c += THREADS * kRowsPerCta<THREADS>)
            out[c] = s_sum[(c & 7) * 32 * CHUNKS + (c >> 3)];
    } else {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = (k * THREADS + t) * 8 + e;
                if (c < cols) out[c] = sum[k][e];
            }
    }
}

constexpr int kSumRows = 16;
__global__ void __launch_bounds__(32 * kSumRows) norm_gain_kernel(const float* partial, uint32_t n, uint32_t cols, float* dgain)
{
    __shared__ float s[kSumRows][33];
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float v = 0.f;
    if (c < cols)
        for (uint32_t i = y; i < n; i += kSumRows) v += partial[static_cast<size_t>(i) * cols + c];
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < kSumRows; ++i) v += s[i][x];
        dgain[c] = v;
    }
}

template <typename T, int THREADS, int CHUNKS> int run_norm(const NormArgs& a, cudaStream_t stream)
{
    constexpr uint32_t kRows = kRowsPerCta<THREADS>;
    norm_kernel<T, THREADS, CHUNKS><<<(a.rows + kRows - 1) / kRows, THREADS * kRows, 0, stream>>>(a);
    return static_cast<int>(cudaGetLastError());
}
// Calls f with the row's form: threads to a row and runs of 8 columns per thread.
template <typename F> int by_width(uint32_t cols, F&& f)
{
    if (cols <= 256) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (cols <= 512) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 2>());
    if (cols <= 1024) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
    if (cols <= 2048) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    if (cols <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    if (cols <= 8192) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    if (cols <= 16384) return f(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
}
// CTAs that walk the rows of a backward pass: the rows, or what the 148 SMs hold at a time (a constant, so that sums are the same
// on every device and the workspace is known without one).
uint32_t grad_ctas(uint32_t rows, uint32_t cols)
{
    const uint32_t per_sm = cols <= 1024 ? 8 : (cols <= 4096 ? 4 : (cols <= 8192 ? 2 : 1));
    const uint32_t ctas = cols <= 1024 ? (rows + 3) / 4 : rows;
    return std::min(ctas, per_sm * 148u);
}

}  // namespace

int launch_norm(int dtype, const NormArgs& a, void* stream)
{
    return by_width(a.cols, [&](auto threads, auto chunks) {
        constexpr int T = decltype(threads)::value, C = decltype(chunks)::value;
        return dtype ? run_norm<bf16, T, C>(a, static_cast<cudaStream_t>(stream)) : run_norm<float, T, C>(a, static_cast<cudaStream_t>(stream));
    });
}

size_t norm_grad_workspace(uint32_t rows, uint32_t cols)
{
    return static_cast<size_t>(grad_ctas(rows, cols)) * cols * sizeof(float);
}

int launch_norm_grad(int dtype, const NormGradArgs& a, int* launched, void* stream)
{
    *launched = 0;
    const uint32_t ctas = grad_ctas(a.rows, a.cols);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int e = by_width(a.cols, [&](auto threads, auto chunks) {
        constexpr int T = decltype(threads)::value, C = decltype(chunks)::value;
        if (dtype) norm_grad_kernel<bf16, T, C><<<ctas, T * kRowsPerCta<T>, 0, s>>>(a);
        else norm_grad_kernel<float, T, C><<<ctas, T * kRowsPerCta<T>, 0, s>>>(a);
        return static_cast<int>(cudaGetLastError());
    });
    if (e) return e;
    *launched = 1;
    if (!a.dgain) return 0;
    norm_gain_kernel<<<(a.cols + 31) / 32, 32 * kSumRows, 0, s>>>(a.partial, ctas, a.cols, a.dgain);
    const int e2 = static_cast<int>(cudaGetLastError());
    if (!e2) *launched = 2;
    return e2;
}

}  // namespace randes
