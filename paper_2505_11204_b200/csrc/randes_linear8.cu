// Products of two matrices in eight bits:  y[t][r] = sum over blocks b of 2^(ex[t][b] + ew[r][b]) sum_c x[t][c] w[r][c]
//
// The tensor core multiplies by the blocks' scales itself (kind::mxf8f6f4: a power of two per row and 32 columns, taken from tensor
// memory), so sums stay in fp32 in tensor memory over all columns and come out once. A block of 128 columns is four
// products of 32 that use one scale; the word of a row holds the scales of four blocks and the instruction names the byte, so
// scales are copied to tensor memory once per 512 columns.
//
// w is operand A (128 rows: tensor memory lanes), x operand B (16 to 128 tokens: columns): few tokens waste nothing, and a warp of
// the epilogue writes 32 neighbouring outputs of a token whatever the row's alignment.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "randes_packed.cuh"
#include "randes_packed8.cuh"

namespace cg = cooperative_groups;

namespace randes {

static __device__ unsigned int g_linear8_giveups;   // CTAs that gave up on a wait (0 in a healthy run)

namespace {

using namespace device;

constexpr int kThreads8 = 192;                      // warp 0 copies, warp 1 products, warps 2-5 results
constexpr uint32_t kTile = 16384, kScales = 512;    // bytes: codes of 128 x 128, scale words of 128 rows

__device__ __forceinline__ void bar_init_n(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// 32 rows of 16 bytes (the scale words of 128 rows) into four columns of tensor memory, for each of the four groups of lanes
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void tc_load16(uint32_t t, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(t)
        : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Operand descriptors: rows of 128 bytes in the 128-byte swizzle, 8 rows 1024 bytes apart; scales without a swizzle, 8 rows of
// 16 bytes 128 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t saddr)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(128 >> 4) << 32) | (1ull << 46);
}

// A wait that ends: when it runs out, or when another role of the CTA has given up, it says so.
__device__ __forceinline__ bool wait8(uint32_t bar, uint32_t parity, volatile uint32_t* aborted)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 15u) == 15u && *aborted) return false;
    }
    if (atomicExch(const_cast<uint32_t*>(aborted), 1u) == 0u) atomicAdd(&g_linear8_giveups, 1u);
    return false;
}

__device__ __forceinline__ void store_y(const Linear8Args& a, uint32_t token, uint32_t row, float v)
{
    const size_t at = static_cast<size_t>(token) * a.y_stride + row;
    if (a.y_bf16) static_cast<bf16*>(a.y)[at] = __float2bfloat16_rn(v);
    else static_cast<float*>(a.y)[at] = v;
}

// N tokens to a tile.
template <int N> struct Geom8 {
    static constexpr uint32_t kStage = kTile + N * 128 + 2 * kScales;
    static constexpr int kStages = (227 * 1024 - 1024 - 512) / kStage;
    static constexpr uint32_t kScaleCols = 2 * N;                       // tensor memory: two accumulators, then two sets of scales
    static constexpr uint32_t kTmem = 2 * N + 16 <= 64 ? 64 : (2 * N + 16 <= 128 ? 128 : (2 * N + 16 <= 256 ? 256 : 512));
    // instruction descriptor: e4m3 both, fp32 sums, scales as exponents; bits 4-5 and 29-30 will say which byte of the scale words of B and A
    static constexpr uint32_t kIdesc = (N >> 3 << 17) | (1u << 23) | (128 >> 4 << 24);
    static constexpr uint32_t kBars = 2 * kStages + 7;                  // full, empty; scales free, sums full, sums free (two each); drained
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStage + 8 * kBars + 16;
    static_assert(kStage % 1024 == 0 && 8 * kBars + 16 <= 512, "stages on the swizzle's boundary");
};

template <int N> __global__ void __launch_bounds__(kThreads8, 1) linear8_kernel(const Linear8Args a)
{
    typedef Geom8<N> G;
    constexpr int S = G::kStages;
    extern __shared__ unsigned char smem_raw[];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t raw = static_cast<uint32_t>(__cvta_generic_to_shared(smem_raw)), base = (raw + 1023u) & ~1023u;
    unsigned char* gen = smem_raw + (base - raw);
    const uint32_t bars = base + S * G::kStage;
    auto full = [&](uint32_t s) { return bars + 8 * s; };
    auto empty = [&](uint32_t s) { return bars + 8 * (S + s); };
    auto scales_free = [&](uint32_t b) { return bars + 8 * (2 * S + b); };
    auto sums_full = [&](uint32_t b) { return bars + 8 * (2 * S + 2 + b); };
    auto sums_free = [&](uint32_t b) { return bars + 8 * (2 * S + 4 + b); };
    const uint32_t drained = bars + 8 * (2 * S + 6);
    volatile uint32_t* words = reinterpret_cast<volatile uint32_t*>(gen + S * G::kStage + 8 * G::kBars);      // tensor memory's address, give-up flag
    volatile uint32_t* aborted = words + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ranks = 1u << a.log_ranks, rank = blockIdx.x & (ranks - 1);
    const Packed8Layout lw(a.rows, a.cols), lx(a.n_tokens, a.cols);
    const uint32_t k0 = static_cast<uint32_t>(static_cast<uint64_t>(lw.col_blocks) * rank >> a.log_ranks);
    const uint32_t k1 = static_cast<uint32_t>(static_cast<uint64_t>(lw.col_blocks) * (rank + 1) >> a.log_ranks);
    const uint32_t token_tiles = (a.n_tokens + N - 1) / N, tiles = lw.row_tiles * token_tiles;
    const uint32_t tile0 = blockIdx.x >> a.log_ranks, tile_step = gridDim.x >> a.log_ranks;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < S; ++s) { bar_init(full(s)); bar_init(empty(s)); }
        for (uint32_t b = 0; b < 2; ++b) { bar_init(scales_free(b)); bar_init(sums_full(b)); bar_init_n(sums_free(b), 128); }
        bar_init(drained);
        *aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(bars + 8 * G::kBars), "r"(G::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = words[0];

    if (warp == 0) {
        if (lane == 0) {
            const char *w = static_cast<const char*>(a.w), *x = static_cast<const char*>(a.x);
            uint32_t it = 0;
            bool ok = true;
            for (uint32_t tile = tile0; ok && tile < tiles; tile += tile_step) {
                const uint32_t rt = tile / token_tiles, n0 = (tile - rt * token_tiles) * N, xt = n0 >> 7;
                for (uint32_t kb = k0; kb < k1; ++kb, ++it) {
                    const uint32_t s = it % S, st = base + s * G::kStage;
                    if (!(ok = wait8(empty(s), (it / S & 1u) ^ 1u, aborted))) break;
                    const bool first = kb == k0 || (kb & 3u) == 0;
                    bar_expect(full(s), kTile + N * 128 + (first ? 2 * kScales : 0));
                    bulk_copy(st, w + lw.tile(rt, kb), kTile, full(s));
                    bulk_copy(st + kTile, x + lx.tile(xt, kb) + (n0 & 127) * 128, N * 128, full(s));
                    if (first) {
                        bulk_copy(st + kTile + N * 128, w + lw.scales(rt, kb >> 2), kScales, full(s));
                        bulk_copy(st + kTile + N * 128 + kScales, x + lx.scales(xt, kb >> 2), kScales, full(s));
                    }
                }
            }
            if (*aborted)      // what is under way has to land before the CTA's shared memory is released
                for (uint32_t i = it > S ? it - S : 0; i < it; ++i) bar_wait(full(i % S), i / S & 1u);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t it = 0, group = 0, turn = 0;
            bool ok = true;
            for (uint32_t tile = tile0; ok && tile < tiles; tile += tile_step, ++turn) {
                const uint32_t acc = tmem + (turn & 1u) * N;
                if (!(ok = wait8(sums_free(turn & 1u), (turn >> 1 & 1u) ^ 1u, aborted))) break;
                tc_after();
                for (uint32_t kb = k0; kb < k1; ++kb, ++it) {
                    const uint32_t s = it % S, st = base + s * G::kStage;
                    if (!(ok = wait8(full(s), it / S & 1u, aborted))) break;
                    tc_after();
                    if (kb == k0 || (kb & 3u) == 0) {
                        ++group;      // of scales; the set is free once the products of the group before last are done
                        if (!(ok = wait8(scales_free(group & 1u), (group >> 1 & 1u) ^ (group & 1u), aborted))) break;
                        const uint32_t to = tmem + G::kScaleCols + (group & 1u) * 8;
                        tc_copy_scales(to, scales_desc(st + kTile + N * 128));
                        tc_copy_scales(to + 4, scales_desc(st + kTile + N * 128 + kScales));
                    }
                    const uint32_t sa = tmem + G::kScaleCols + (group & 1u) * 8, id = (kb & 3u) << 29 | (kb & 3u) << 4 | G::kIdesc;
                    const uint64_t da = operand_desc(st), db = operand_desc(st + kTile);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) tc_mma8(acc, da + 2 * k, db + 2 * k, id, sa, sa + 4, kb > k0 || k ? 1u : 0u);
                    tc_commit(empty(s));
                    if ((kb & 3u) == 3u || kb + 1 == k1) tc_commit(scales_free(group & 1u));
                }
                if (ok) tc_commit(sums_full(turn & 1u));
            }
            if (!ok) {
                tc_commit(drained);
                bar_wait(drained, 0);
            }
        }
        __syncwarp();
    } else {
        const uint32_t quarter = warp & 3, lanes = quarter * 32 << 16;
        uint32_t turn = 0;
        bool ok = true;
        for (uint32_t tile = tile0; tile < tiles; tile += tile_step, ++turn) {
            const uint32_t rt = tile / token_tiles, n0 = (tile - rt * token_tiles) * N, row = rt * 128 + quarter * 32 + lane;
            ok = ok && wait8(sums_full(turn & 1u), turn >> 1 & 1u, aborted);
            ok = __all_sync(~0u, ok);
            tc_after();
#pragma unroll 1
            for (uint32_t j0 = 0; j0 < N; j0 += 16) {
                uint32_t v[16];
                if (ok) {
                    tc_load16(tmem + lanes + (turn & 1u) * N + j0, v);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = 0x7FFFFFFFu;      // a sum that was not made is NaN
                }
                if (ranks > 1) {      // the ring is idle: one tile to a cluster, and its products are done
                    float* part = reinterpret_cast<float*>(gen);
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(j0 + j) * 128 + quarter * 32 + lane] = __uint_as_float(v[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (n0 + j0 + j < a.n_tokens && row < a.rows) store_y(a, n0 + j0 + j, row, __uint_as_float(v[j]));
                }
            }
            tc_before();
            bar_arrive(sums_free(turn & 1u));
        }
    }
    if (ranks > 1) {
        // each CTA adds its share of the tokens over all CTAs, in their order
        cluster.sync();
        const uint32_t rt = tile0 / token_tiles, n0 = (tile0 - rt * token_tiles) * N;
        const uint32_t row = rt * 128 + (threadIdx.x & 127);
        if (threadIdx.x < 128 && row < a.rows) {
            const float* part = reinterpret_cast<const float*>(gen);
            bool bad = false;
            for (uint32_t k = 0; k < ranks; ++k) bad = bad || *cluster.map_shared_rank(const_cast<uint32_t*>(aborted), k);
            for (uint32_t j = rank; j < N && n0 + j < a.n_tokens; j += ranks) {
                float y = 0.f;
                for (uint32_t k = 0; k < ranks; ++k) y += cluster.map_shared_rank(part, k)[j * 128 + threadIdx.x];
                store_y(a, n0 + j, row, bad ? __uint_as_float(0x7FFFFFFFu) : y);
            }
        }
        cluster.sync();      // nobody leaves while its sums may still be read
    }
    tc_before();
    __syncthreads();
    if (warp == 1) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(G::kTmem) : "memory");
    }
}

constexpr int kDevices8 = 64;

template <int N> int run_linear8(Linear8Args& a, int sm_count, int device, cudaStream_t stream)
{
    typedef Geom8<N> G;
    static std::atomic<bool> granted[kDevices8];
    if (device >= kDevices8 || !granted[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(linear8_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(G::kSmem));
        if (e != cudaSuccess) return static_cast<int>(e);
        if (device < kDevices8) granted[device].store(true, std::memory_order_relaxed);
    }
    const Packed8Layout lw(a.rows, a.cols);
    const uint64_t tiles = static_cast<uint64_t>(lw.row_tiles) * ((a.n_tokens + N - 1) / N);
    if (tiles > 0x7FFFFFFFu) return static_cast<int>(cudaErrorInvalidValue);
    a.log_ranks = 0;      // CTAs share a tile's columns as long as all fit the SMs at once
    while (a.log_ranks < 3 && (tiles << (a.log_ranks + 1)) <= static_cast<uint64_t>(sm_count) && (2u << a.log_ranks) <= lw.col_blocks) ++a.log_ranks;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.log_ranks ? tiles << a.log_ranks : std::min<uint64_t>(tiles, sm_count)));
    cfg.blockDim = dim3(kThreads8);
    cfg.dynamicSmemBytes = G::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 1u << a.log_ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = a.log_ranks ? 1 : 0;
    return static_cast<int>(cudaLaunchKernelEx(&cfg, linear8_kernel<N>, a));
}

}  // namespace

int launch_linear8(Linear8Args& a, int sm_count, int device, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.n_tokens <= 16) return run_linear8<16>(a, sm_count, device, s);
    if (a.n_tokens <= 32) return run_linear8<32>(a, sm_count, device, s);
    if (a.n_tokens <= 64) return run_linear8<64>(a, sm_count, device, s);
    return run_linear8<128>(a, sm_count, device, s);
}

int linear8_giveups(unsigned int* count)
{
    return static_cast<int>(cudaMemcpyFromSymbol(count, g_linear8_giveups, sizeof(unsigned int)));
}

}  // namespace randes
