// Products of 9 to 64 tokens with packed weights, on the fifth-generation tensor cores.
//
// The scale of a weight belongs to a row and a group of columns, so the tensor core can only add up within a group: codes
// (q / 64, exact in bf16) x activations over the columns of one group, in tensor memory; the group's sums then come back
// to registers and are added to the row's totals with the group's scale, one fp32 multiply-add each. A CTA works on 128
// rows and a contiguous run of column blocks over all segments (see randes_packed.cu for segments); the CTAs of a cluster
// share the rows and meet through distributed shared memory.
//
//   warps 0-7  workers. Per tile of 64 columns a warp decodes 16 rows of codes into the A operand (K-major, 128-byte
//              swizzle), all of them bring the tokens' activations into the B operand (signs applied; an fp32 activation
//              as three bf16 terms), then they take the group sums of the tile before out of tensor memory: a thread owns
//              one row and half the tokens.
//   warp 8     copies the records (one lane, bulk copies, two stages of 128 columns), owns tensor memory.
//   warp 9     issues tcgen05.mma (one lane): M = 128 rows, N = tokens of the segment rounded up to 16.
//
// Every wait is bounded; a CTA whose wait runs out raises a flag, all roles leave, what is in flight is waited for, tensor
// memory is freed, its sums become NaN and a device counter records the event.
#include <atomic>
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "randes_packed.cuh"

namespace cg = cooperative_groups;

namespace randes {

static __device__ unsigned int g_wide_giveups;     // CTAs that gave up waiting (0 in a healthy run)

namespace {

using namespace device;

constexpr int kWorkers = 8;                        // warps
constexpr int kThreads = (kWorkers + 2) * 32;
constexpr uint32_t kTileRows = 128;
constexpr uint32_t kRecStages = 2, kOpStages = 2, kAccs = 4;
constexpr uint32_t kATile = kTileRows * 128;       // 128 rows x 64 bf16

// ---- mbarriers with any count, bounded waits that also end when the CTA has given up
__device__ __forceinline__ void bar_init_n(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool wait_or_leave(uint32_t bar, uint32_t parity, volatile uint32_t* gone)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63u) == 63u && *gone) return false;
    }
    if (atomicExch(const_cast<uint32_t*>(gone), 1u) == 0u) atomicAdd(&g_wide_giveups, 1u);
    return false;
}

// ---- tcgen05
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_load16(uint32_t addr, uint32_t* v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr) : "memory");
}
// K-major operand of 64 bf16 columns (128 bytes) per row with the 128-byte swizzle: 16-byte chunk c of row r lies at
// chunk c ^ (r % 8) of its row; groups of eight rows 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr)
{
    return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// NT = 32 or 64 token columns.
template <int NT, typename XT, int GROUP> struct Wide {
    static constexpr bool HALF = GROUP == 32;
    static constexpr uint32_t kTerms = sizeof(XT) == 4 ? 3 : 1;
    static constexpr uint32_t kBlockTiles = GROUP == 128 ? 2 : 1;
    static constexpr uint32_t kCodeBytes = kBlockTiles * 4 * 512, kRecord = kCodeBytes + (HALF ? 256 : 128);
    static constexpr uint32_t kUnitBytes = 2 / kBlockTiles * kRecord;       // 64 rows x 128 columns
    static constexpr uint32_t kBTile = NT * 128;
    static constexpr uint32_t kOpBytes = kATile + kTerms * kBTile;
    static constexpr uint32_t kOpsAt = 0;                                   // 1024-byte aligned operands first
    static constexpr uint32_t kRecAt = kOpsAt + kOpStages * kOpBytes;
    static constexpr uint32_t kBarsAt = kRecAt + kRecStages * 2 * kUnitBytes;
    static constexpr uint32_t kYAt = kBarsAt + 256;
    static constexpr uint32_t kTmem = kAccs * NT;
    static size_t smem(uint32_t n_tokens) { return 1024 + kYAt + static_cast<size_t>(n_tokens) * kTileRows * sizeof(float); }
};

template <int NT, typename XT, int GROUP>
__global__ void __launch_bounds__(kThreads, 2) packed_wide_kernel(const __grid_constant__ PackedLinearArgs<kWideTokens> a)
{
    typedef Wide<NT, XT, GROUP> W;
    typedef Acts<XT> Act;
    constexpr uint32_t kLanes = 256 / NT, kCols = NT / 4, kChunks = kCols / 8;    // threads per token; columns and 16-byte chunks of each
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_at = static_cast<uint32_t>(__cvta_generic_to_shared(smem_raw));
    const uint32_t base = (raw_at + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - raw_at);
    float* ysum = reinterpret_cast<float*>(gbase + W::kYAt);                      // [token][row]
    const uint32_t bars = base + W::kBarsAt;
    auto rec_full = [&](uint32_t s) { return bars + 8 * s; };
    auto rec_free = [&](uint32_t s) { return bars + 16 + 8 * s; };
    auto op_full = [&](uint32_t s) { return bars + 32 + 8 * s; };
    auto op_done = [&](uint32_t s) { return bars + 48 + 8 * s; };
    auto acc_free = [&](uint32_t s) { return bars + 64 + 8 * s; };
    volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(gbase + W::kBarsAt + 128);
    volatile uint32_t* gone = tmem_ptr + 1;

    cg::cluster_group cluster = cg::this_cluster();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t lr = a.log_ranks, ranks = 1u << lr, rank = blockIdx.x & (ranks - 1);
    const uint32_t block = blockIdx.x >> lr;                                      // 128 rows = row blocks 2 block, 2 block + 1
    const uint32_t kts = (a.cols + 63) / 64, units = max((kts + 1) / 2, 1u);
    const uint32_t kbs = W::kBlockTiles == 2 ? units : kts;                       // records per row block
    const bool second = (2 * block + 1) * 64 < a.rows;                            // the second row block exists
    const uint64_t total = kts ? static_cast<uint64_t>(units) * a.n_seg : 0u;
    const uint32_t lo = static_cast<uint32_t>(total * rank >> lr), hi = static_cast<uint32_t>(total * (rank + 1) >> lr);

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < 2; ++s) {
            bar_init_n(rec_full(s), 1);
            bar_init_n(rec_free(s), kWorkers);
            bar_init_n(op_full(s), kWorkers);
            bar_init_n(op_done(s), 1);
        }
        for (uint32_t s = 0; s < kAccs; ++s) bar_init_n(acc_free(s), kWorkers);
        *gone = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kWorkers) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + W::kBarsAt + 128), "r"(W::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    for (uint32_t i = threadIdx.x; i < a.n_tokens * kTileRows; i += kThreads) ysum[i] = 0.f;
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_ptr;

    if (warp == kWorkers) {
        // ---- records
        if (lane == 0) {
            uint32_t seg = lo / units, unit = lo - seg * units, n_issued = 0;
            for (uint32_t u = lo; u < hi; ++u, ++n_issued) {
                const uint32_t s = n_issued % kRecStages;
                if (!wait_or_leave(rec_free(s), ((n_issued / kRecStages) & 1u) ^ 1u, gone)) break;
                const uint32_t kb = W::kBlockTiles == 2 ? unit : 2 * unit;
                const uint32_t bytes = min(2 / W::kBlockTiles, kbs - kb) * W::kRecord;
                const char* src = static_cast<const char*>(a.seg[seg].packed) + (static_cast<size_t>(2 * block) * kbs + kb) * W::kRecord;
                const uint32_t to = base + W::kRecAt + s * 2 * W::kUnitBytes;
                bar_expect(rec_full(s), second ? 2 * bytes : bytes);
                bulk_copy(to, src, bytes, rec_full(s));
                if (second) bulk_copy(to + W::kUnitBytes, src + static_cast<size_t>(kbs) * W::kRecord, bytes, rec_full(s));
                if (++unit == units) { unit = 0; ++seg; }
            }
            if (*gone)      // let what was issued land before the CTA's shared memory is released
                for (uint32_t k = n_issued > kRecStages ? n_issued - kRecStages : 0; k < n_issued; ++k)
                    (void)bar_wait(rec_full(k % kRecStages), (k / kRecStages) & 1u);
        }
    } else if (warp == kWorkers + 1) {
        // ---- products
        if (lane == 0) {
            uint32_t seg = lo / units, unit = lo - seg * units, it = 0, acc = 0;
            bool ok = true;
            for (uint32_t u = lo; u < hi && ok; ++u) {
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (((a.seg[seg].count + 15) / 16 * 16 >> 3) << 17) | ((kTileRows >> 4) << 24);
                const uint32_t nt = min(2u, kts - 2 * unit);
                for (uint32_t i = 0; i < nt && ok; ++i, ++it) {
                    const uint32_t s = it % kOpStages;
                    ok = wait_or_leave(op_full(s), (it / kOpStages) & 1u, gone);
                    if (!ok) break;
                    tc_after();
                    const uint32_t op = base + W::kOpsAt + s * W::kOpBytes;
                    const uint64_t da = operand_desc(op);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool fresh = k == 0 ? (GROUP != 128 || i == 0) : (W::HALF && k == 2);
                        if (fresh) {
                            ok = wait_or_leave(acc_free(acc % kAccs), ((acc / kAccs) & 1u) ^ 1u, gone);
                            if (!ok) break;
                            tc_after();
                            ++acc;
                        }
                        const uint32_t d = tmem + (acc - 1) % kAccs * NT;
#pragma unroll
                        for (uint32_t term = 0; term < W::kTerms; ++term)
                            tc_mma(d, da + 2 * k, operand_desc(op + kATile + term * W::kBTile) + 2 * k, idesc, !(fresh && term == 0));
                    }
                    tc_commit(op_done(s));
                }
                if (++unit == units) { unit = 0; ++seg; }
            }
            if (!ok) {      // what was issued ends before tensor memory is freed: one more commit on a barrier that nobody waits for now
                tc_commit(op_done(it % kOpStages));
                (void)bar_wait(op_done(it % kOpStages), (it / kOpStages) & 1u);
            }
        }
    } else {
        // ---- workers
        const int g = lane >> 2, t = lane & 3, tid = threadIdx.x;
        const uint32_t token = tid / kLanes, tl = tid % kLanes;
        const uint32_t quadrant = warp & 3, half = warp >> 2, trow = quadrant * 32 + lane;      // this thread's row and half of the tokens
        const uint32_t own_scale = (trow >> 6) * W::kUnitBytes + W::kCodeBytes + ((trow & 63) >> 4) * 32 + (trow & 7) * 4 + ((trow >> 3) & 1) * 2;
        const XT* x = static_cast<const XT*>(a.x);
        const uint32_t whole = a.x_vec ? a.cols / 64 : 0u;
        float tot[NT / 2];
        uint32_t seg = lo / units, unit = lo - seg * units, it = 0, acc = 0, n_rec = 0;
        bool ok = true, pending = false;
        float ps0 = 0.f, ps1 = 0.f;          // scale(s) of the group(s) that wait to be added up
        uint32_t p_it = 0;
        uint32_t count = 0;
        auto drain_one = [&](float scale) {
            const uint32_t b = acc % kAccs;
            const uint32_t at = tmem + (quadrant << 21) + b * NT + half * (NT / 2);
#pragma unroll
            for (int c = 0; c < NT / 2; c += 16) {
                if (half * (NT / 2) + c < count) {
                    uint32_t v[16];
                    tc_load16(at + c, v);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int j = 0; j < 16; ++j) tot[c + j] = __fmaf_rn(scale, __uint_as_float(v[j]), tot[c + j]);
                }
            }
            tc_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_free(b));
            ++acc;
        };
        auto drain = [&]() {
            if (!pending) return;
            pending = false;
            ok = wait_or_leave(op_done(p_it % kOpStages), (p_it / kOpStages) & 1u, gone);
            ok = __all_sync(~0u, ok);
            if (!ok) return;
            tc_after();
            drain_one(ps0);
            if (W::HALF) drain_one(ps1);
        };
        while (lo + n_rec < hi && ok) {
            // ---- one segment's part of the run
            const PackedSegment& sg = a.seg[seg];
            count = sg.count;
            const bool on = token < count, signs = sg.flip != 0;
            const uint32_t pos = sg.first + (on ? token : 0);
            const XT* xt = x + a.token[pos] * a.x_stride + tl * kCols;
            DevTask task = {0, 0, 0, 0};
            if (signs) task = a.task[a.token_task[pos]];
#pragma unroll
            for (int j = 0; j < NT / 2; ++j) tot[j] = 0.f;
            uint4 blk = make_uint4(0, 0, 0, 0);
            uint32_t blk0 = ~0u;
            typename Act::Raw raw[kChunks];
            auto load = [&](uint32_t kt) {
#pragma unroll
                for (uint32_t h = 0; h < kChunks; ++h) {
                    const uint32_t c = kt * 64 + tl * kCols + h * 8;
                    if (kt < whole) raw[h] = Act::words(xt + kt * 64 + h * 8);
                    else raw[h] = c < a.cols ? Act::gather(xt - tl * kCols, c, a.cols) : Act::zero();
                }
            };
            const uint32_t kt_end = min(kts, 2 * (unit + (hi - lo - n_rec)));
            load(2 * unit);
            for (; unit < units && lo + n_rec < hi && ok; ++unit, ++n_rec) {
                const uint32_t rs = n_rec % kRecStages, rec = base + W::kRecAt + rs * 2 * W::kUnitBytes;
                ok = __all_sync(~0u, wait_or_leave(rec_full(rs), (n_rec / kRecStages) & 1u, gone));
                const uint32_t nt = min(2u, kts - 2 * unit);
#pragma unroll 1
                for (uint32_t i = 0; i < nt && ok; ++i, ++it) {
                    const uint32_t kt = 2 * unit + i, os = it % kOpStages, op = base + W::kOpsAt + os * W::kOpBytes;
                    // the stage's products of two tiles ago have read it
                    if (it >= kOpStages) ok = __all_sync(~0u, wait_or_leave(op_done(os), ((it / kOpStages) & 1u) ^ 1u, gone));
                    if (!ok) break;
                    // A: 16 rows of codes. Lanes with odd g take the right half of the tile first, so that eight lanes' stores
                    // fall into different banks.
                    {
                        const uint32_t tile = rec + (warp >> 2) * W::kUnitBytes + (W::kBlockTiles == 2 ? i * 2048 : i * W::kRecord) + (warp & 3) * 512 + lane * 16;
                        const uint4 cw = lds128(tile);
                        const bool odd = g & 1;
                        const uint32_t w[4] = {odd ? cw.z : cw.x, odd ? cw.w : cw.y, odd ? cw.x : cw.z, odd ? cw.y : cw.w};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t q0[4], q1[4];
                            decode(w[2 * h], q0);
                            decode(w[2 * h + 1], q1);
                            const uint32_t chunk = ((h ^ (g & 1)) * 4 + t) ^ g;
                            const uint32_t to = op + (warp * 16 + g) * 128 + chunk * 16;
                            sts128(to, make_uint4(q0[0], q0[2], q1[0], q1[2]));
                            sts128(to + 8 * 128, make_uint4(q0[1], q0[3], q1[1], q1[3]));
                        }
                    }
                    // B: this thread's columns of its token
                    if (signs) {
                        if (blk0 == ~0u || (kt >> 1) - blk0 >= kLanes) {
                            blk0 = kt >> 1;      // lane tl of a token makes the block of columns 128 (blk0 + tl) ..
                            blk = philox4x32_10(blk0 + tl, sg.slot, kTagSign, task.id, task.key0, task.key1);
                        }
                        const int src = static_cast<int>((lane & ~(kLanes - 1)) | ((kt >> 1) - blk0));
                        const uint32_t w0 = __shfl_sync(~0u, kt & 1 ? blk.z : blk.x, src), w1 = __shfl_sync(~0u, kt & 1 ? blk.w : blk.y, src);
                        const uint32_t bits = (tl * kCols >= 32 ? w1 : w0) >> (tl * kCols & 31);
#pragma unroll
                        for (uint32_t h = 0; h < kChunks; ++h) {
                            uint32_t wt[Act::kTerms][4];
                            Act::terms(raw[h], wt);
                            const uint32_t byte = (bits >> (8 * h)) & 0xFFu, chunk = (tl * kChunks + h) ^ (token & 7);
#pragma unroll
                            for (int k = 0; k < Act::kTerms; ++k) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) wt[k][e] ^= (byte * ((1u << (15 - 2 * e)) + (1u << (30 - 2 * e)))) & 0x80008000u;
                                if (on) sts128(op + kATile + k * W::kBTile + token * 128 + chunk * 16, make_uint4(wt[k][0], wt[k][1], wt[k][2], wt[k][3]));
                            }
                        }
                    } else {
#pragma unroll
                        for (uint32_t h = 0; h < kChunks; ++h) {
                            uint32_t wt[Act::kTerms][4];
                            Act::terms(raw[h], wt);
                            const uint32_t chunk = (tl * kChunks + h) ^ (token & 7);
#pragma unroll
                            for (int k = 0; k < Act::kTerms; ++k)
                                if (on) sts128(op + kATile + k * W::kBTile + token * 128 + chunk * 16, make_uint4(wt[k][0], wt[k][1], wt[k][2], wt[k][3]));
                        }
                    }
                    if (kt + 1 < kt_end) load(kt + 1);
                    const uint32_t sat = rec + own_scale + (W::kBlockTiles == 1 ? i * W::kRecord : 0u);
                    const float s0 = __uint_as_float(lds_u16(sat) << 16);
                    const float s1 = W::HALF ? __uint_as_float(lds_u16(sat + 128) << 16) : 0.f;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the tensor core reads through the async proxy
                    __syncwarp();
                    if (lane == 0) {
                        bar_arrive(op_full(os));
                        if (i + 1 == nt) bar_arrive(rec_free(rs));
                    }
                    drain();                      // the tile before
                    if (GROUP != 128 || i + 1 == nt) {
                        pending = true;
                        p_it = it;
                        ps0 = s0;
                        ps1 = s1;
                    }
                }
            }
            if (ok) drain();
            if (!ok) break;
            // this segment's sums: at most two (base and slot) meet in an element, so their order does not matter
            const float factor = seg ? kCodeUnit * a.lambda : kCodeUnit;
#pragma unroll
            for (uint32_t j = 0; j < NT / 2; ++j) {
                const uint32_t i = half * (NT / 2) + j;
                if (i < count) atomicAdd(ysum + a.token[sg.first + i] * kTileRows + trow, factor * tot[j]);
            }
            unit = 0;
            ++seg;
        }
    }
    tc_before();
    __syncthreads();
    if (warp == kWorkers) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(W::kTmem) : "memory");
    }
    if (*gone) {
        for (uint32_t i = threadIdx.x; i < a.n_tokens * kTileRows; i += kThreads) ysum[i] = NAN;
        __syncthreads();
    }
    auto store = [&](uint32_t o, float y) {
        const uint64_t row = static_cast<uint64_t>(block) * kTileRows + o % kTileRows;
        if (row >= a.rows) return;
        const size_t at = o / kTileRows * a.y_stride + row;
        if (a.y_bf16) static_cast<bf16*>(a.y)[at] = __float2bfloat16_rn(y);
        else static_cast<float*>(a.y)[at] = y;
    };
    const uint32_t n_out = a.n_tokens * kTileRows;
    if (ranks == 1) {
        for (uint32_t o = threadIdx.x; o < n_out; o += kThreads) store(o, ysum[o]);
    } else {
        cluster.sync();
        for (uint32_t o = rank * kThreads + threadIdx.x; o < n_out; o += ranks * kThreads) {
            float y = 0.f;
            for (uint32_t k = 0; k < ranks; ++k) y += cluster.map_shared_rank(ysum, k)[o];
            store(o, y);
        }
        cluster.sync();          // nobody leaves while its sums may still be read
    }
}

constexpr int kDevices = 64;

template <int NT, typename XT, int GROUP> cudaError_t launch_wide(PackedLinearArgs<kWideTokens>& a, int sm_count, int device, cudaStream_t s)
{
    typedef Wide<NT, XT, GROUP> W;
    const uint64_t blocks = (static_cast<uint64_t>(a.rows) + kTileRows - 1) / kTileRows;
    const uint64_t units = ((a.cols + 63ull) / 64 + 1) / 2 * a.n_seg;
    // two CTAs per SM, as long as each has a few units to itself
    a.log_ranks = 0;
    while (a.log_ranks < 3 && (blocks << (a.log_ranks + 1)) <= static_cast<uint64_t>(sm_count) * 2 && (4ull << a.log_ranks) <= units) ++a.log_ranks;
    const uint32_t ranks = 1u << a.log_ranks;
    const size_t smem = W::smem(a.n_tokens);
    static std::atomic<size_t> granted[kDevices];      // a kernel has to opt in beyond 48 KiB, per device
    if (device >= kDevices || smem > granted[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(packed_wide_kernel<NT, XT, GROUP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(W::smem(NT)));
        if (e != cudaSuccess) return e;
        if (device < kDevices) granted[device].store(W::smem(NT), std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = ranks > 1;
    return cudaLaunchKernelEx(&cfg, packed_wide_kernel<NT, XT, GROUP>, a);
}

template <int NT, typename XT> cudaError_t launch_group(PackedLinearArgs<kWideTokens>& a, int sm_count, int device, cudaStream_t s)
{
    if (a.group == 32) return launch_wide<NT, XT, 32>(a, sm_count, device, s);
    if (a.group == 64) return launch_wide<NT, XT, 64>(a, sm_count, device, s);
    return launch_wide<NT, XT, 128>(a, sm_count, device, s);
}

}  // namespace

int launch_packed_wide(PackedLinearArgs<kWideTokens>& a, bool x_bf16, int sm_count, int device, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.n_tokens <= 32) return static_cast<int>(x_bf16 ? launch_group<32, bf16>(a, sm_count, device, s) : launch_group<32, float>(a, sm_count, device, s));
    return static_cast<int>(x_bf16 ? launch_group<64, bf16>(a, sm_count, device, s) : launch_group<64, float>(a, sm_count, device, s));
}

int packed_wide_giveups(unsigned int* count)
{
    return static_cast<int>(cudaMemcpyFromSymbol(count, g_wide_giveups, sizeof(unsigned int)));
}

}  // namespace randes
