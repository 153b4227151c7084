// Products of more than a few tokens (up to 64 a launch), and of few fp32 tokens on large matrices, with packed weights, on the
// fifth-generation tensor cores.
//
// The scale of a weight belongs to a row and a group of columns, so the tensor core can only add up within a group: codes
// (q / 64, exact in bf16) x activations over the columns of one group, in tensor memory; the group's sums then come back
// to registers and are added to the row's totals with the group's scale, one fp32 multiply-add each. A CTA works on 128
// rows and a contiguous run of column blocks over all segments (see randes_packed.cu for segments); the CTAs of a cluster
// share the rows and meet through distributed shared memory.
//
// The activations are the same for every block of rows, so a first kernel lays them out once as operand B in the caller's
// workspace (signs applied; an fp32 activation as three bf16 terms), one tile of 64 columns after the other, swizzled as
// the tensor core wants them. The product kernel has one CTA per SM, whose warps keep to one task each:
//   warps 0-7    group sums: a thread owns one row and half the tokens
//   warps 8-15   operand A: codes to bf16, 16 rows each, straight into tensor memory (by way of shared memory: a fifth slower)
//   warp 16      copies records (one lane, bulk copies), owns tensor memory
//   warp 17      issues tcgen05.mma (one lane): M = 128 rows, N = tokens of the segment rounded up to 16
//   warp 18      copies operand B (one lane, bulk copies)
// The order of the columns in a product step is the one in which the lanes hold the codes (operand B is laid out alike), so
// that a decoded word is four registers of operand A as they are. A hand-over between roles costs hundreds of cycles however
// little it hands over: stages are 128 or 256 columns, and what is passed on also frees what came before.
//
// What bounds it: about 8 to 10 us that do not depend on the columns (two launches, set-up, first hand-overs, the join), then the
// chain of hand-overs. In groups of 128 a stage of 256 columns costs 0.60 us with 16 bf16 tokens and 0.64 with 64 (from 16384 to
// 32768 columns at 16384 rows: 46.4 -> 85.0 and 51.2 -> 92.5 us, 3.4 TB/s of packed weights), and no unit is full at 64 tokens
// (issue 0.60 of the slots, waiting warps' questions included; tensor pipe 0.33, HBM 0.27): operand A has two stages, and
// each goes record, decode, tensor memory, products, free again. 64 fp32 tokens pay for their three products, 1.4 us per 256
// columns (16384 x 16384: 99.7 us). Smaller groups hand over more sums: 64 tokens 73 us in groups of 64, 118 in groups of 32.
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

constexpr int kSumWarps = 8, kAWarps = 8;
constexpr int kAFirst = kSumWarps, kCopyWarp = kAFirst + kAWarps, kMmaWarp = kCopyWarp + 1, kCopyBWarp = kMmaWarp + 1;
constexpr int kThreads = (kCopyBWarp + 1) * 32;
constexpr uint32_t kTileRows = 128;

// ---- mbarriers with any count, bounded waits that also end when the CTA has given up: of one lane, and of a whole warp (every
// lane asks and the warp votes, so that no branch diverges: 20 cycles where nothing has to be waited for, a loop per lane takes 80)
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

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gone)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (__all_sync(~0u, bar_try(bar, parity))) return true;
        if ((i & 63u) == 63u && __any_sync(~0u, *gone != 0)) return false;
    }
    if ((threadIdx.x & 31) == 0 && atomicExch(const_cast<uint32_t*>(gone), 1u) == 0u) atomicAdd(&g_wide_giveups, 1u);
    __syncwarp();
    return false;
}

// ---- tcgen05
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)      // A in tensor memory
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_load16(uint32_t addr, uint32_t* v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr) : "memory");
}
// 16 rows x 32 words: lane 4 g + t holds words 4 i + t of rows g (v[2 i]) and g + 8 (v[2 i + 1])
__device__ __forceinline__ void tc_store16x32(uint32_t addr, const uint32_t* v)
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
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
    // Column tiles per stage: as many as shared memory allows with a second stage behind it, since what a warp does per stage
    // besides its work costs as much as the work (64 tokens, 16384 x 16384: 53 us, 73 with half of that)
    static constexpr uint32_t kTiles = kTerms == 3 && NT == 64 ? 2 : 4;
    static constexpr uint32_t kUnitBytes = kTiles / kBlockTiles * kRecord;  // 64 rows
    static constexpr uint32_t kBTile = NT * 128;
    // Stages: operand A (half of tensor memory), operand B and records (as shared memory allows). What they hide is one
    // hand-over for A, an L2 latency for B, an HBM latency for the records.
    static constexpr uint32_t kAWords = kTiles * 32, kBBytes = kTiles * kTerms * kBTile;
    static constexpr uint32_t kAStages = 256 / kAWords, kBStages = kTerms == 3 ? (NT == 64 ? 3 : 2) : 3;
    static constexpr uint32_t kRecStages = kTiles == 2 ? 5 : 4;
    // The sums of a stage's groups go over to the other warps together -- in batches where they take more than 128 columns
    // of tensor memory --, and the hand-over also says that operands A and B of what came before are free.
    static constexpr uint32_t kGroups = kTiles * 64 / GROUP, kBatches = kGroups * NT > 128 ? kGroups * NT / 128 : 1, kPer = kGroups / kBatches;
    static constexpr uint32_t kRing = 256 / (kPer * NT);                    // batches of sums in tensor memory
    static constexpr uint32_t kDone = 16;                                   // barriers that batches complete in turn
    static_assert(kDone >= kBatches * kBStages && kDone >= kBatches * kAStages && kDone >= kBatches * kRecStages && kDone >= kRing, "nobody may miss a whole turn");
    static constexpr uint32_t kBAt = 0, kRecAt = kBStages * kBBytes;        // 1024-byte aligned operand first
    static constexpr uint32_t kBarsAt = kRecAt + kRecStages * 2 * kUnitBytes;
    static constexpr uint32_t kYAt = kBarsAt + 512;
    static_assert(kYAt + NT * kTileRows * 4 + 1024 <= 227 * 1024, "shared memory of a CTA");
    static constexpr uint32_t kTmem = 512, kTmemA = 256;                    // sums, operand A
    static size_t smem(uint32_t n_tokens) { return 1024 + kYAt + static_cast<size_t>(n_tokens) * kTileRows * sizeof(float); }
};

// Rows of operand B that a segment with that many tokens takes up: whole groups of eight, the swizzle's period. (Rows that
// no token fills are whatever was there: their columns of the product go nowhere.)
__host__ __device__ constexpr uint32_t operand_rows(uint32_t count) { return (count + 7) / 8 * 8; }

// One thread per position of the token lists and eight columns.
template <typename XT>
__global__ void __launch_bounds__(256) operand_kernel(const __grid_constant__ PackedLinearArgs<kWideTokens> a)
{
    typedef Acts<XT> Act;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the product kernel sets itself up meanwhile
    const uint32_t kts = (a.cols + 63) / 64, chunk = blockIdx.x * 256 + threadIdx.x, pos = blockIdx.y;
    if (chunk >= kts * 8) return;
    uint32_t seg = 0;
    while (pos >= a.seg[seg].first + a.seg[seg].count) ++seg;
    const uint32_t row = pos - a.seg[seg].first, rows = operand_rows(a.seg[seg].count), c = chunk * 8;
    const XT* x = static_cast<const XT*>(a.x) + a.token[pos] * a.x_stride;
    typename Act::Raw raw;
    if (a.x_vec && c + 8 <= a.cols) raw = Act::words(x + c);
    else raw = c < a.cols ? Act::gather(x, c, a.cols) : Act::zero();
    uint32_t w[Act::kTerms][4];
    Act::terms(raw, w);
    if (a.seg[seg].flip) {
        const DevTask task = a.task[a.token_task[pos]];
        const uint4 blk = philox4x32_10(c >> 7, a.seg[seg].slot, kTagSign, task.id, task.key0, task.key1);
        const uint32_t q = (c >> 5) & 3u, word = q == 0 ? blk.x : (q == 1 ? blk.y : (q == 2 ? blk.z : blk.w)), byte = (word >> (c & 31)) & 0xFFu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t mask = (byte * ((1u << (15 - 2 * e)) + (1u << (30 - 2 * e)))) & 0x80008000u;
#pragma unroll
            for (int k = 0; k < Act::kTerms; ++k) w[k][e] ^= mask;
        }
    }
    // pair e of this lane's eight columns (t of the tile's half h) goes where operand A has it: word t of 16-byte chunk 4 h + e
    char* to = static_cast<char*>(a.operands) + a.operand_at[seg] * (static_cast<size_t>(kts) * 128 * Act::kTerms) +
               static_cast<size_t>(chunk >> 3) * rows * 128 * Act::kTerms + row * 128 + (chunk & 3) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t at = (((chunk & 4) + e) ^ (row & 7)) * 16;
#pragma unroll
        for (int k = 0; k < Act::kTerms; ++k) *reinterpret_cast<uint32_t*>(to + static_cast<size_t>(k) * rows * 128 + at) = w[k][e];
    }
}

template <int NT, typename XT, int GROUP>
__global__ void __launch_bounds__(kThreads, 1) packed_wide_kernel(const __grid_constant__ PackedLinearArgs<kWideTokens> a)
{
    typedef Wide<NT, XT, GROUP> W;
    constexpr uint32_t kAStages = W::kAStages, kBStages = W::kBStages, kRecStages = W::kRecStages, kRing = W::kRing;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw_at = static_cast<uint32_t>(__cvta_generic_to_shared(smem_raw));
    const uint32_t base = (raw_at + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - raw_at);
    float* ysum = reinterpret_cast<float*>(gbase + W::kYAt);                      // [token][row]
    const uint32_t bars = base + W::kBarsAt;
    auto rec_full = [&](uint32_t s) { return bars + 8 * s; };
    auto b_full = [&](uint32_t s) { return bars + 64 + 8 * s; };
    auto a_full = [&](uint32_t s) { return bars + 128 + 8 * s; };
    auto done = [&](uint32_t n) { return bars + 160 + 8 * (n % W::kDone); };      // batch n of sums is in tensor memory
    auto summed = [&](uint32_t n) { return bars + 288 + 8 * (n % W::kDone); };    // and has been read
    const uint32_t flushed = bars + 416, drained = bars + 424;
    volatile uint32_t* tmem_ptr = reinterpret_cast<volatile uint32_t*>(gbase + W::kBarsAt + 432);
    volatile uint32_t* gone = tmem_ptr + 1;
    auto last_batch = [&](uint32_t i) { return i * W::kBatches + W::kBatches - 1; };      // of the CTA's i-th stage

    cg::cluster_group cluster = cg::this_cluster();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t lr = a.log_ranks, ranks = 1u << lr, rank = blockIdx.x & (ranks - 1);
    const uint32_t block = blockIdx.x >> lr;                                      // 128 rows = row blocks 2 block, 2 block + 1
    const uint32_t kts = (a.cols + 63) / 64, units = max((kts + W::kTiles - 1) / W::kTiles, 1u);
    const uint32_t kbs = (kts + W::kBlockTiles - 1) / W::kBlockTiles;                       // records per row block
    const bool second = (2 * block + 1) * 64 < a.rows;                            // the second row block exists
    const uint64_t total = kts ? static_cast<uint64_t>(units) * a.n_seg : 0u;
    const uint32_t lo = static_cast<uint32_t>(total * rank >> lr), hi = static_cast<uint32_t>(total * (rank + 1) >> lr);

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kRecStages; ++s) bar_init_n(rec_full(s), 1);
        for (uint32_t s = 0; s < kBStages; ++s) bar_init_n(b_full(s), 1);
        for (uint32_t s = 0; s < kAStages; ++s) bar_init_n(a_full(s), kAWarps);
        for (uint32_t s = 0; s < W::kDone; ++s) {
            bar_init_n(done(s), 1);
            bar_init_n(summed(s), kSumWarps);
        }
        bar_init_n(drained, 1);
        bar_init_n(flushed, kSumWarps);
        *gone = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kCopyWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + W::kBarsAt + 432), "r"(W::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    for (uint32_t i = threadIdx.x; i < a.n_tokens * kTileRows; i += kThreads) ysum[i] = 0.f;
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *tmem_ptr;

    if (warp == kCopyWarp) {
        // ---- records
        if (lane == 0) {
            uint32_t seg = lo / units, unit = lo - seg * units, n_issued = 0;
            for (uint32_t u = lo; u < hi; ++u, ++n_issued) {
                const uint32_t s = n_issued % kRecStages;
                if (n_issued >= kRecStages) {      // whose codes went into products that have been read, and whose scales with them
                    const uint32_t n = last_batch(n_issued - kRecStages);
                    if (!wait_or_leave(summed(n), (n / W::kDone) & 1u, gone)) break;
                }
                const uint32_t kb = unit * (W::kTiles / W::kBlockTiles);
                const uint32_t bytes = min(W::kTiles / W::kBlockTiles, kbs - kb) * W::kRecord;
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
    } else if (warp == kCopyBWarp) {
        // ---- operand B
        if (lane == 0) {
            asm volatile("griddepcontrol.wait;" ::: "memory");       // for the kernel that lays it out
            uint32_t seg = lo / units, unit = lo - seg * units, n_issued = 0;
            for (uint32_t u = lo; u < hi; ++u, ++n_issued) {
                const uint32_t s = n_issued % kBStages, bytes = operand_rows(a.seg[seg].count) * 128 * W::kTerms, all = min(W::kTiles, kts - W::kTiles * unit) * bytes;
                if (n_issued >= kBStages) {
                    const uint32_t n = last_batch(n_issued - kBStages);
                    if (!wait_or_leave(done(n), (n / W::kDone) & 1u, gone)) break;
                }
                bar_expect(b_full(s), all);
                bulk_copy(base + W::kBAt + s * W::kBBytes,
                          static_cast<const char*>(a.operands) + a.operand_at[seg] * (static_cast<size_t>(kts) * 128 * W::kTerms) +
                              static_cast<size_t>(W::kTiles * unit) * bytes, all, b_full(s));
                if (++unit == units) { unit = 0; ++seg; }
            }
            if (*gone)      // let what was issued land
                for (uint32_t k = n_issued > kBStages ? n_issued - kBStages : 0; k < n_issued; ++k)
                    (void)bar_wait(b_full(k % kBStages), (k / kBStages) & 1u);
        }
    } else if (warp == kMmaWarp) {
        // ---- products. The whole warp walks the loop, so that descriptors stay in uniform registers; one lane issues.
        uint32_t seg = lo / units, unit = lo - seg * units, sa = 0, a_parity = 0, sb = 0, b_parity = 0, batch = 0, slot = 0;
        const bool leader = elect_one();
        const uint64_t desc_b = operand_desc(base + W::kBAt);
        bool ok = true;
        for (uint32_t u = lo; u < hi; ++u) {
            const uint32_t rows = operand_rows(a.seg[seg].count), nt = min(W::kTiles, kts - W::kTiles * unit), term = rows * 128 / 16;
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((rows + 8) / 16 << 18) | ((kTileRows >> 4) << 24);     // N = rows rounded up to 16
            ok = warp_wait(b_full(sb), b_parity, gone) && warp_wait(a_full(sa), a_parity, gone);
            if (!ok) break;
            const uint32_t at_a = tmem + W::kTmemA + sa * W::kAWords;
            const uint64_t db = desc_b + sb * (W::kBBytes / 16);
            constexpr uint32_t kSteps = GROUP / 16;       // product steps of 16 columns per group
#pragma unroll
            for (uint32_t b = 0; b < W::kBatches; ++b) {
                if (batch >= kRing) ok = warp_wait(summed(batch - kRing), ((batch - kRing) / W::kDone) & 1u, gone);
                if (!ok) break;
                tc_after();
                if (leader) {
#pragma unroll
                    for (uint32_t k = b * W::kPer * kSteps; k < (b + 1) * W::kPer * kSteps; ++k)
                        if (k / 4 < nt) {
                            const uint32_t d = tmem + (slot * W::kPer + (k / kSteps) % W::kPer) * NT;
#pragma unroll
                            for (uint32_t h = 0; h < W::kTerms; ++h)
                                tc_mma(d, at_a + 8 * k, db + (k / 4) * W::kTerms * term + h * term + 2 * (k % 4), idesc, !(k % kSteps == 0 && h == 0));
                        }
                    tc_commit(done(batch));
                }
                ++batch;
                if (++slot == kRing) slot = 0;
            }
            if (!ok) break;
            if (++sa == kAStages) { sa = 0; a_parity ^= 1u; }
            if (++sb == kBStages) { sb = 0; b_parity ^= 1u; }
            if (++unit == units) { unit = 0; ++seg; }
            __syncwarp();
        }
        if (!ok && leader) {    // what was issued ends before tensor memory is freed
            tc_commit(drained);
            (void)bar_wait(drained, 0u);
        }
        __syncwarp();
    } else if (warp >= kAFirst) {
        // ---- operand A: one row tile. A warp reaches the quarter of tensor memory that its number modulo four names.
        const uint32_t tile = (warp & 3) * 2 + ((warp >> 2) & 1);
        const uint32_t from = base + W::kRecAt + (tile >> 2) * W::kUnitBytes + (tile & 3) * 512 + lane * 16;
        const uint32_t to = tmem + W::kTmemA + (tile << 20);
        uint32_t unit = lo % units, rs = 0, rec_parity = 0, sa = 0;
        for (uint32_t u = lo; u < hi; ++u) {
            if (!warp_wait(rec_full(rs), rec_parity, gone)) break;
            const uint32_t rec = from + rs * 2 * W::kUnitBytes;
            const uint32_t nt = min(W::kTiles, kts - W::kTiles * unit);
            uint4 c[W::kTiles];
#pragma unroll
            for (uint32_t i = 0; i < W::kTiles; ++i)       // (a tile that does not exist: not used)
                c[i] = lds128(rec + i / W::kBlockTiles * W::kRecord + i % W::kBlockTiles * 2048);
            if (u - lo >= kAStages) {        // the products have read the stage
                const uint32_t n = last_batch(u - lo - kAStages);
                if (!warp_wait(done(n), (n / W::kDone) & 1u, gone)) break;
                tc_after();
            }
            __syncwarp();
#pragma unroll
            for (uint32_t i = 0; i < W::kTiles; ++i) {
                if (i >= nt) break;
                uint32_t q[4][4];          // word j: operand registers, the 16 columns of product step 4 i + j
                decode(c[i].x, q[0]);
                decode(c[i].y, q[1]);
                decode(c[i].z, q[2]);
                decode(c[i].w, q[3]);
                tc_store16x32(to + sa * W::kAWords + 32 * i, &q[0][0]);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            tc_before();
            __syncwarp();
            if (lane == 0) bar_arrive(a_full(sa));
            if (++rs == kRecStages) { rs = 0; rec_parity ^= 1u; }
            if (++sa == kAStages) sa = 0;
            if (++unit == units) unit = 0;
        }
    } else {
        // ---- group sums
        const uint32_t quadrant = warp & 3, half = warp >> 2, trow = quadrant * 32 + lane;      // this thread's row and half of the tokens
        const uint32_t own_scale = (trow >> 6) * W::kUnitBytes + W::kCodeBytes + ((trow & 63) >> 4) * 32 + (trow & 7) * 4 + ((trow >> 3) & 1) * 2;
        uint32_t seg = lo / units, unit = lo - seg * units, batch = 0, n_rec = 0, n_flush = 0;
        bool ok = true;
        for (uint32_t u = lo; u < hi && ok; unit = 0, ++seg) {
            const PackedSegment& sg = a.seg[seg];
            const uint32_t count = sg.count;
            f32x2 tot[NT / 4];             // two tokens each
#pragma unroll
            for (int j = 0; j < NT / 4; ++j) tot[j] = 0;
            for (; unit < units && u < hi && ok; ++unit, ++u, ++n_rec) {
                const uint32_t rs = n_rec % kRecStages, sat = base + W::kRecAt + rs * 2 * W::kUnitBytes + own_scale;
                ok = warp_wait(rec_full(rs), (n_rec / kRecStages) & 1u, gone);
                if (!ok) break;
                const uint32_t nt = min(W::kTiles, kts - W::kTiles * unit);
                float scale[W::kGroups];
#pragma unroll
                for (int k = 0; k < static_cast<int>(W::kGroups); ++k)      // (a tile that does not exist: never used)
                    scale[k] = __uint_as_float(lds_u16(sat + (W::HALF ? (k >> 1) * W::kRecord + (k & 1) * 128 : k * W::kRecord)) << 16);
#pragma unroll
                for (uint32_t b = 0; b < W::kBatches; ++b, ++batch) {
                    ok = warp_wait(done(batch), (batch / W::kDone) & 1u, gone);
                    if (!ok) break;
                    tc_after();
                    __syncwarp();
                    const uint32_t slot = batch % kRing;
#pragma unroll
                    for (uint32_t k = b * W::kPer; k < (b + 1) * W::kPer; ++k) {
                        if (k * GROUP / 64 >= nt) break;
                        const uint32_t at = tmem + (quadrant << 21) + (slot * W::kPer + k % W::kPer) * NT + half * (NT / 2);
                        const f32x2 scale2 = pack2(__float_as_uint(scale[k]), __float_as_uint(scale[k]));
                        uint32_t v[NT / 2];
#pragma unroll
                        for (int c = 0; c < NT / 2; c += 16)
                            if (half * (NT / 2) + c < count) tc_load16(at + c, v + c);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int c = 0; c < NT / 2; c += 16)
                            if (half * (NT / 2) + c < count) {
#pragma unroll
                                for (int j = 0; j < 16; j += 2) tot[(c + j) / 2] = fma2(pack2(v[c + j], v[c + j + 1]), scale2, tot[(c + j) / 2]);
                            }
                    }
                    tc_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(summed(batch));
                }
            }
            if (!ok) break;
            // This segment's sums join the others' (an element gets one from the base and one from its token's slot, perhaps
            // from another warp): one segment after the other.
            if (n_flush && !warp_wait(flushed, (n_flush & 1u) ^ 1u, gone)) break;
            ++n_flush;
            const float factor = seg ? kCodeUnit * a.lambda : kCodeUnit;
#pragma unroll
            for (uint32_t j = 0; j < NT / 2; ++j) {
                const uint32_t i = half * (NT / 2) + j;
                float even, odd;
                unpack2(tot[j / 2], even, odd);
                if (i < count) ysum[a.token[sg.first + i] * kTileRows + trow] += factor * (j & 1 ? odd : even);
            }
            __syncwarp();
            if (lane == 0) bar_arrive(flushed);
        }
    }
    tc_before();
    __syncthreads();
    if (warp == kCopyWarp) {
        __syncwarp();            // the copies were one lane's; what follows is the whole warp's
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

template <int NT, typename XT, int GROUP> cudaError_t launch_wide(PackedLinearArgs<kWideTokens>& a, int sm_count, int device, int* launched, cudaStream_t s)
{
    typedef Wide<NT, XT, GROUP> W;
    const uint64_t blocks = (static_cast<uint64_t>(a.rows) + kTileRows - 1) / kTileRows;
    const uint64_t tiles = (a.cols + 63ull) / 64 * a.n_seg;
    // One CTA per SM, as long as each has a few units to itself. Clusters of four: not all those of eight that 128 CTAs make
    // fit the processor clusters at once (2000 x 2000, 24 tokens: 17.4 us against 11.8 us).
    a.log_ranks = 0;
    while (a.log_ranks < 2 && (blocks << (a.log_ranks + 1)) <= static_cast<uint64_t>(sm_count) && (8ull << a.log_ranks) <= tiles) ++a.log_ranks;
    const uint32_t ranks = 1u << a.log_ranks;
    const size_t smem = W::smem(a.n_tokens);
    static std::atomic<size_t> granted[kDevices];      // a kernel has to opt in beyond 48 KiB, per device
    if (device >= kDevices || smem > granted[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(packed_wide_kernel<NT, XT, GROUP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(W::smem(NT)));
        if (e != cudaSuccess) return e;
        if (device < kDevices) granted[device].store(W::smem(NT), std::memory_order_relaxed);
    }
    uint32_t rows = 0;
    for (uint32_t k = 0; k < a.n_seg; ++k) {
        a.operand_at[k] = static_cast<uint16_t>(rows);
        rows += operand_rows(a.seg[k].count);
    }
    const uint32_t kts = (a.cols + 63) / 64;
    static std::atomic<int> same_split[kDevices];
    if (kts) {
        if (device >= kDevices || !same_split[device].exchange(1, std::memory_order_relaxed)) {
            // the same division of L1 and shared memory as the kernel that follows: changing it costs microseconds
            const cudaError_t e = cudaFuncSetAttribute(operand_kernel<XT>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
            if (e != cudaSuccess) return e;
        }
        operand_kernel<XT><<<dim3((kts * 8 + 255) / 256, a.seg[a.n_seg - 1].first + a.seg[a.n_seg - 1].count), 256, 0, s>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        ++*launched;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    // The kernel may start while the one that lays out operand B (launched the ordinary way, behind everything before it) runs
    at[ranks > 1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[ranks > 1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = (ranks > 1) + (kts > 0);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, packed_wide_kernel<NT, XT, GROUP>, a);
    if (e == cudaSuccess) ++*launched;
    return e;
}

template <int NT, typename XT> cudaError_t launch_group(PackedLinearArgs<kWideTokens>& a, int sm_count, int device, int* launched, cudaStream_t s)
{
    if (a.group == 32) return launch_wide<NT, XT, 32>(a, sm_count, device, launched, s);
    if (a.group == 64) return launch_wide<NT, XT, 64>(a, sm_count, device, launched, s);
    return launch_wide<NT, XT, 128>(a, sm_count, device, launched, s);
}

}  // namespace

// The other form takes 8 tokens a launch and needs no second kernel, which small matrices notice most: 8 bf16 tokens on
// 2000 x 2000 take 4.9 us against 8.3, on 16384 x 8192 20 against 26. Two launches of it are slower nearly everywhere (16
// tokens: 9.6 against 8.9 and 38 against 27 us). fp32 tokens cost it three products and the splitting of the activations for
// every row block: it loses them where the matrix is large (one token, 16384 x 8192: 35 us against 29; with a superposition
// 67 against 52; 4096 x 4096: 7.6 against 8.9 and 13.0 against 12.1), unless the rows are short, so that a CTA of this form has little to
// do once it has set itself up (50257 x 768: 14.4 against 17.7; with a superposition, so with twice the columns, 28.7 against 27.9).
// Nothing was measured between 2^24 and 2^25 codes; and a superposition counts as one slot, however many the tokens use (the
// workspace is asked for before their tasks are known).
bool packed_is_wide(uint32_t rows, uint32_t cols, bool x_bf16, uint32_t n_tokens, bool tasks)
{
    const uint64_t columns = static_cast<uint64_t>(cols) << tasks;       // base, and one slot of the superposition
    return n_tokens > kNarrowTokens || (!x_bf16 && n_tokens && columns >= 1536 && rows * columns >= (1u << 25));
}

size_t packed_wide_workspace(uint32_t rows, uint32_t cols, bool x_bf16, uint32_t n_tokens, bool tasks)
{
    const uint32_t n = n_tokens < kWideTokens ? n_tokens : kWideTokens;
    if (!packed_is_wide(rows, cols, x_bf16, n_tokens, tasks)) return 0;
    // the base with every token; at worst every token has a slot of its own
    const size_t lines = operand_rows(n) + (tasks ? 8u * n : 0u);
    return lines * ((static_cast<size_t>(cols) + 63) / 64) * 128 * (x_bf16 ? 1 : 3);
}

int launch_packed_wide(PackedLinearArgs<kWideTokens>& a, bool x_bf16, int sm_count, int device, int* launched, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.n_tokens <= 32) return static_cast<int>(x_bf16 ? launch_group<32, bf16>(a, sm_count, device, launched, s) : launch_group<32, float>(a, sm_count, device, launched, s));
    return static_cast<int>(x_bf16 ? launch_group<64, bf16>(a, sm_count, device, launched, s) : launch_group<64, float>(a, sm_count, device, launched, s));
}

int packed_wide_giveups(unsigned int* count)
{
    return static_cast<int>(cudaMemcpyFromSymbol(count, g_wide_giveups, sizeof(unsigned int)));
}

}  // namespace randes
