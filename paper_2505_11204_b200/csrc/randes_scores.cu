// Log probabilities of given tokens, entropy and the top alternatives out of logits, in one pass; and their gradient.
//
// With u = scale * z (scale = one over the temperature), M = max z, d = z - M, S = sum exp(scale d), T = sum exp(scale d) d:
//     log p_j = scale * d_j - ln S        H = -sum p log p = ln S - scale * T / S
//     dz_j = scale * ( g_lp (1[j = target] - p_j) - g_H p_j (log p_j + H) )
// Everything is kept in powers of two: with c = scale log2 e an element counts 2^a, a = (z - m) c, m the greatest logit a thread
// has read. The difference is taken before anything is scaled, so no term carries the rounding of a large exponent, and a row
// that is sure of one token gets log probability 0 (one multiply-add z c - m c in place of the two steps would not give
// that). Each thread keeps (m, S = sum 2^a, T = sum 2^a a) and rescales S and T when its maximum rises.
//
// Top alternatives without sorting: four threads know the greatest of the elements they read; the k-th largest of those 64
// maxima cannot be above the k-th largest element. What reaches it is ranked, and to find that almost nothing is read again:
// a thread remembers which batch of loads held its maximum and the greatest of its other batches, so a thread whose maximum
// reaches the threshold (about k of 256) reads one batch again, or everything if a second batch reaches it too. Equal
// logits are ordered by index.
//
// A row may be shared by a cluster of CTAs (few rows); their sums and top lists meet in the first CTA through distributed
// shared memory.
//
// What bounds it: fp32 logits HBM (512 x 50257: 18 us, 5.7 TB/s); bf16 logits the special-function unit -- one exponential per
// two bytes, 25 us of it for 2048 x 50257 --, and between the last load of a row and its results some 5000 cycles in which
// the other rows of the SM go on (4096 x 32128: 52 us, 5.0 TB/s; with 20 alternatives 68 us). Fetching the next rows
// into L2 meanwhile gains nothing.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cooperative_groups.h>

#include <cfloat>

#include "randes_device.cuh"
#include "randes_internal.h"

namespace cg = cooperative_groups;

namespace randes {
namespace {

using namespace device;

constexpr int kScoreThreads = 256;
constexpr int kScoreWarps = kScoreThreads / 32;
constexpr int kGroups = kScoreThreads / 4;      // at least kMaxTop
constexpr int kCandidates = 768;
constexpr int kMaxCluster = 8;
static_assert(kGroups >= static_cast<int>(kMaxTop), "the threshold is the k-th largest group maximum");
static_assert(kCandidates >= kMaxCluster * static_cast<int>(kMaxTop), "the lists of a cluster are ranked together");

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// what one has read: greatest logit m, S = sum 2^a, T = sum 2^a a with a = (z - m) c
struct Sums { float m, s, t; };

// S and T relative to another maximum (at least the own one): 2^(a + x) (a + x) = 2^x (2^a a + x 2^a)
__device__ __forceinline__ void rebase(Sums& v, float m, float c)
{
    if (v.m == m) return;
    const float x = (v.m - m) * c, f = ex2(x);
    const float fx = f == 0.f ? 0.f : f * x;          // also from m = -inf: nothing was summed yet
    v.t = f == 0.f ? 0.f : __fmaf_rn(v.s, fx, v.t * f);
    v.s = f == 0.f ? 0.f : v.s * f;
    v.m = m;
}
// order of (logit, index): larger logit first, then lower index; -0 counts as +0
__device__ __forceinline__ uint32_t order_of(float z)
{
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }

// the sums of N lanes (a power of two), in every one of them
template <int N> __device__ __forceinline__ Sums join_lanes(Sums v, float c)
{
    float m = v.m;
    if (N == 32) m = value_of(__reduce_max_sync(~0u, order_of(m)));        // (a NaN out of max_nan has the greatest order)
    else
#pragma unroll
        for (int o = N / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, o));
    rebase(v, m, c);
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) {
        v.s += __shfl_xor_sync(~0u, v.s, o);
        v.t += __shfl_xor_sync(~0u, v.t, o);
    }
    return v;
}

__device__ __forceinline__ unsigned long long key_of(float z, uint32_t idx)
{
    return (static_cast<unsigned long long>(order_of(z)) << 32) | (0xFFFFFFFFu - idx);
}
__device__ __forceinline__ float value_of(unsigned long long key) { return value_of(static_cast<uint32_t>(key >> 32)); }
__device__ __forceinline__ uint32_t index_of(unsigned long long key) { return 0xFFFFFFFFu - static_cast<uint32_t>(key); }

// greatest and least of a lane's 16 bytes (a NaN wins both)
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <typename T, int N> __device__ __forceinline__ void extremes(const uint4 (&w)[N], float& top, float& low)
{
    if (sizeof(T) == 4) {
        top = -INFINITY;
        low = INFINITY;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const float a = __uint_as_float(w[u].x), b = __uint_as_float(w[u].y), c = __uint_as_float(w[u].z), d = __uint_as_float(w[u].w);
            top = max3_nan(top, a, max3_nan(b, c, d));
            low = min3(low, a, min3(b, c, d));
        }
    } else {
        uint32_t hi = w[0].x, lo = w[0].x;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (u) { hi = max2_nan(hi, w[u].x); lo = min2_nan(lo, w[u].x); }
            hi = max2_nan(hi, max2_nan(w[u].y, max2_nan(w[u].z, w[u].w)));
            lo = min2_nan(lo, min2_nan(w[u].y, min2_nan(w[u].z, w[u].w)));
        }
        top = max_nan(__uint_as_float(hi << 16), __uint_as_float(hi & 0xFFFF0000u));
        low = fminf(__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u));
    }
}

// A CTA's share of a row: vectors [v0, v1) of the row's 16-byte aligned middle, and up to CPL - 1 single elements at
// either end (given to the first and the last CTA).
template <typename T> struct Share {
    static constexpr int CPL = Store<T>::CPL;
    const T* row;
    uint32_t lead;            // elements before the aligned middle
    uint32_t v0, v1;
    uint32_t head, tail0, tail;   // single elements: 0 .. head - 1, tail0 .. tail0 + tail - 1
    __device__ __forceinline__ Share(const T* r, uint32_t vocab, uint32_t rank, uint32_t ranks) : row(r)
    {
        const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T);
        lead = min(off ? CPL - off : 0u, vocab);
        const uint32_t n = (vocab - lead) / CPL;
        v0 = static_cast<uint32_t>(static_cast<uint64_t>(n) * rank / ranks);
        v1 = static_cast<uint32_t>(static_cast<uint64_t>(n) * (rank + 1) / ranks);
        head = rank == 0 ? lead : 0u;
        tail0 = lead + n * CPL;
        tail = rank == ranks - 1 ? vocab - tail0 : 0u;
    }
    __device__ __forceinline__ uint4 load(uint32_t v) const { return __ldg(reinterpret_cast<const uint4*>(row + lead) + v); }
    // single element e (0 .. 2 CPL - 1) of this CTA: its index, or false
    __device__ __forceinline__ bool single(uint32_t e, uint32_t& idx) const
    {
        if (e < static_cast<uint32_t>(CPL)) { idx = e; return e < head; }
        idx = tail0 + e - CPL;
        return e - CPL < tail;
    }
};

template <typename T>
__global__ void __launch_bounds__(kScoreThreads, 5) score_kernel(const __grid_constant__ ScoreArgs a, uint32_t ranks)
{
    constexpr int CPL = Store<T>::CPL, U = 6;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t row = blockIdx.x / ranks, rank = blockIdx.x - row * ranks;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ Sums s_warp[kScoreWarps];
    __shared__ Sums s_cta;
    __shared__ __align__(16) uint32_t s_group[kGroups];
    __shared__ float s_tau, s_log;
    __shared__ unsigned int s_count;
    __shared__ unsigned long long s_cand[kCandidates];
    __shared__ unsigned long long s_top[kMaxTop];          // this CTA's top list, best first; 0 = no element
    __shared__ unsigned long long s_best[kScoreWarps];
    // The last warp joins the sums and writes the row, while the others still order the list. The target's logit is wanted
    // at the very end: its two dependent loads start here.
    const bool writer = tid == kScoreThreads - 32;

    const Share<T> sh(static_cast<const T*>(a.logits) + row * a.stride, a.vocab, rank, ranks);
    long long target = -1;
    float target_logit = 0.f;
    if (rank == 0 && writer && a.targets) {
        target = a.targets[row];
        if (target >= 0 && target < static_cast<long long>(a.vocab)) target_logit = Store<T>::load1(sh.row + target);
    }
    const float c = a.scale * kLog2e;
    const f32x2 c2 = pack2(__float_as_uint(c), __float_as_uint(c));
    float m = -INFINITY;
    f32x2 s2 = 0, t2 = 0;                    // two partial sums each
    auto raise = [&](float to) {             // a new maximum (or a NaN)
        const float x = (m - to) * c, f = ex2(x);
        const float fx = f == 0.f ? 0.f : f * x;      // (also from m = -inf: nothing was summed yet)
        m = to;
        const f32x2 f2 = pack2(__float_as_uint(f), __float_as_uint(f)), g2 = pack2(__float_as_uint(fx), __float_as_uint(fx));
        t2 = fma2(s2, g2, mul2(t2, f2));
        s2 = mul2(s2, f2);
    };
    auto add = [&](f32x2 a2) {               // two elements 2^a
        float a0, a1;
        unpack2(a2, a0, a1);
        const f32x2 e = pack2(__float_as_uint(ex2(a0)), __float_as_uint(ex2(a1)));
        s2 = add2(s2, e);
        t2 = fma2(e, a2, t2);
    };
    auto exponent = [&](float z) { return max_nan((z - m) * c, -1e30f); };      // masked logits: 2^a is 0, and 0 times a finite number is 0
    float second = -INFINITY;                // greatest element outside the batch that holds the maximum
    uint32_t best = 0;
    auto take = [&](const auto& raw, uint32_t v) {       // N words of 16 bytes, from vector v on
        constexpr int N = sizeof(raw) / 16;
        float top, low;
        extremes<T, N>(raw, top, low);
        if (!(top <= m)) {
            second = m;
            best = 8 * v + N;
            raise(max_nan(m, top));
        } else {
            second = fmaxf(second, top);
        }
        if (m == -INFINITY) return;
        const f32x2 neg = pack2(__float_as_uint(-m), __float_as_uint(-m));
        if ((low - m) * c > -1e30f) {        // no exponent of the batch leaves fp32's range, at either end of the logits
#pragma unroll
            for (int u = 0; u < N; ++u) {
                f32x2 z[CPL / 2];
                Store<T>::widen2(raw[u], z);
#pragma unroll
                for (int e = 0; e < CPL / 2; ++e) add(mul2(add2(z[e], neg), c2));
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                f32x2 z[CPL / 2];
                Store<T>::widen2(raw[u], z);
#pragma unroll
                for (int e = 0; e < CPL / 2; ++e) {
                    float z0, z1;
                    unpack2(z[e], z0, z1);
                    add(pack2(__float_as_uint(exponent(z0)), __float_as_uint(exponent(z1))));
                }
            }
        }
    };
    uint32_t v = sh.v0 + tid;
    for (; v + (U - 1) * kScoreThreads < sh.v1; v += kScoreThreads * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = sh.load(v + u * kScoreThreads);
        take(raw, v);
    }
    // what is left, fewer than U: all loads first, then four, two and one of them at a time
    const uint32_t left = v < sh.v1 ? (sh.v1 - v + kScoreThreads - 1) / kScoreThreads : 0u;
    static_assert(U <= 8, "the rest is three bits");
    uint4 four[4], two[2], one[1];
#pragma unroll
    for (uint32_t u = 0; u < 4; ++u)
        if (left & 4u) four[u] = sh.load(v + u * kScoreThreads);
#pragma unroll
    for (uint32_t u = 0; u < 2; ++u)
        if (left & 2u) two[u] = sh.load(v + ((left & 4u) + u) * kScoreThreads);
    if (left & 1u) one[0] = sh.load(v + (left & 6u) * kScoreThreads);
    uint32_t idx = 0;
    float edge = -INFINITY;                  // this thread's single element
    const bool has_edge = tid < 2 * CPL && sh.single(tid, idx);
    if (has_edge) edge = Store<T>::load1(sh.row + idx);
    if (left & 4u) take(four, v);
    if (left & 2u) take(two, v + (left & 4u) * kScoreThreads);
    if (left & 1u) take(one, v + (left & 6u) * kScoreThreads);
    const float own_max = m;                 // of the vectors: single elements are offered one by one
    if (has_edge) {
        if (!(edge <= m)) raise(max_nan(m, edge));
        if (m != -INFINITY)                  // the second of the pair counts 0
            add(pack2(__float_as_uint(exponent(edge)), __float_as_uint(-1e30f)));
    }
    Sums me;
    {
        float s0, s1, t0, t1;
        unpack2(s2, s0, s1);
        unpack2(t2, t0, t1);
        me = join_lanes<32>(Sums{m, s0 + s1, t0 + t1}, c);
    }
    if (lane == 0) s_warp[warp] = me;
    if (a.top_k) {
        // four threads' maximum as a whole number in the logits' order; the last bits hold the group, so that no two are equal
        float gm = max_nan(m, __shfl_xor_sync(~0u, m, 1));
        gm = max_nan(gm, __shfl_xor_sync(~0u, gm, 2));
        if ((tid & 3) == 0) s_group[tid >> 2] = (order_of(gm) & ~(kGroups - 1u)) | (tid >> 2);
        if (tid == 0) s_count = 0;
        if (tid < static_cast<int>(kMaxTop)) s_top[tid] = 0ull;
    }
    __syncthreads();
    auto log_sum = [](const Sums& all) { return all.m == -INFINITY ? -INFINITY : logf(all.s); };
    auto write_row = [&](const Sums& all, float ln) {        // by the thread that holds the target
        const bool none = all.m == -INFINITY;
        a.stats[row] = all.m;
        a.stats[static_cast<size_t>(a.n_rows) + row] = ln;
        a.entropy[row] = none ? 0.f : __fmaf_rn(-kLn2, all.t / all.s, ln);
        if (a.targets) {
            float lp;
            if (target < 0) lp = 0.f;
            else if (target >= static_cast<long long>(a.vocab)) lp = NAN;
            else if (none) lp = -INFINITY;
            else lp = __fmaf_rn(a.scale, target_logit - all.m, -ln);
            a.logprob[row] = lp;
        }
    };
    auto finish_sums = [&] {
        if (warp != kScoreWarps - 1) return;
        const Sums all = join_lanes<kScoreWarps>(s_warp[lane % kScoreWarps], c);
        if (!writer) return;
        s_cta = all;
        if (ranks == 1) write_row(all, s_log = log_sum(all));
    };
    if (!a.top_k) finish_sums();
    // ---- top list of the CTA
    if (a.top_k) {
        const uint32_t mine = s_group[tid >> 2];
        uint32_t before = 0;                 // groups in front of this one; each of its threads counts in a quarter
#pragma unroll
        for (int j = 0; j < kGroups / 16; ++j) {
            const uint4 o = reinterpret_cast<const uint4*>(s_group)[(tid & 3) * (kGroups / 16) + j];
            before += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
        before += __shfl_xor_sync(~0u, before, 1);
        before += __shfl_xor_sync(~0u, before, 2);
        // (the group's number cut off: at most the maximum itself; below the order of the lowest finite number there is only -inf)
        if (before == a.top_k - 1 && (tid & 3) == 0) s_tau = mine < 0x00800000u ? -INFINITY : value_of(mine & ~(kGroups - 1u));
        __syncthreads();
        const float tau = s_tau;
        auto offer = [&](float z, uint32_t i) {
            if (z >= tau && z > -INFINITY) {
                const unsigned int at = atomicAdd(&s_count, 1u);
                if (at < kCandidates) s_cand[at] = key_of(z, i);
            }
        };
        auto look_again = [&](uint32_t v) {
            const uint4 raw[1] = {sh.load(v)};
            float top, low;
            extremes<T, 1>(raw, top, low);
            if (!(top >= tau)) return;
            float z[CPL];
            Store<T>::widen(raw[0], z);
            uint32_t found = 0;
#pragma unroll
            for (int e = 0; e < CPL; ++e) found |= (z[e] >= tau ? 1u : 0u) << e;
            for (; found; found &= found - 1) {
                const uint32_t i = sh.lead + v * CPL + __ffs(found) - 1;
                offer(Store<T>::load1(sh.row + i), i);
            }
        };
        // each warp reads again for its own threads: eight lanes for one's batch, or all of them for everything one has read
        const bool hot = own_max >= tau && own_max > -INFINITY;
        for (uint32_t some = __ballot_sync(~0u, hot && second < tau); some;) {
            int src = -1;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (lane >> 3 == q) src = __ffs(some) - 1;
                some &= some - 1;            // (0 stays 0)
            }
            const uint32_t b = __shfl_sync(~0u, best, src < 0 ? 0 : src);
            if (src >= 0 && (lane & 7u) < (b & 7u)) look_again((b >> 3) + (lane & 7u) * kScoreThreads);
        }
        for (uint32_t some = __ballot_sync(~0u, hot && !(second < tau)); some; some &= some - 1)
            for (uint32_t v = sh.v0 + warp * 32 + __ffs(some) - 1 + lane * kScoreThreads; v < sh.v1; v += 32 * kScoreThreads) look_again(v);
        offer(edge, idx);
        __syncthreads();
        finish_sums();
        const unsigned int n = s_count;
        if (n <= kCandidates) {
            for (unsigned int first = 0; first < n; first += kScoreThreads / 8) {        // eight threads rank a candidate
                const unsigned int i = first + (tid >> 3);
                const unsigned long long key = i < n ? s_cand[i] : ~0ull;
                unsigned int ahead = 0;
#pragma unroll 4
                for (unsigned int j = tid & 7; j < n; j += 8) ahead += s_cand[j] > key;
                ahead += __shfl_xor_sync(~0u, ahead, 1);
                ahead += __shfl_xor_sync(~0u, ahead, 2);
                ahead += __shfl_xor_sync(~0u, ahead, 4);
                if (i < n && ahead < a.top_k && (tid & 7) == 0) s_top[ahead] = key;
            }
        } else {
            // more equal (or nearly equal) logits than the list holds: the best below the last, k times over
            unsigned long long last = ~0ull;
            for (uint32_t k = 0; k < a.top_k; ++k) {
                unsigned long long best = 0;
                auto look = [&](float z, uint32_t i) {
                    const unsigned long long key = z > -INFINITY ? key_of(z, i) : 0ull;
                    if (key < last && key > best) best = key;
                };
                for (uint32_t v = sh.v0 + tid; v < sh.v1; v += kScoreThreads) {
                    float z[CPL];
                    Store<T>::widen(sh.load(v), z);
#pragma unroll
                    for (int e = 0; e < CPL; ++e) look(z[e], sh.lead + v * CPL + e);
                }
                look(edge, idx);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long b = __shfl_xor_sync(~0u, best, o);
                    if (b > best) best = b;
                }
                if (lane == 0) s_best[warp] = best;
                __syncthreads();
                best = s_best[0];
                for (int w = 1; w < kScoreWarps; ++w)
                    if (s_best[w] > best) best = s_best[w];
                if (tid == 0) s_top[k] = best;
                last = best;
                __syncthreads();
                if (!best) break;            // the same in every thread
            }
        }
    }
    // ---- the row: sums and top lists of the cluster's CTAs meet in the first one
    if (ranks > 1) cluster.sync(); else __syncthreads();
    if (rank == 0) {
        Sums all = s_cta;
        if (ranks > 1) {
            const uint32_t r = lane % kMaxCluster;
            all = join_lanes<kMaxCluster>(r < ranks ? *cluster.map_shared_rank(&s_cta, r) : Sums{-INFINITY, 0.f, 0.f}, c);
        }
        const float ln = ranks == 1 ? s_log : log_sum(all);
        const bool bad = all.m != -INFINITY && !(all.s < INFINITY);       // a NaN or +inf among the logits: NaN sum
        if (ranks > 1 && writer) write_row(all, ln);
        if (a.top_k) {
            if (ranks > 1) {
                // the other CTAs' lists join this one's; k * ranks entries, ranked like the candidates
                const unsigned int n = a.top_k * ranks;
                for (unsigned int i = tid; i < n; i += kScoreThreads) s_cand[i] = cluster.map_shared_rank(s_top, i / a.top_k)[i % a.top_k];
                __syncthreads();
                if (tid < static_cast<int>(kMaxTop)) s_top[tid] = 0ull;
                __syncthreads();
                // each list is in order: `ranks` lanes (a power of two) look up one entry's place in each of them
                for (unsigned int first = 0; first < n * ranks; first += kScoreThreads) {
                    const unsigned int i = (first + tid) / ranks, list = (first + tid) % ranks;
                    const unsigned long long mine = i < n ? s_cand[i] : 0ull;
                    unsigned int lo = 0, hi = a.top_k;           // entries before lo are greater, those from hi on are not
                    while (lo < hi) {
                        const unsigned int mid = (lo + hi) / 2;
                        if (s_cand[list * a.top_k + mid] > mine) lo = mid + 1;
                        else hi = mid;
                    }
                    for (uint32_t o = 1; o < ranks; o *= 2) lo += __shfl_xor_sync(~0u, lo, o);
                    if (mine && lo < a.top_k && list == 0) s_top[lo] = mine;
                }
                __syncthreads();
            }
            if (tid < static_cast<int>(a.top_k)) {
                const unsigned long long key = bad ? 0ull : s_top[tid];
                const size_t at = static_cast<size_t>(row) * a.top_k + tid;
                a.top_ids[at] = key ? static_cast<long long>(index_of(key)) : -1;
                a.top_logprobs[at] = bad ? NAN : (key ? __fmaf_rn(a.scale, value_of(key) - all.m, -ln) : -INFINITY);
            }
        }
    }
    if (ranks > 1) cluster.sync();           // nobody leaves while its shared memory may still be read
}

// ---- gradient ---------------------------------------------------------------------------------
constexpr int kGradThreads = 256;
constexpr int kGradVectors = 4;       // per thread

// p and log p come back from the row's stats; one exponential per element, one read, one write. Bound by HBM, now that two
// elements share their instructions: 4096 x 32128 bf16 80.6 us, 6.5 TB/s; rows off 16-byte boundaries, 2048 x 50257, 66 us (one
// element at a time: a twentieth and a ninth slower). It takes 32 registers, eight CTAs per SM: the same work in 34 (six CTAs)
// 83.5 and 69.7 us.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) score_grad_kernel(const __grid_constant__ ScoreGradArgs a, uint32_t chunks)
{
    constexpr int CPL = Store<T>::CPL;
    const uint32_t row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    T* dz = static_cast<T*>(a.grad) + row * a.grad_stride;
    const uint32_t per = kGradThreads * kGradVectors * CPL;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T);
    const uint32_t lead = min(off ? CPL - off : 0u, a.vocab);
    // rows of the two tensors that sit alike in their 16-byte words go word by word, others element by element
    const bool alike = (reinterpret_cast<uintptr_t>(dz) & 15) == (reinterpret_cast<uintptr_t>(z) & 15);
    const uint32_t n = alike ? (a.vocab - lead) / CPL : 0u, v0 = chunk * (kGradThreads * kGradVectors) + threadIdx.x;
    float m = a.stats[row], ln = a.stats[static_cast<size_t>(a.n_rows) + row];
    const long long tk = a.targets && a.g_logprob ? a.targets[row] : -1;
    float gl = tk >= 0 ? a.g_logprob[row] : 0.f;
    if (tk >= static_cast<long long>(a.vocab)) gl = NAN;
    float gh = a.g_entropy ? a.g_entropy[row] : 0.f;
    if (m == -INFINITY) m = ln = gl = gh = 0.f;           // nothing left in the row: the gradient is 0
    const uint32_t target = tk >= 0 && tk < static_cast<long long>(a.vocab) ? static_cast<uint32_t>(tk) : ~0u;
    // dz = p (a_p + a_pl log p) [+ scale g_lp at the target], two at a time. A p of 0 has to give 0, so the bracket has to be a
    // number there. For masked logits log p stops at -1000, where p has long been 0; and gradients that may overflow the bracket
    // are taken in parts of 2^64, for which p counts 2^64 (2^-64 is exact).
    const float h = a.g_entropy ? a.entropy[row] : 0.f, at_target = a.scale * gl, c = a.scale * kLog2e;
    const bool parts = a.scale * (fabsf(gl) + fabsf(gh) * (h + 1100.f)) == INFINITY;
    const float part = parts ? 0x1p-64f : 1.f;
    gl *= part;
    gh *= part;
    const float a_p = -a.scale * __fmaf_rn(gh, h, gl), a_pl = -a.scale * gh;
    auto both = [](float x) { return pack2(__float_as_uint(x), __float_as_uint(x)); };
    const f32x2 neg_m = both(-m), scale2 = both(a.scale), neg_ln = both(-ln), c2 = both(c), ln2 = both(-ln * kLog2e + (parts ? 64.f : 0.f)), a_p2 = both(a_p), a_pl2 = both(a_pl);
    auto grad2 = [&](f32x2 x) {
        const f32x2 d = add2(x, neg_m);
        float l0, l1, e0, e1;
        unpack2(fma2(scale2, d, neg_ln), l0, l1);
        const f32x2 lp = pack2(__float_as_uint(max_nan(l0, -1000.f)), __float_as_uint(max_nan(l1, -1000.f)));
        unpack2(fma2(d, c2, ln2), e0, e1);
        return mul2(pack2(__float_as_uint(ex2(e0)), __float_as_uint(ex2(e1))), fma2(a_pl2, lp, a_p2));
    };
    auto grad = [&](float x) {
        float y, other;
        unpack2(grad2(both(x)), y, other);
        return y;
    };
    if (alike) {
        uint4 raw[kGradVectors];
#pragma unroll
        for (int u = 0; u < kGradVectors; ++u)
            if (v0 + u * kGradThreads < n) raw[u] = __ldcs(reinterpret_cast<const uint4*>(z + lead) + v0 + u * kGradThreads);
#pragma unroll
        for (int u = 0; u < kGradVectors; ++u) {
            const uint32_t v = v0 + u * kGradThreads;
            if (v >= n) break;
            f32x2 z2[CPL / 2];
            Store<T>::widen2(raw[u], z2);
            float x[CPL];
#pragma unroll
            for (int e = 0; e < CPL / 2; ++e) unpack2(grad2(z2[e]), x[2 * e], x[2 * e + 1]);
            const uint32_t at = target - (lead + v * CPL);      // beyond CPL also when there is no target: a row has fewer than 2^31 elements
            if (at < CPL) {
#pragma unroll
                for (int e = 0; e < CPL; ++e)
                    if (e == static_cast<int>(at)) x[e] += at_target;
            }
            Out<T>::template store<CPL>(dz + lead + v * CPL, x);
        }
        if (chunk == 0 && threadIdx.x < 2 * CPL) {
            const uint32_t e = threadIdx.x, tail0 = lead + n * CPL;
            const uint32_t j = e < static_cast<uint32_t>(CPL) ? e : tail0 + e - CPL;
            if (e < static_cast<uint32_t>(CPL) ? e < lead : j < a.vocab) Out<T>::store1(dz + j, grad(Store<T>::load1(z + j)) + (j == target ? at_target : 0.f));
        }
    } else {
        for (uint32_t i = threadIdx.x; i < per; i += kGradThreads) {
            const uint64_t j = static_cast<uint64_t>(chunk) * per + i;
            if (j < a.vocab) Out<T>::store1(dz + j, grad(Store<T>::load1(z + j)) + (j == target ? at_target : 0.f));
        }
    }
}

template <typename T> cudaError_t launch_scores_t(const ScoreArgs& a, int sm_count, cudaStream_t s)
{
    // a cluster shares a row while the rows alone do not fill the SMs and a share still is a few thousand elements
    uint32_t ranks = 1;
    while (ranks < kMaxCluster && static_cast<uint64_t>(a.n_rows) * ranks * 2 <= static_cast<uint64_t>(sm_count) * 4 && a.vocab / (ranks * 2) >= 2048) ranks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.n_rows * ranks);
    cfg.blockDim = dim3(kScoreThreads);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = ranks > 1;
    return cudaLaunchKernelEx(&cfg, score_kernel<T>, a, ranks);
}

template <typename T> cudaError_t launch_grad_t(const ScoreGradArgs& a, cudaStream_t s)
{
    constexpr uint32_t per = kGradThreads * kGradVectors * Store<T>::CPL;
    const uint32_t chunks = (a.vocab + per - 1) / per;
    if (!chunks) return cudaSuccess;
    if (static_cast<uint64_t>(chunks) * a.n_rows > 0x7FFFFFFFull) return cudaErrorInvalidConfiguration;
    score_grad_kernel<T><<<static_cast<unsigned>(chunks * a.n_rows), kGradThreads, 0, s>>>(a, chunks);
    return cudaGetLastError();
}

}  // namespace

int launch_scores(int dtype, const ScoreArgs& a, int sm_count, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return static_cast<int>(dtype == 1 ? launch_scores_t<bf16>(a, sm_count, s) : launch_scores_t<float>(a, sm_count, s));
}

int launch_score_grad(int dtype, const ScoreGradArgs& a, void* stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return static_cast<int>(dtype == 1 ? launch_grad_t<bf16>(a, s) : launch_grad_t<float>(a, s));
}

}  // namespace randes
