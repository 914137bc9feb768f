// das_sample.cu -- sampling with temperature, top-k, top-p and min-p from
// given random numbers, and the acceptance of proposals against the draws.
//
// A filter keeps a prefix of the tokens ordered by logit (largest first,
// equal ones by index), so each is one threshold: a key (the logit's bits made
// monotone) and how many of the tokens equal to it, lowest index first, stay.
// The threshold is where a sum over keys >= t first reaches a target: a sum of
// ones for top-k, of the whole-number weights for top-p.  The row is not sorted for
// it; the few candidates of a small top-k are.
//
// sample_kernel: a cluster of CTAs holds a row in shared memory, read once.  A
// threshold is found from a histogram of kBins bins in shared memory, over
// the logits (top-k) or the exponents (top-p), summed over the cluster; what
// falls into the threshold's bin, rarely more than some dozens, is compared
// pair by pair, or binned again by its keys if it is more than kList.  16-bit
// logits have a bin for each value.  The token is found from sums over
// segments in index order.  The candidates of a small top-k, if they are no
// more than a CTA's threads, are sorted instead (128 rows of 32000: 3.5 us less
// than with the thresholds above over the candidates).
//
// The row is read from memory once, which would take 2.4 us for 128 rows of
// 32000 binary32 logits or 64 of 128257 in bf16 (16.4 MB).  Measured: 17.1 us
// (top-k 200, top-p 0.95, min-p 0.02) and 34.5 us (top-p 0.9 alone): the time goes to the
// passes over the row in shared memory (the largest, the candidates or the
// bins, the sums), which each thread makes over 32 to 128 logits with some
// dozens of instructions each, and to eight or so barriers of the cluster.  The
// smallest call, one row of 32000 in a cluster of eight, takes 15.1 us, all
// latency: the launch, the row from memory, and those barriers in turn.
// Sorting the row would take a pass over it for every few bits of the key.
//
// Every kernel here is launched as a programmatic dependent of the previous
// kernel in the stream: it reads nothing before griddepcontrol.wait, and
// every CTA executes that wait.
#include <algorithm>
#include <atomic>
#include <cstddef>
#include <type_traits>

#include <cooperative_groups.h>

#include "das_internal.h"

namespace cg = cooperative_groups;

namespace das {
namespace {

using u64 = unsigned long long;
constexpr int kLongThreads = 1024;
constexpr int kScanWarps = 4;
constexpr uint32_t kFull = 0xffffffffu;

// A logit as a key that compares like the number: -0 equals 0, NaN is -inf.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (!(x == x)) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyNone = 0x007fffffu;  // key of -inf

__device__ __forceinline__ float e_of(uint32_t key, uint32_t top, float m, float T) {
    if (key == top) return 1.f;
    if (key == kKeyNone) return 0.f;
    return expf((logit_of(key) - m) / T);
}
__device__ __forceinline__ u64 w_of(float e) { return __float2ull_rn(e * 4294967296.f); }

template <typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, T *sums, F f) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(kFull, v, d));
    if (lane == 0) sums[warp] = v;
    __syncthreads();
    v = sums[lane];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = f(v, __shfl_xor_sync(kFull, v, d));
    __syncthreads();
    return v;
}

// ---- a row in the shared memory of a cluster ---------------------------------------
constexpr int kThreads = 1024, kWarps = kThreads / 32;
static_assert(kWarps == 32, "a warp scans the warps' sums");
constexpr int kMaxRowCtas = 8;                 // a portable cluster
// Logits per CTA, as they come: what shared memory holds, and fewer than 2^16, so that
// a bin's sums of 16-bit pieces stay below 2^32.
template <bool BF16>
constexpr int kSliceBytes = BF16 ? 131072 : 180224;
constexpr int kMaxSegs = 512;  // of one warp's 32 groups of four
static_assert(kSliceBytes<true> / 2 <= kMaxSegs * 128 && kSliceBytes<false> / 4 <= kMaxSegs * 128, "segments");
constexpr int kBins = 2048;
constexpr int kList = 256;
constexpr int kValues = 4096;               // bins of 16-bit values, sixteen octaves of each sign
constexpr uint32_t kValueBase = 0x3b80u;    // bf16 bits of 2^-8
constexpr int kCand = 2048;
constexpr int kSmall = 2 * kMaxSegs;
// exponents past the last bin have weights that round to 0: e^-23 < 2^-33
constexpr float kNats = 23.f;
constexpr uint32_t kOne = 0xffffffffu;  // stands for the weight 2^32

struct alignas(16) Shared {
    float cand[kCand];              // the candidates left by a small top-k,
    int cand_at[kCand];             // in index order
    uint32_t hist[2 * kBins];       // bin i's sum: [i] + 2^16 [kBins + i]; or kValues counts
    u64 scan[kWarps];
    u64 seg[kMaxSegs];
    uint32_t n_seg[kMaxSegs];
    u64 xch[2][3][kMaxRowCtas];  // values of every CTA of the cluster
    uint32_t list[kList];  // the CTA's keys in a bin
    uint2 all[kList];      // the cluster's, with their weights
    uint32_t list_n, key_min, key_max;
    int bin, where;
    uint32_t cut;
    u64 above, target, sum, equal;
};

// With one proposal a sequence its acceptance needs no other row.
__device__ __forceinline__ void accept_one(const SampleArgs &a, size_t row, int token) {
    if (!a.draft) return;
    const int d = a.draft[row];
    a.accepted[row] = token >= 0 && d == token;
    a.next_token[row] = token;  // the proposal itself, where it was accepted
    if (a.committed) a.committed[row] = 1;
}

// (apart, as few calls need it: inlined it would be in every loop)
__device__ __noinline__ float plain_e(float l, float m, float T) { return expf((l - m) / T); }

__device__ __forceinline__ u64 wide(uint32_t w) { return (u64)w + (w == kOne); }

template <bool BF16>
__global__ void __launch_bounds__(kThreads, 1) sample_kernel(const SampleArgs a, int slice) {
    __shared__ Shared s;
    extern __shared__ uint4 held[];  // the CTA's logits in groups of four, padded with -inf
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const size_t row = blockIdx.x / C;
    const int b = (int)(row / a.W);
    auto of = [&](int r) { return C > 1 ? cluster.map_shared_rank(&s, r) : &s; };
    auto sync = [&] {  // the cluster's threads, or the CTA's
        if (C > 1) cluster.sync();
        else __syncthreads();
    };
    int turn = 0;
    // Three values of each CTA to every CTA, in s.xch[returned]; two sets in
    // turn, so that none is written while another CTA may still read it.
    auto exchange = [&](u64 x, u64 y, u64 z) {  // the same in all threads
        turn ^= 1;
        if (tid < C) {
            u64(*to)[kMaxRowCtas] = of(tid)->xch[turn];
            to[0][rank] = x;
            to[1][rank] = y;
            to[2][rank] = z;
        }
        sync();
        return turn;
    };
    auto warp_scan = [&](u64 v) {  // inclusive
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const u64 y = __shfl_up_sync(kFull, v, d);
            if (lane >= d) v += y;
        }
        return v;
    };
    auto scan = [&](u64 v, u64 &total) {  // exclusive sum over the CTA
        const u64 x = warp_scan(v);
        if (lane == 31) s.scan[warp] = x;
        __syncthreads();
        const u64 sums = warp_scan(s.scan[lane]);  // by every warp for itself
        total = __shfl_sync(kFull, sums, 31);
        const u64 before = __shfl_sync(kFull, sums, warp > 0 ? warp - 1 : 0);
        __syncthreads();
        return (warp > 0 ? before : 0) + x - v;
    };

    if (tid == 0) {
        s.key_max = 0;
        s.list_n = 0;
    }
    if (BF16)
        for (int i = tid; i < kValues / 4; i += kThreads)
            reinterpret_cast<uint4 *>(s.hist)[i] = make_uint4(0, 0, 0, 0);
    sync();  // every CTA of the cluster has started
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    float T = a.sampling.temperature ? a.sampling.temperature[b] : 1.f;
    long long k = a.sampling.top_k ? a.sampling.top_k[b] : 0;
    const float p = a.sampling.top_p ? a.sampling.top_p[b] : 1.f;
    float floor_p = a.sampling.min_p ? a.sampling.min_p[b] : 0.f;
    floor_p = floor_p > 0.f ? fminf(floor_p, 1.f) : 0.f;  // NaN: none
    if (!(T > 0.f)) {
        T = 1.f;
        k = 1;
    }
    T = fminf(T, 3.4028234e38f);
    if (k <= 0 || k > a.vocab) k = a.vocab;

    // Bins of 16-bit values in falling order: 2^8 > l >= 2^-8, then -2^-8 >= l > -2^8.
    auto value_bin = [](float l) {
        const uint32_t bits = __float_as_uint(l), size = ((bits & 0x7fffffffu) >> 16) - kValueBase;
        return size < kValues / 2 ? kValues / 2 + (bits >> 31 ? size : ~size) : 0xffffffffu;
    };
    auto value_of = [](int bin) {
        const uint32_t size = bin < kValues / 2 ? kValues / 2 - 1 - bin : bin - kValues / 2;
        return __uint_as_float((size + kValueBase) << 16 | (bin < kValues / 2 ? 0u : 0x80000000u));
    };

    // ---- the row: NaN as -inf, -0 as 0 ----
    // With top-p alone the values' bins (of search, below) are counted as the row comes
    // (64 rows of 128257: 35.1 us, 36.5 with a pass of its own); the logits between
    // the two signs' bins are listed in s.seg.
    bool counted = BF16 && k >= a.vocab && p < 1.f;
    // Groups of four lie as the vector loads do: the CTA's first token is number
    // `shift` of group 0, and index `base` + 4 g + i - shift is token i of group g.
    using Elem = std::conditional_t<BF16, uint16_t, float>;
    const int base = rank * slice, len = max(0, min(slice, a.vocab - base));
    const Elem *src = static_cast<const Elem *>(a.logits) + row * (size_t)a.row_stride + base;
    const int shift = (int)(reinterpret_cast<uintptr_t>(src) / sizeof(Elem) & 3);
    int groups = len ? (len + shift + 3) / 4 : 0;
    bool few = false;  // whether the candidates alone are left
    float mine = -INFINITY;
    src -= shift;
#pragma unroll 4
    for (int g = tid; g < groups; g += kThreads) {
        float f[4];
        if (4 * g >= shift && 4 * g + 4 <= len + shift) {
            if constexpr (BF16) {
                const uint2 u = __ldcs(reinterpret_cast<const uint2 *>(src) + g);
                f[0] = __uint_as_float(u.x << 16);
                f[1] = __uint_as_float(u.x & 0xffff0000u);
                f[2] = __uint_as_float(u.y << 16);
                f[3] = __uint_as_float(u.y & 0xffff0000u);
            } else {
                const float4 u = __ldcs(reinterpret_cast<const float4 *>(src) + g);
                f[0] = u.x;
                f[1] = u.y;
                f[2] = u.z;
                f[3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = -INFINITY;
                if (4 * g + i >= shift && 4 * g + i < len + shift) {
                    if constexpr (BF16) f[i] = __uint_as_float((uint32_t)src[4 * g + i] << 16);
                    else f[i] = src[4 * g + i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = f[i] == f[i] ? f[i] + 0.f : -INFINITY;
            mine = fmaxf(mine, f[i]);
        }
        if (counted)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at = value_bin(f[i]);
                if (at < kValues) {
                    atomicAdd(s.hist + at, 1u);
                } else if (fabsf(f[i]) < 1.f) {
                    const uint32_t n = atomicAdd(&s.list_n, 1u);
                    if (n < kSmall) reinterpret_cast<float *>(s.seg)[n] = f[i];
                }
            }
        if (BF16)
            reinterpret_cast<uint2 *>(held)[g] =
                make_uint2(__float_as_uint(f[0]) >> 16 | (__float_as_uint(f[1]) & 0xffff0000u),
                           __float_as_uint(f[2]) >> 16 | (__float_as_uint(f[3]) & 0xffff0000u));
        else
            reinterpret_cast<float4 *>(held)[g] = make_float4(f[0], f[1], f[2], f[3]);
    }
    auto load4 = [&](int g, float (&l)[4]) {
        if (g >= groups) {
            l[0] = l[1] = l[2] = l[3] = -INFINITY;
        } else if (BF16 && !few) {
            const uint2 u = reinterpret_cast<const uint2 *>(held)[g];
            l[0] = __uint_as_float(u.x << 16);
            l[1] = __uint_as_float(u.x & 0xffff0000u);
            l[2] = __uint_as_float(u.y << 16);
            l[3] = __uint_as_float(u.y & 0xffff0000u);
        } else {
            const float4 u = few ? reinterpret_cast<const float4 *>(s.cand)[g]
                                 : reinterpret_cast<const float4 *>(held)[g];
            l[0] = u.x;
            l[1] = u.y;
            l[2] = u.z;
            l[3] = u.w;
        }
    };
    auto store4 = [&](int g, const float (&l)[4]) {
        if (BF16 && !few)
            reinterpret_cast<uint2 *>(held)[g] =
                make_uint2(__float_as_uint(l[0]) >> 16 | (__float_as_uint(l[1]) & 0xffff0000u),
                           __float_as_uint(l[2]) >> 16 | (__float_as_uint(l[3]) & 0xffff0000u));
        else if (few)
            reinterpret_cast<float4 *>(s.cand)[g] = make_float4(l[0], l[1], l[2], l[3]);
        else
            reinterpret_cast<float4 *>(held)[g] = make_float4(l[0], l[1], l[2], l[3]);
    };

    // ---- the largest logit m, and a logit that at least k are not below ----
    // Of k' = ceil(k / C) logits, in each CTA: where j n >= k', the j-th largest of the
    // warps' n-th largest of the threads' largest (the least such over the cluster).
    // n = ceil(k' / warps) + 1 leaves some 350 candidates of 32000 for k = 200, which
    // are sorted as 512; with n one less and the least of all warps they were 450 on
    // average and more than 512 in every third row (128 rows of 32000: 19.2 us, 17.1 now).
    float m, low = -INFINITY;
    {
        auto sorted32 = [&](uint32_t x) {  // a warp's keys, the largest in lane 0
#pragma unroll
            for (int size = 2; size <= 32; size *= 2)
#pragma unroll
                for (int d = size / 2; d > 0; d /= 2) {
                    const uint32_t o = __shfl_xor_sync(kFull, x, d);
                    x = !(lane & size) == !(lane & d) ? max(x, o) : min(x, o);
                }
            return x;
        };
        const uint32_t key = key_of(mine), top = __reduce_max_sync(kFull, key);
        const long long kc = (k + C - 1) / C, n = min((kc + kWarps - 1) / kWarps + 1, 32ll);
        const bool bound = k < a.vocab && kc <= n * kWarps;
        if (bound) {
            const uint32_t nth = __shfl_sync(kFull, sorted32(key), (int)n - 1);
            if (lane == 0) s.list[warp] = nth;
        }
        if (lane == 0) atomicMax(&s.key_max, top);
        __syncthreads();
        uint32_t here = kKeyNone;
        if (bound && warp == 0)
            here = __shfl_sync(kFull, sorted32(s.list[lane]), (int)((kc + n - 1) / n) - 1);
        const int t = exchange(s.key_max, here, 0);  // (by warp 0)
        uint32_t most = 0, least = kOne;
        for (int r = 0; r < C; ++r) {
            most = max(most, (uint32_t)s.xch[t][0][r]);
            least = min(least, (uint32_t)s.xch[t][1][r]);
        }
        if (most <= kKeyNone) {  // the same in every CTA
            if (rank == 0 && tid == 0) {
                accept_one(a, row, -1);
                a.tokens[row] = -1;
                if (a.logprobs) a.logprobs[row] = -INFINITY;
            }
            return;
        }
        m = logit_of(most);
        low = logit_of(max(least, kKeyNone + 1));
    }
    if (m == INFINITY) {  // the infinite ones alone have weight, and the same
        for (int g = tid; g < groups; g += kThreads) {
            float l[4];
            load4(g, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) l[i] = l[i] == INFINITY ? 0.f : -INFINITY;
            store4(g, l);
        }
        m = 0.f;
        low = -3.4028234e38f;
        counted = false;
    }

    // (l - m) / T as binary32 division rounds it.  With r = 1 / T rounded, q =
    // rn(x r), the exact remainder x - q T and one more fused step give the
    // quotient rounded to nearest (Markstein, 1990) unless T's significand is
    // all ones; quotients below -100, whose weight is 0, need no care (but no NaN).
    const float rT = __frcp_rn(T);
    const bool quick = T > 1e-18f && T < 1e18f && (__float_as_uint(T) & 0x7fffffu) != 0x7fffffu;
    auto quick_e = [&](float l) {
        const float d = l - m, q = fmaxf(d * rT, -100.f);
        return expf(fmaf(fmaf(-q, T, d), rT, q));
    };
    auto es_of = [&](const float (&l)[4], float (&e)[4]) {  // four, so that their steps overlap
        if (T == 1.f) {  // (the usual one; 64 rows of 128257: 36.5 us, 37.8 with the steps below)
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = expf(l[i] - m);
        } else if (quick) {
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = quick_e(l[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = plain_e(l[i], m, T);
        }
    };
    auto code_of = [](float e) { return __float2uint_rn(e * 4294967296.f); };  // 2^32 saturates
    auto weight = [&](float l) { return code_of(quick ? quick_e(l) : plain_e(l, m, T)); };

    // The draw from n <= kThreads candidates (s.cand, in index order) that hold the
    // k largest, by one CTA: sorted by falling logit and rising index, the kept ones
    // are the first k of them whose predecessors' weights sum to less than the target.
    auto draw_sorted = [&](int n) {
        u64 x = 0;  // (a key above 0 marks a candidate)
        if (tid < n) x = (u64)key_of(s.cand[tid]) << 32 | (uint32_t)(kThreads - 1 - tid);
        u64 *const there = reinterpret_cast<u64 *>(s.hist);  // [2][kThreads]
        static_assert(sizeof s.hist >= 2 * kThreads * sizeof(u64));
        int set = 0, span = 32;  // a bitonic sort, by the warps that it takes
        while (span < n) span *= 2;
        if (tid < span)
            for (int size = 2; size <= span; size *= 2)
                for (int d = size / 2; d > 0; d /= 2) {
                    u64 y;
                    if (d >= 32) {
                        there[set + tid] = x;
                        asm volatile("bar.sync 1, %0;" ::"r"(span) : "memory");
                        y = there[set + (tid ^ d)];
                        set ^= kThreads;
                    } else {
                        y = __shfl_xor_sync(kFull, x, d);
                    }
                    if ((x < y) == (!(tid & size) == !(tid & d))) x = y;
                }
        const bool mine_in = tid < n && tid < k;
        const int at = kThreads - 1 - (int)(uint32_t)x;  // its place in s.cand
        float e[4] = {};
        uint32_t code = 0;
        if (mine_in) {
            const float l = logit_of((uint32_t)(x >> 32));
            e[0] = quick ? quick_e(l) : plain_e(l, m, T);
            code = code_of(e[0]);
        }
        if (p < 1.f) {
            u64 all;
            const u64 before = scan(wide(code), all);
            if (tid == 0) {
                const double want = ceil((double)p * (double)all);
                s.target = want < 1.0 ? 1 : (u64)want;
            }
            __syncthreads();
            if (before >= min(s.target, all)) code = 0;
        }
        if (floor_p > 0.f && !(e[0] >= floor_p)) code = 0;
        __syncthreads();  // (the last reads of `there`)
        if (tid < n) s.hist[at] = code;
        __syncthreads();
        code = tid < n ? s.hist[tid] : 0;
        u64 total;
        const u64 before = scan(wide(code), total);
        if (tid == 0) {
            float u = a.uniforms[row];
            if (!(u >= 0.f)) u = 0.f;
            const u64 r = (u64)((double)u * (double)total);
            s.target = r < total ? r : total - 1;
        }
        __syncthreads();
        const u64 r = s.target;
        if (before <= r && r < before + wide(code)) {
            const float l = s.cand[tid];
            a.tokens[row] = s.cand_at[tid];
            accept_one(a, row, s.cand_at[tid]);
            if (a.logprobs) {
                const float z = l == m ? 0.f : (l - m) / T;
                a.logprobs[row] = z - logf((float)((double)total * (1.0 / 4294967296.0)));
            }
        }
    };

    // ---- a small top-k leaves few candidates: those not below `low`, in index order ----
    // Four bits of each group of a thread say which; their numbers, in eight bits of
    // a word per round of groups, are summed over the warp for four rounds at once.
    if (k < a.vocab && k <= kCand / 4) {
        constexpr int kRounds = kSliceBytes<BF16> / (BF16 ? 2 : 4) / 4 / kThreads;
        static_assert(kRounds * 4 * kThreads * (BF16 ? 2 : 4) == kSliceBytes<BF16> && kRounds * kWarps <= kMaxSegs);
        constexpr int kHits = (kRounds + 7) / 8, kCounts = (kRounds + 3) / 4;
        uint32_t hits[kHits], count[kCounts];
#pragma unroll
        for (int i = 0; i < kHits; ++i) hits[i] = 0;
#pragma unroll
        for (int i = 0; i < kCounts; ++i) count[i] = 0;
#pragma unroll
        for (int it = 0; it < kRounds; ++it) {
            if (it * kThreads >= groups) continue;
            float l[4];
            load4(it * kThreads + tid, l);
            const uint32_t in = (uint32_t)(l[0] >= low) | (uint32_t)(l[1] >= low) << 1 |
                                (uint32_t)(l[2] >= low) << 2 | (uint32_t)(l[3] >= low) << 3;
            hits[it / 8] |= in << (it % 8 * 4);
            count[it / 4] |= __popc(in) << (it % 4 * 8);
        }
        uint32_t before[kCounts];  // exclusive, over the warp
#pragma unroll
        for (int i = 0; i < kCounts; ++i) {
            uint32_t x = count[i];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t y = __shfl_up_sync(kFull, x, d);
                if (lane >= d) x += y;
            }
            before[i] = x - count[i];
            if (lane == 31)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (4 * i + j < kRounds) s.seg[(4 * i + j) * kWarps + warp] = x >> (8 * j) & 0xffu;
        }
        __syncthreads();
        u64 n_all;
        const u64 ex = scan(tid < kRounds * kWarps ? s.seg[tid] : 0, n_all);
        if (tid < kRounds * kWarps) s.seg[tid] = ex;
        const int t = exchange(n_all, 0, 0);
        bool fit = true;  // in every CTA of the cluster, which all go one way
        int n_row = 0, n_before = 0;
        for (int r = 0; r < C; ++r) {
            fit = fit && s.xch[t][0][r] <= kCand;
            n_row += (int)min(s.xch[t][0][r], (u64)kCand);
            if (r < rank) n_before += (int)min(s.xch[t][0][r], (u64)kCand);
        }
        // few enough for a thread of the first CTA to have one each
        const bool sorted = fit && n_row <= kThreads;
        Shared *const to = sorted ? of(0) : &s;
        const int at0 = sorted ? n_before : 0;
        if (fit) {
#pragma unroll
            for (int it = 0; it < kRounds; ++it) {
                uint32_t in = hits[it / 8] >> (it % 8 * 4) & 15u;
                if (!in) continue;
                const int g = it * kThreads + tid;
                int at = at0 + (int)s.seg[it * kWarps + warp] + (int)(before[it / 4] >> (it % 4 * 8) & 0xffu);
                float l[4];
                load4(g, l);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (in >> i & 1) {
                        to->cand[at] = l[i];
                        to->cand_at[at++] = base + 4 * g + i - shift;
                    }
            }
            if (sorted) {
                sync();
                if (rank == 0) draw_sorted(n_row);
                return;
            }
            few = true;
            groups = ((int)n_all + 3) / 4;
            if (tid < 4 * groups - (int)n_all) s.cand[n_all + tid] = -INFINITY;
            // of the cluster: from here on other CTAs store their bins over the row, which
            // every CTA has to have taken its candidates out of
            sync();
        }
    }

    // Of the first `words` words of s.hist (one row, or two of kBins), the parts
    // [r per_cta, (r + 1) per_cta) go to CTA r, to [rank][row][per_cta] with `stride`
    // words a rank, and are there after the next barrier.  Stores are not waited
    // for as reads of the other CTAs' bins would be: one row of 32000 takes 15.1 us,
    // 15.8 with those.  Returns the place: the candidates', or the row's if the
    // candidates are in use.
    auto send_bins = [&](int words, int per_cta, int stride) -> const uint32_t * {
        uint32_t *const place = few ? reinterpret_cast<uint32_t *>(held) : reinterpret_cast<uint32_t *>(s.cand);
        if (C == 1) return s.hist;
        if (4 * tid < words) {
            const int row = stride > per_cta ? 4 * tid / kBins : 0, bin = 4 * tid - row * kBins;
            const int r = bin / per_cta, off = bin - r * per_cta;
            uint32_t *const there = cluster.map_shared_rank(place, r);
            *reinterpret_cast<uint4 *>(there + rank * stride + row * per_cta + off) =
                reinterpret_cast<const uint4 *>(s.hist)[tid];
        }
        return place;
    };
    static_assert(sizeof s.cand + sizeof s.cand_at >= sizeof s.hist && kValues == 2 * kBins &&
                  2 * kBins == 4 * kThreads && offsetof(Shared, cand_at) == sizeof s.cand, "bins sent");

    // ---- the threshold of a sum over the logits from `from` up ----
    // Finds the largest t with the sum of f over logits > t below the target
    // (then s.above), leaves its key in s.cut and how many have it in s.equal;
    // false if the sum of all is below the target, which thread 0 makes of it
    // (s.target).
    auto search = [&](auto weights, float from, float per_logit, auto target_of) {
        constexpr bool kWeights = decltype(weights)::value;
        float lo = from, hi = m;  // logits considered
        u64 target = 0, above = 0;
        int level = 0;
        if constexpr (BF16) {
            // 16-bit logits have few values: those of a size in [2^-8, 2^8) have a bin each,
            // of how often they come, and the product with the value's weight is the bin's
            // sum.  The smaller ones, between the two signs' bins, are summed one by one.
            // One atomic a logit and no exponential, where the bins below take two and one,
            // and no second pass for what is in the bin: 64 rows of 128257 took 38 us, 62 us
            // with the bins below, which remain for rows with logits out of this range.
            const float lim = kWeights ? fmaxf(lo, m - (kNats + 0.5f) * T) : lo;
            if (!few && fabsf(m) < 256.f && (!kWeights || m - (kNats + 0.5f) * T > -256.f)) {
                u64 small = 0;
                if (kWeights && counted && s.list_n <= kSmall) {
                    // (the bins below lim hold what has no weight)
                    for (int i = tid; i < (int)s.list_n; i += kThreads)
                        small += wide(weight(reinterpret_cast<const float *>(s.seg)[i]));
                } else {
                    for (int i = tid; i < kValues / 4; i += kThreads)
                        reinterpret_cast<uint4 *>(s.hist)[i] = make_uint4(0, 0, 0, 0);
                    __syncthreads();
                    for (int g = tid; g < groups; g += kThreads) {
                        float l[4];
                        load4(g, l);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t at = value_bin(l[i]);
                            if (l[i] >= lim) {
                                if (at < kValues) atomicAdd(s.hist + at, 1u);
                                else if (fabsf(l[i]) < 1.f) small += kWeights ? wide(weight(l[i])) : 1;
                            }
                        }
                    }
                }
                const u64 small_all = [&] {  // the CTA's
                    u64 sum;
                    scan(small, sum);
                    return sum;
                }();
                const int per_cta = kValues / C, per_thread = max(1, per_cta / kThreads);
                const uint32_t *bins = send_bins(kValues, per_cta, per_cta);
                const int ts = exchange(small_all, 0, 0);  // (and the bins are there)
                small = 0;
                for (int r = 0; r < C; ++r) small += s.xch[ts][0][r];
                // as the linear bins below: 1 / C of the bins to a CTA, up to four a thread
                u64 v[4] = {0, 0, 0, 0}, own = 0;
                uint32_t n[4] = {0, 0, 0, 0};
                const int i0 = rank * per_cta + tid * per_thread;
                if (tid * per_thread < per_cta) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i >= per_thread) break;
                        for (int r = 0; r < C; ++r) n[i] += bins[r * per_cta + tid * per_thread + i];
                        if (n[i]) v[i] = kWeights ? n[i] * wide(weight(value_of(i0 + i))) : n[i];
                        own += v[i];
                    }
                }
                u64 total;
                u64 before = scan(own, total);
                {
                    const int t = exchange(total, 0, 0);
                    total = small;
                    for (int r = 0; r < C; ++r) {
                        if (r < rank) before += s.xch[t][0][r];
                        total += s.xch[t][0][r];
                    }
                }
                if (i0 >= kValues / 2) before += small;
                if (tid == 0) {
                    s.target = target_of(total);
                    s.bin = -1;
                }
                __syncthreads();
                target = s.target;
                if (kWeights && target > total) return false;  // (the same in every CTA)
                if (target <= total) {
                    sync();  // no CTA's s.bin is set from here on
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (n[i] && before < target && before + v[i] >= target)
                            for (int r = 0; r < C; ++r) {
                                Shared *o = of(r);
                                o->bin = i0 + i;
                                o->above = before;
                                o->equal = n[i];
                            }
                        // the small ones lie before the first bin of the negative values
                        if (i0 + i == kValues / 2 && i < per_thread && before - small < target && before >= target)
                            for (int r = 0; r < C; ++r) of(r)->above = before - small;
                        before += v[i];
                    }
                    sync();
                    if (s.bin >= 0) {
                        if (tid == 0) s.cut = key_of(value_of(s.bin));
                        __syncthreads();
                        return true;
                    }
                    // among the small ones: by their keys
                    above = s.above;
                    hi = value_of(kValues / 2 - 1) * (1.f - 0x1p-8f);
                    lo = fmaxf(lo, -hi);
                    level = 1;
                    sync();  // bins may be cleared again
                }  // else (a count that goes past those bins) all logits, below
            }
        }
        for (;; ++level) {
            const uint32_t k_hi = key_of(hi);
            const int key_shift = level ? max(0, 21 - __clz(k_hi - key_of(lo))) : 0;
            // Bins in order of falling logits: of the first level by a linear map
            // (adding 2^23 rounds to the whole number), of later ones by key.
            auto linear = [&](float l) { return fminf((m - l) * per_logit, (float)(kBins - 1)) + 8388608.f; };
            auto bin_of = [&](float l) {
                return level ? (k_hi - key_of(l)) >> key_shift
                             : __float_as_uint(linear(l)) & (2 * kBins - 1);
            };
            for (int i = tid; i < kBins / 2; i += kThreads)
                reinterpret_cast<uint4 *>(s.hist)[i] = make_uint4(0, 0, 0, 0);
            if (tid == 0) {
                s.list_n = 0;
                s.key_min = kOne;
                s.key_max = 0;
            }
            __syncthreads();
            // (the first level's code is apart: every logit of the row goes through it, at
            // the pace of the integer pipe and of the shared-memory atomics, 3.4 wavefronts
            // each.  The sum's bits less those of 2^23 are the bin.)
            auto add = [&](uint32_t *at, uint32_t code) {
                if (kWeights) {
                    uint32_t low = code & 0xffffu, high = code >> 16;
                    if (code == kOne) {
                        low = 0;
                        high = 0x10000u;
                    }
                    atomicAdd(at, low);
                    atomicAdd(at + kBins, high);
                } else {
                    atomicAdd(at, 1u);
                }
            };
            if (level == 0) {
                for (int g = tid; g - lane < groups; g += kThreads) {
                    float l[4];
                    load4(g, l);
                    if (!__any_sync(kFull, fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= lo)) continue;
                    float e[4] = {0.f, 0.f, 0.f, 0.f};
                    if (kWeights) es_of(l, e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t bin = __float_as_uint(linear(l[i])) - 0x4b000000u;
                        if (l[i] >= lo) add(s.hist + bin, code_of(e[i]));
                    }
                }
            } else {
                for (int g = tid; g < groups; g += kThreads) {
                    float l[4];
                    load4(g, l);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (l[i] >= lo && l[i] <= hi)
                            add(s.hist + bin_of(l[i]), kWeights ? weight(l[i]) : 0u);
                }
            }
            // The bins' sums over the cluster: each CTA takes 1 / C of the bins,
            // one or two a thread in order, and tells the others its total.
            const int per_cta = kBins / C, per_thread = max(1, per_cta / kThreads);
            if (C > 1) __syncthreads();
            const uint32_t *bins = send_bins(kWeights ? 2 * kBins : kBins, per_cta, 2 * per_cta);
            sync();
            u64 v[2] = {0, 0};
            if (tid * per_thread < per_cta) {
                const int i0 = rank * per_cta + tid * per_thread;
                if (C == 1) {
                    const uint2 low = *reinterpret_cast<const uint2 *>(s.hist + i0);
                    const uint2 high = *reinterpret_cast<const uint2 *>(s.hist + kBins + i0);
                    v[0] = low.x + ((u64)high.x << 16);
                    v[1] = low.y + ((u64)high.y << 16);
                } else {  // (C >= 2: one bin a thread)
                    for (int r = 0; r < C; ++r) {
                        v[0] += bins[2 * r * per_cta + tid];
                        if (kWeights) v[0] += (u64)bins[(2 * r + 1) * per_cta + tid] << 16;
                    }
                }
            }
            u64 total;
            u64 before = scan(v[0] + v[1], total);
            if (C > 1) {
                const int t = exchange(total, 0, 0);
                total = 0;
                for (int r = 0; r < C; ++r) {
                    if (r < rank) before += s.xch[t][0][r];
                    total += s.xch[t][0][r];
                }
            }
            if (level == 0) {
                if (tid == 0) s.target = target_of(total);
                __syncthreads();
                target = s.target;
                if (target > total) return false;  // (the same in every CTA)
            }
            before += above;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (before < target && before + v[i] >= target)
                    for (int r = 0; r < C; ++r) {
                        Shared *o = of(r);
                        o->bin = rank * per_cta + tid * per_thread + i;
                        o->above = before;
                    }
                before += v[i];
            }
            sync();
            const uint32_t bin = (uint32_t)s.bin;
            above = s.above;
            // what is in the bin
            uint32_t kmin = kOne, kmax = 0, in_bin_n = 0;
            const float in_bin = (float)bin + 8388608.f;
            for (int g = tid; g < groups; g += kThreads) {
                float l[4];
                load4(g, l);
                uint32_t in = 0;
                if (level == 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        in |= (uint32_t)(linear(l[i]) == in_bin && l[i] >= lo) << i;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        in |= (uint32_t)(l[i] >= lo && l[i] <= hi && bin_of(l[i]) == bin) << i;
                }
                if (!in) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!(in >> i & 1)) continue;
                    const uint32_t key = key_of(l[i]);
                    kmin = min(kmin, key);
                    kmax = max(kmax, key);
                    if (BF16 && !few) {  // mostly many of one key: counted, not listed
                        ++in_bin_n;
                    } else {
                        const uint32_t n = atomicAdd(&s.list_n, 1u);
                        if (n < kList) s.list[n] = key;
                    }
                }
            }
            if (BF16 && !few) {
                in_bin_n = __reduce_add_sync(kFull, in_bin_n);
                if (lane == 0 && in_bin_n) atomicAdd(&s.list_n, in_bin_n);
            }
            kmin = __reduce_min_sync(kFull, kmin);
            kmax = __reduce_max_sync(kFull, kmax);
            if (lane == 0 && kmax) {
                atomicMin(&s.key_min, kmin);
                atomicMax(&s.key_max, kmax);
            }
            __syncthreads();
            const int t = exchange(s.list_n, s.key_min, s.key_max);
            u64 n = 0;
            for (int r = 0; r < C; ++r) {
                n += s.xch[t][0][r];
                kmin = min(kmin, (uint32_t)s.xch[t][1][r]);
                kmax = max(kmax, (uint32_t)s.xch[t][2][r]);
            }
            if (kmin == kmax) {  // one key
                if (tid == 0) {
                    s.cut = kmin;
                    s.above = above;
                    s.equal = n;
                }
                break;
            }
            if (n <= kList && !(BF16 && !few)) {
                if (tid < (int)n) {
                    int r = 0, at = tid;
                    while (at >= (int)s.xch[t][0][r]) at -= (int)s.xch[t][0][r++];
                    const uint32_t key = of(r)->list[at];
                    s.all[tid] = make_uint2(key, kWeights ? weight(logit_of(key)) : 1u);
                }
                __syncthreads();
                if (tid - lane < 4 * (int)n) {  // four threads to an entry, each every fourth
                    const uint32_t key = s.all[min(tid >> 2, (int)n - 1)].x;
                    u64 more = 0, equal = 0, count = 0;
#pragma unroll 4
                    for (int i = tid & 3; i < (int)n; i += 4) {
                        const uint2 o = s.all[i];
                        const u64 w = wide(o.y);
                        if (o.x > key) more += w;
                        if (o.x == key) {
                            equal += w;
                            ++count;
                        }
                    }
#pragma unroll
                    for (int d = 1; d < 4; d <<= 1) {
                        more += __shfl_xor_sync(kFull, more, d);
                        equal += __shfl_xor_sync(kFull, equal, d);
                        count += __shfl_xor_sync(kFull, count, d);
                    }
                    // threads of equal keys write the same
                    if (above + more < target && above + more + equal >= target) {
                        s.cut = key;
                        s.above = above + more;
                        s.equal = count;
                    }
                }
                break;
            }
            lo = logit_of(kmin);
            hi = logit_of(kmax);
            sync();  // lists and bins may be written again
        }
        sync();
        return true;
    };

    // ---- kept: keys > cut, and the first `ties` of those equal to it ----
    uint32_t cut = kKeyNone;
    u64 ties = 0, equal = 0;  // of `equal` tokens equal to the cut `ties` stay
    if (k < a.vocab) {
        const float span = m - low;
        const float per_logit = span > 0.f && span < 3e38f ? (kBins - 1) / span : 0.f;
        if (search(std::false_type(), low, per_logit, [&](u64) { return (u64)k; })) {
            cut = s.cut;
            ties = (u64)k - s.above;
            equal = s.equal;
        }  // else fewer than k tokens are above -inf: all stay
    }
    if (p < 1.f) {
        const u64 w_cut = ties ? wide(weight(logit_of(cut))) : 0;
        const bool here = search(std::true_type(), logit_of(cut + 1), (kBins - 1) / kNats / T, [&](u64 total) {
            s.sum = total;
            const u64 all = total + ties * w_cut;
            const double want = ceil((double)p * (double)all);
            const u64 target = want < 1.0 ? 1 : (u64)want;
            return target < all ? target : all;
        });
        if (here) {
            cut = s.cut;
            const u64 w = wide(weight(logit_of(cut)));
            ties = (s.target - s.above + w - 1) / w;
            equal = s.equal;
        } else {  // it ends among the tokens equal to the top-k cut
            ties = (s.target - s.sum + w_cut - 1) / w_cut;
        }
    }
    // Of the tokens equal to the cut the first `ties` in index order stay.  Where
    // that is not all of them, they are counted apart, and what stays of a segment's
    // is added when the counts before it are known.
    const float at_cut = logit_of(cut);
    const bool part = ties && ties < equal;
    const float from = ties && !part ? at_cut : logit_of(cut + 1);
    // codes of a group's kept weights (those equal to the cut aside where `part`)
    auto kept = [&](const float (&l)[4], uint32_t (&w)[4]) {
        float e[4];
        es_of(l, e);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = l[i] >= from ? code_of(e[i]) : 0u;
        if (floor_p > 0.f)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!(e[i] >= floor_p)) w[i] = 0;
    };
    uint32_t code_cut = 0;  // of a token equal to the cut
    if (part) {
        const float l[4] = {at_cut, at_cut, at_cut, at_cut};
        float e[4];
        es_of(l, e);
        code_cut = floor_p > 0.f && !(e[0] >= floor_p) ? 0u : code_of(e[0]);
    }

    // ---- the token at which the running sum in index order passes r ----
    const int segs = (groups + 31) / 32;
    for (int g0 = warp * 32; g0 < groups; g0 += kThreads) {  // segments of 32 groups
        float l[4];
        load4(g0 + lane, l);
        const float most = fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3]));
        u64 sum = 0;
        if (__any_sync(kFull, most >= from)) {
            uint32_t w[4];
            kept(l, w);
            sum = (u64)w[0] + w[1] + w[2] + w[3];
            // the few weights of 2^32, which the code has as one less
            if (max(max(w[0], w[1]), max(w[2], w[3])) == kOne)
                sum += (w[0] == kOne) + (w[1] == kOne) + (w[2] == kOne) + (w[3] == kOne);
            sum = __reduce_add_sync(kFull, (uint32_t)sum & 0xfffffu) +
                  ((u64)__reduce_add_sync(kFull, (uint32_t)(sum >> 20)) << 20);
        }
        uint32_t n = 0;
        if (part) {
#pragma unroll
            for (int i = 0; i < 4; ++i) n += l[i] == at_cut;
            n = __reduce_add_sync(kFull, n);
        }
        if (lane == 0) {
            s.seg[g0 / 32] = sum;
            s.n_seg[g0 / 32] = n;
        }
    }
    __syncthreads();
    u64 seg = tid < segs ? s.seg[tid] : 0, ties_before = 0;
    if (part) {
        const u64 n = tid < segs ? s.n_seg[tid] : 0;
        u64 here, before = 0;
        ties_before = scan(n, here);
        const int t = exchange(here, 0, 0);
        for (int r = 0; r < rank; ++r) before += s.xch[t][0][r];
        ties_before += before;
        seg += (ties > ties_before ? min(n, ties - ties_before) : 0) * wide(code_cut);
    }
    u64 mine_all;
    const u64 seg_before = scan(seg, mine_all);
    u64 total = 0, before = 0;
    {
        const int t = exchange(mine_all, 0, 0);
        for (int r = 0; r < C; ++r) {
            if (r < rank) before += s.xch[t][0][r];
            total += s.xch[t][0][r];
        }
    }
    if (tid == 0) {
        float u = a.uniforms[row];
        if (!(u >= 0.f)) u = 0.f;
        const u64 r = (u64)((double)u * (double)total);
        s.target = r < total ? r : total - 1;
    }
    __syncthreads();
    u64 r = s.target;
    if (r < before || r >= before + mine_all) return;  // another CTA of the cluster has it
    r -= before;
    if (seg_before <= r && r < seg_before + seg) {
        s.where = tid;
        s.above = seg_before;
        s.equal = ties_before;
    }
    __syncthreads();
    if (warp != 0) return;
    r -= s.above;
    const int g = s.where * 32 + lane;
    float l[4];
    load4(g, l);
    uint32_t code[4];
    kept(l, code);
    if (part) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += l[i] == at_cut;
        u64 place = s.equal + warp_scan(n) - n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (l[i] == at_cut && place++ < ties) code[i] = code_cut;
    }
    u64 inc = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) inc += wide(code[i]);
    u64 at = warp_scan(inc) - inc;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u64 w = wide(code[i]);
        if (at <= r && r < at + w) {
            a.tokens[row] = few ? s.cand_at[4 * g + i] : base + 4 * g + i - shift;
            accept_one(a, row, few ? s.cand_at[4 * g + i] : base + 4 * g + i - shift);
            if (a.logprobs) {
                const float z = l[i] == m ? 0.f : (l[i] - m) / T;
                a.logprobs[row] = z - logf((float)((double)total * (1.0 / 4294967296.0)));
            }
        }
        at += w;
    }
}

// ---- longer rows --------------------------------------------------------------------
// Rows of more than kMaxRowCtas * kMaxSlice logits (360,416 in binary32, 524,256 in
// bf16): one CTA per row, which reads the row (from L2 at best) for every step.
// Kept simple, and slow: 5.1 ms for one row of 400,009 where a cluster takes 44 us
// for 360,000.
template <bool BF16>
__global__ void __launch_bounds__(kLongThreads) long_row_kernel(const SampleArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ u64 sums[32];
    __shared__ u64 hist[256];
    __shared__ u64 s_sum;
    __shared__ int s_bin;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const size_t row = blockIdx.x;
    const int b = (int)(row / a.W), V = a.vocab;
    auto key = [&](int i) {
        const size_t at = row * a.row_stride + i;
        return key_of(BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(a.logits)[at] << 16)
                           : static_cast<const float *>(a.logits)[at]);
    };
    float T = a.sampling.temperature ? a.sampling.temperature[b] : 1.f;
    long long k = a.sampling.top_k ? a.sampling.top_k[b] : 0;
    const float p = a.sampling.top_p ? a.sampling.top_p[b] : 1.f;
    float floor_p = a.sampling.min_p ? a.sampling.min_p[b] : 0.f;
    floor_p = floor_p > 0.f ? fminf(floor_p, 1.f) : 0.f;  // NaN: none
    if (!(T > 0.f)) {
        T = 1.f;
        k = 1;
    }
    T = fminf(T, 3.4028234e38f);
    if (k <= 0 || k > V) k = V;

    auto add = [](u64 x, u64 y) { return x + y; };
    uint32_t mine = 0;
    for (int i = tid; i < V; i += kLongThreads) mine = max(mine, key(i));
    const uint32_t top =
        (uint32_t)block_reduce<u64>(mine, sums, [](u64 x, u64 y) { return x > y ? x : y; });
    if (top <= kKeyNone) {
        if (tid == 0) {
            accept_one(a, row, -1);
            a.tokens[row] = -1;
            if (a.logprobs) a.logprobs[row] = -INFINITY;
        }
        return;
    }
    const float m = logit_of(top);

    // The largest key t for which f over keys > t sums to less than the
    // target; above is that sum.  Keys are searched byte by byte.
    auto threshold = [&](u64 target, uint32_t least, auto f, u64 &above) {
        uint32_t t = 0;
        above = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += kLongThreads) {
                const uint32_t x = key(i);
                if (x >= least && (shift == 24 || (x >> (shift + 8)) == (t >> (shift + 8))))
                    atomicAdd(&hist[(x >> shift) & 255], f(x));
            }
            __syncthreads();
            if (tid == 0) {
                int c = 255;
                while (c > 0 && above + hist[c] < target) above += hist[c--];
                s_bin = c;
                s_sum = above;
            }
            __syncthreads();
            t |= (uint32_t)s_bin << shift;
            above = s_sum;
            __syncthreads();
        }
        return t;
    };
    auto count_equal = [&](uint32_t t) {
        u64 n = 0;
        for (int i = tid; i < V; i += kLongThreads) n += key(i) == t;
        return block_reduce<u64>(n, sums, add);
    };

    // kept: keys > cut, and the first `ties` of those equal to it
    uint32_t cut = 0;
    u64 ties = (u64)V;
    if (k < V) {
        u64 above;
        cut = threshold((u64)k, 0u, [](uint32_t) { return (u64)1; }, above);
        ties = (u64)k - above;
    }
    auto weight = [&](uint32_t x) { return w_of(e_of(x, top, m, T)); };
    if (p < 1.f) {
        u64 s = 0;
        for (int i = tid; i < V; i += kLongThreads) {
            const uint32_t x = key(i);
            if (x > cut) s += weight(x);
        }
        s = block_reduce<u64>(s, sums, add);
        const u64 s_above = s;
        const u64 equal = min(ties, k < V ? count_equal(cut) : (u64)0);
        s += equal * (k < V ? weight(cut) : 0);
        const double want = ceil((double)p * (double)s);
        u64 target = want < 1.0 ? 1 : (u64)want;
        if (target > s) target = s;
        if (k < V && target > s_above) {  // ends among the tokens equal to the top-k cut
            ties = (target - s_above + weight(cut) - 1) / weight(cut);
        } else {
            u64 above;
            cut = threshold(target, cut + (k < V ? 1u : 0u), weight, above);
            ties = (target - above + weight(cut) - 1) / weight(cut);
        }
    }
    // the index of the last kept token equal to the cut
    __shared__ int s_last;
    if (tid == 0) s_last = V;
    __syncthreads();
    if (count_equal(cut) > ties) {
        u64 seen = 0;
        for (int i0 = 0; i0 < V; i0 += kLongThreads) {
            const int i = i0 + tid;
            const bool eq = i < V && key(i) == cut;
            const unsigned bal = __ballot_sync(kFull, eq);
            if (lane == 0) sums[warp] = __popc(bal);
            __syncthreads();
            u64 before = seen, all = 0;
            for (int w = 0; w < 32; ++w) {
                if (w < warp) before += sums[w];
                all += sums[w];
            }
            if (eq && before + __popc(bal & ((1u << lane) - 1)) == ties - 1) s_last = i;
            seen += all;
            __syncthreads();
            if (seen >= ties) break;
        }
    }
    __syncthreads();
    const int last = s_last;
    auto kept = [&](int i) -> u64 {
        const uint32_t x = key(i);
        if (x < cut || (x == cut && i > last)) return 0;
        const float e = e_of(x, top, m, T);
        return floor_p > 0.f && !(e >= floor_p) ? 0 : w_of(e);
    };
    u64 total = 0;
    for (int i = tid; i < V; i += kLongThreads) total += kept(i);
    total = block_reduce<u64>(total, sums, add);
    float u = a.uniforms[row];
    if (!(u >= 0.f)) u = 0.f;
    u64 r = (u64)((double)u * (double)total);
    if (r > total - 1) r = total - 1;
    // the token at which the running sum in index order passes r
    __shared__ int s_token;
    u64 seen = 0;
    for (int i0 = 0; i0 < V; i0 += kLongThreads) {
        const int i = i0 + tid;
        const u64 w = i < V ? kept(i) : 0;
        u64 x = w;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const u64 y = __shfl_up_sync(kFull, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) sums[warp] = x;
        __syncthreads();
        u64 before = seen, all = 0;
        for (int v = 0; v < 32; ++v) {
            if (v < warp) before += sums[v];
            all += sums[v];
        }
        if (before + x > r && before + x - w <= r) s_token = i;
        seen += all;
        __syncthreads();
        if (seen > r) break;
    }
    if (tid == 0) {
        const int t = s_token;
        accept_one(a, row, t);
        a.tokens[row] = t;
        if (a.logprobs) {
            const float l = logit_of(key(t));
            const float z = key(t) == top ? 0.f : (l - m) / T;
            a.logprobs[row] = z - logf((float)((double)total * (1.0 / 4294967296.0)));
        }
    }
}

// accepted[b] = first i with draft[b][i] != target_ids[b][i] (W if none),
// next_token and committed from it.  One warp per sequence.
__global__ void __launch_bounds__(kScanWarps * 32)
    sample_accept_kernel(const int32_t *__restrict__ target_ids, const int32_t *__restrict__ draft,
                         int B, int W, int32_t *__restrict__ accepted,
                         int32_t *__restrict__ next_token, int32_t *__restrict__ committed) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const long long b = (long long)blockIdx.x * kScanWarps + (threadIdx.x >> 5);
    if (b >= B) return;
    const int32_t *t = target_ids + b * W, *d = draft + b * W;
    int first = W;
    for (int i0 = 0; i0 < W; i0 += 32) {
        const int i = i0 + lane;
        const unsigned m = __ballot_sync(kFull, i < W && (d[i] != t[i] || t[i] < 0));
        if (m) {
            first = i0 + __ffs(m) - 1;
            break;
        }
    }
    if (lane == 0) {
        accepted[b] = first;
        next_token[b] = first < W ? t[first] : d[W - 1];
        if (committed) committed[b] = min(first + 1, W);
    }
}

template <typename... Params, typename... Args>
cudaError_t launch_pdl(void (*kernel)(Params...), dim3 grid, dim3 block, unsigned cluster,
                       size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

template <bool BF16>
cudaError_t sample_launch_t(const SampleArgs &a, cudaStream_t stream) {
    const long long rows = (long long)a.B * a.W;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int sms = attn_grid_size(dev);
    if (sms <= 0) return cudaErrorInvalidDevice;
    // CTAs per row: enough to hold the row, and as many as fill the SMs
    constexpr int kMaxSlice = kSliceBytes<BF16> / (BF16 ? 2 : 4) - 4;  // (with the shift of a first group)
    const int hold = (int)(((long long)a.vocab + kMaxSlice - 1) / kMaxSlice);
    if (hold > kMaxRowCtas)
        return launch_pdl(long_row_kernel<BF16>, dim3((unsigned)rows), dim3(kLongThreads), 1, 0,
                          stream, a);
    int C = 1;  // a power of two: the bins divide by it
    while (C < kMaxRowCtas && (C < hold || (rows * C * 2 <= sms && a.vocab > C * 4 * kThreads)))
        C *= 2;
    const int slice = ((a.vocab + C - 1) / C + 3) / 4 * 4;
    const dim3 grid((unsigned)(rows * C)), block(kThreads);
    size_t smem = (size_t)(slice + 4) * (BF16 ? 2 : 4);  // (a group more where rows begin within one)
    if (C > 1) smem = std::max(smem, 2 * kBins * sizeof(uint32_t));  // (bins may be sent there)
    static std::atomic<bool> configured[64];  // the shared-memory opt-in, once per device
    if (dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(sample_kernel<BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSliceBytes<BF16>);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    return launch_pdl(sample_kernel<BF16>, grid, block, C, smem, stream, a, slice);
}

}  // namespace

cudaError_t sample_launch(const SampleArgs &a, cudaStream_t stream) {
    if ((long long)a.B * a.W == 0) return cudaSuccess;
    return a.bf16 ? sample_launch_t<true>(a, stream) : sample_launch_t<false>(a, stream);
}

cudaError_t sample_accept_launch(SampleArgs a, const int32_t *draft, int32_t *accepted,
                                 int32_t *next_token, int32_t *committed, cudaStream_t stream) {
    if (a.B == 0) return cudaSuccess;
    if (a.W == 1) {  // one kernel: the launch and the dependency cost 3 us
        a.draft = draft;
        a.accepted = accepted;
        a.next_token = next_token;
        a.committed = committed;
        return sample_launch(a, stream);
    }
    const cudaError_t e = sample_launch(a, stream);
    if (e != cudaSuccess) return e;
    return launch_pdl(sample_accept_kernel, dim3((unsigned)((a.B + kScanWarps - 1) / kScanWarps)),
                      dim3(kScanWarps * 32), 1, 0, stream, static_cast<const int32_t *>(a.tokens),
                      draft, a.B, a.W, accepted, next_token, committed);
}

}  // namespace das
