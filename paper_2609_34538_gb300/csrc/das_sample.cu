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
// sample_kernel: a cluster of CTAs holds a row in shared memory, read once (rows that are
// recorded for speculative acceptance are read again instead).  A
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
constexpr int kDrawThreads = 1024;
// Rows that are recorded are not held but read again, from L2: two CTAs of half the threads
// share an SM, and one's waits are the other's time (2 x 128 rows of 32000 and the acceptance, as measured
// when it was chosen: 28.7 us, 40 with the rows held).
constexpr int kRecordThreads = 512;
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
static_assert(kRecordThreads >= kMaxSegs, "a thread has a segment");
constexpr int kSmall = 2 * kMaxSegs;
// exponents past the last bin have weights that round to 0: e^-23 < 2^-33
constexpr float kNats = 23.f;
constexpr uint32_t kOne = 0xffffffffu;  // stands for the weight 2^32

struct alignas(16) Shared {
    float cand[kCand];              // the candidates left by a small top-k,
    int cand_at[kCand];             // in index order
    uint32_t hist[2 * kBins];       // bin i's sum: [i] + 2^16 [kBins + i]; or kValues counts
    u64 scan[32];
    u64 seg[kMaxSegs];
    uint32_t n_seg[kMaxSegs];
    u64 xch[2][3][kMaxRowCtas];  // values of every CTA of the cluster
    uint32_t list[kList];  // the CTA's keys in a bin
    uint2 all[kList];      // the cluster's, with their weights
    uint32_t list_n, key_min, key_max;
    int n_cand;
    uint4 edge[3];  // a recorded part's first and last group, where they are not whole, and padding
    int bin, where;
    uint32_t cut;
    u64 above, target, sum, equal;
};

// Where a row comes from: of two sets of rows, if rows are recorded.
struct Source {
    const void *logits;
    size_t row;
    long long stride;
    const das_sampling *sampling;
    int b;
};
template <bool RECORD>
__device__ __forceinline__ Source source_of(const SampleArgs &a, size_t row) {
    if constexpr (RECORD) {
        const size_t rows = (size_t)a.B * a.W;
        if (row >= rows)
            return {a.second, row - rows, a.second_stride, &a.second_sampling, (int)((row - rows) / a.W)};
    }
    return {a.logits, row, a.row_stride, &a.sampling, (int)(row / a.W)};
}

__device__ __forceinline__ RowRecord record_of(uint32_t top, uint32_t key, int last, float T, float floor, u64 total) {
    return {top, key, last, T, floor, 1.f / (float)((double)total * (1.0 / 4294967296.0)), total};
}

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

// With RECORD rows are not drawn from: what their filters leave is recorded, of the rows of
// a.logits and then of a.second.
template <bool BF16, bool RECORD>
__global__ void __launch_bounds__(RECORD ? kRecordThreads : kDrawThreads, RECORD ? 2 : 1)
    sample_kernel(const SampleArgs a, int slice) {
    constexpr int kThreads = RECORD ? kRecordThreads : kDrawThreads, kWarps = kThreads / 32;
    static_assert(kWarps <= 32, "a warp scans the warps' sums");
    __shared__ Shared s;
    // the CTA's logits in groups of four, padded with -inf (RECORD: bins of other CTAs alone)
    extern __shared__ uint4 held[];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const size_t row = blockIdx.x / C;
    const Source from_row = source_of<RECORD>(a, row);
    const int b = from_row.b;
    const das_sampling &sampling = *from_row.sampling;
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
        const u64 sums = warp_scan(lane < kWarps ? s.scan[lane] : 0);  // by every warp for itself
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

    float T = sampling.temperature ? sampling.temperature[b] : 1.f;
    long long k = sampling.top_k ? sampling.top_k[b] : 0;
    const float p = sampling.top_p ? sampling.top_p[b] : 1.f;
    float floor_p = sampling.min_p ? sampling.min_p[b] : 0.f;
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
    const Elem *src = static_cast<const Elem *>(from_row.logits) + from_row.row * (size_t)from_row.stride + base;
    const int shift = (int)(reinterpret_cast<uintptr_t>(src) / sizeof(Elem) & 3);
    int groups = len ? (len + shift + 3) / 4 : 0;
    bool few = false;  // whether the candidates alone are left
    float mine = -INFINITY;
    src -= shift;
    bool infinite = false;
    using Vec = std::conditional_t<BF16, uint2, float4>;
    auto whole = [&](int g) { return 4 * g >= shift && 4 * g + 4 <= len + shift; };
    auto vector_of = [&](int g) {
        const Vec *at = reinterpret_cast<const Vec *>(src) + g;
        return RECORD ? *at : __ldcs(at);
    };
    auto part_of = [&](int g) {  // a group that is not whole, padded
        Elem e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) e[i] = 0xff80;
            else e[i] = -INFINITY;
            if (4 * g + i >= shift && 4 * g + i < len + shift) e[i] = src[4 * g + i];
        }
        if constexpr (BF16) return make_uint2(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16);
        else return make_float4(e[0], e[1], e[2], e[3]);
    };
    if constexpr (RECORD) {  // (out of the loops, whose code would be three times as long)
        if (tid < 3) reinterpret_cast<Vec &>(s.edge[tid]) = part_of(tid == 0 ? 0 : groups - 2 + tid);
        __syncthreads();
    }
    auto split = [](const Vec &u, float (&f)[4]) {  // as they come
        if constexpr (BF16) {
            f[0] = __uint_as_float(u.x << 16);
            f[1] = __uint_as_float(u.x & 0xffff0000u);
            f[2] = __uint_as_float(u.y << 16);
            f[3] = __uint_as_float(u.y & 0xffff0000u);
        } else {
            f[0] = u.x;
            f[1] = u.y;
            f[2] = u.z;
            f[3] = u.w;
        }
    };
    auto unpack = [&](const Vec &u, float (&f)[4]) {
        split(u, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = f[i] == f[i] ? f[i] + 0.f : -INFINITY;
        if (infinite)  // (those have weight, and the same)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = f[i] == INFINITY ? 0.f : -INFINITY;
    };
    // f(g, vector) of kBatch groups from g on, `step` apart: all loads before the first is used
    auto batch = [&](auto groups_at_once, int g, int step, int end, auto f) {
        constexpr int kBatch = decltype(groups_at_once)::value;
        Vec u[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int at = g + j * step;
            if (whole(at)) u[j] = vector_of(at);
            else u[j] = reinterpret_cast<const Vec &>(s.edge[at >= groups ? 2 : at > 0]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (g + j * step - lane >= end) return;  // the same in the warp
            f(g + j * step, u[j]);
        }
    };
    // f(g, vector) of each group, those of a warp together
    auto sweep = [&](auto f) {
        for (int g = tid; g - lane < groups; g += 4 * kThreads)
            batch(std::integral_constant<int, 4>(), g, kThreads, groups, f);
    };
    auto first_seen = [&](const float (&f)[4]) {
        if (!(RECORD && BF16)) mine = fmaxf(fmaxf(mine, fmaxf(f[0], f[1])), fmaxf(f[2], f[3]));
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
    };
    if constexpr (RECORD) {
        // (fmaxf and the bins take no NaN; key_of takes -0 for 0)
        uint32_t most = 0xff80ff80u;  // bf16 pairs
        sweep([&](int, const Vec &u) {
            if constexpr (BF16)
                asm("{\n .reg .b32 t;\n max.bf16x2 t, %1, %2;\n max.bf16x2 %0, %0, t;\n}" : "+r"(most) : "r"(u.x), "r"(u.y));
            float f[4];
            split(u, f);
            first_seen(f);
        });
        if (BF16) mine = fmaxf(__uint_as_float(most << 16), __uint_as_float(most & 0xffff0000u));
    }
#pragma unroll 4
    for (int g = tid; !RECORD && g < groups; g += kThreads) {
        float f[4];
        unpack(whole(g) ? vector_of(g) : part_of(g), f);
        first_seen(f);
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
        } else if (RECORD && !few) {
            unpack(whole(g) ? vector_of(g) : part_of(g), l);
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
    // With the 16 warps of a recorded row n is one more: 395 candidates, and 512 or fewer of
    // 200 rows in all, where one more row in 200 had more with n as above.
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
        const long long kc = (k + C - 1) / C, n = min((kc + kWarps - 1) / kWarps + (RECORD ? 2 : 1), 32ll);
        const bool bound = k < a.vocab && kc <= n * kWarps;
        if (bound) {
            const uint32_t nth = __shfl_sync(kFull, sorted32(key), (int)n - 1);
            if (lane == 0) s.list[warp] = nth;
        }
        if (lane == 0) atomicMax(&s.key_max, top);
        __syncthreads();
        uint32_t here = kKeyNone;
        if (bound && warp == 0)
            here = __shfl_sync(kFull, sorted32(lane < kWarps ? s.list[lane] : 0u), (int)((kc + n - 1) / n) - 1);
        const int t = exchange(s.key_max, here, 0);  // (by warp 0)
        uint32_t most = 0, least = kOne;
        for (int r = 0; r < C; ++r) {
            most = max(most, (uint32_t)s.xch[t][0][r]);
            least = min(least, (uint32_t)s.xch[t][1][r]);
        }
        if (most <= kKeyNone) {  // the same in every CTA
            if (rank == 0 && tid == 0) {
                if constexpr (RECORD) {
                    a.records[row] = RowRecord{};
                } else {
                    accept_one(a, row, -1);
                    a.tokens[row] = -1;
                    if (a.logprobs) a.logprobs[row] = -INFINITY;
                }
            }
            return;
        }
        m = logit_of(most);
        low = logit_of(max(least, kKeyNone + 1));
    }
    infinite = m == INFINITY;
    const uint32_t top = key_of(m);
    // (a key that load4 gives is one of the row, but for the infinite logits')
    auto record = [&](uint32_t cut, int last, u64 total) {
        if (infinite && cut == key_of(0.f)) cut = top;
        a.records[row] = record_of(top, cut, last, T, floor_p, total);
    };
    if (infinite) {  // the infinite ones alone have weight, and the same
        if constexpr (!RECORD)
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
        if (tid < n)  // (a record's candidates are in no order)
            x = (u64)key_of(s.cand[tid]) << 32 | (RECORD ? ~(uint32_t)s.cand_at[tid] : (uint32_t)(kThreads - 1 - tid));
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
        bool in = mine_in;
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
            if (before >= min(s.target, all)) {
                code = 0;
                in = false;
            }
        }
        in = in && (floor_p <= 0.f || e[0] >= floor_p);
        if (floor_p > 0.f && !(e[0] >= floor_p)) code = 0;
        if constexpr (RECORD) {
            // what is kept is the first of the sorted ones, though the last may have no weight
            u64 total;
            scan(wide(code), total);
            const int n_kept = __syncthreads_count(in);
            if (tid == n_kept - 1) record((uint32_t)(x >> 32), (int)~(uint32_t)x, total);
            return;
        }
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

    // ---- a small top-k leaves few candidates: those not below `low` ----
    int n_cand = 0;
    if constexpr (RECORD) {
        // (as they come: they are sorted by their indexes too, or what is found needs no order)
        if (k < a.vocab && k <= kCand / 4) {
            const float least = infinite ? INFINITY : low;
            sweep([&](int g, const Vec &u) {
                float l[4];
                split(u, l);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (l[i] >= least) {
                        const uint32_t n = atomicAdd(&s.list_n, 1u);
                        if (n >= kCand) continue;
                        s.cand[n] = infinite ? 0.f : l[i] + 0.f;
                        s.cand_at[n] = base + 4 * g + i - shift;
                    }
            });
            __syncthreads();
            n_cand = (int)s.list_n;
            const int t = exchange(n_cand, 0, 0);
            bool fit = true;
            int n_row = 0, n_before = 0;
            for (int r = 0; r < C; ++r) {
                const int n = (int)min(s.xch[t][0][r], (u64)kCand + 1);
                fit = fit && n <= kCand;
                n_row += n;
                if (r < rank) n_before += n;
            }
            if (fit && n_row <= kThreads) {
                if (C > 1) {
                    Shared *const to = of(0);
                    for (int i = tid; rank > 0 && i < n_cand; i += kThreads) {
                        to->cand[n_before + i] = s.cand[i];
                        to->cand_at[n_before + i] = s.cand_at[i];
                    }
                    sync();
                }
                if (rank == 0) draw_sorted(n_row);
                return;
            }
            if (fit) {
                few = true;
                groups = (n_cand + 3) / 4;
                if (tid < 4 * groups - n_cand) s.cand[n_cand + tid] = -INFINITY;
                if (tid == 0) s.n_cand = n_cand;
            }
            sync();
        }
    } else if (k < a.vocab && k <= kCand / 4) {
        // In index order: four bits of each group of a thread say which; their numbers, in eight bits of
        // a word per round of groups, are summed over the warp for four rounds at once.
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
        for (int i = tid; 4 * i < words; i += kThreads) {
            const int row = stride > per_cta ? 4 * i / kBins : 0, bin = 4 * i - row * kBins;
            const int r = bin / per_cta, off = bin - r * per_cta;
            uint32_t *const there = cluster.map_shared_rank(place, r);
            *reinterpret_cast<uint4 *>(there + rank * stride + row * per_cta + off) =
                reinterpret_cast<const uint4 *>(s.hist)[i];
        }
        return place;
    };
    static_assert(sizeof s.cand + sizeof s.cand_at >= sizeof s.hist && kValues == 2 * kBins &&
                  offsetof(Shared, cand_at) == sizeof s.cand, "bins sent");

    // f(g, logits) of each group of the row, or of the candidates if they are in use
    auto each_group = [&](auto f) {
        if (RECORD && !few) {
            sweep([&](int g, const Vec &u) {
                float l[4];
                unpack(u, l);
                f(g, l);
            });
        } else {
            for (int g = tid; g - lane < groups; g += kThreads) {
                float l[4];
                load4(g, l);
                f(g, l);
            }
        }
    };

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
                    each_group([&](int, const float (&l)[4]) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t at = value_bin(l[i]);
                            if (l[i] >= lim) {
                                if (at < kValues) atomicAdd(s.hist + at, 1u);
                                else if (fabsf(l[i]) < 1.f) small += kWeights ? wide(weight(l[i])) : 1;
                            }
                        }
                    });
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
                // as the linear bins below: 1 / C of the bins to a CTA, some a thread
                // (not unrolled, and the bins of the thread that has the threshold added up again: code that is run
                // once costs its fetching)
                const int i0 = rank * per_cta + tid * per_thread;
                const bool has = tid * per_thread < per_cta;
                auto bin_sum = [&](int i, uint32_t &n) -> u64 {
                    n = 0;
                    for (int r = 0; r < C; ++r) n += bins[r * per_cta + tid * per_thread + i];
                    return !n ? 0 : kWeights ? n * wide(weight(value_of(i0 + i))) : n;
                };
                u64 own = 0;
                uint32_t n;
#pragma unroll 1
                for (int i = 0; has && i < per_thread; ++i) own += bin_sum(i, n);
                u64 total;
                u64 before = scan(own, total);
                {
                    if (tid == 0) s.bin = -1;
                    const int t = exchange(total, 0, 0);  // (no CTA's s.bin is set from here on)
                    total = small;
                    for (int r = 0; r < C; ++r) {
                        if (r < rank) before += s.xch[t][0][r];
                        total += s.xch[t][0][r];
                    }
                }
                if (i0 >= kValues / 2) before += small;
                if (tid == 0) s.target = target_of(total);
                __syncthreads();
                target = s.target;
                if (kWeights && target > total) return false;  // (the same in every CTA)
                if (target <= total) {
                    if (has && before < target && before + own >= target)
#pragma unroll 1
                        for (int i = 0; i < per_thread; ++i) {
                            const u64 v = bin_sum(i, n);
                            if (n && before + v >= target) {
                                for (int r = 0; r < C; ++r) {
                                    Shared *o = of(r);
                                    o->bin = i0 + i;
                                    o->above = before;
                                    o->equal = n;
                                }
                                break;
                            }
                            before += v;
                        }
                    // the small ones lie before the first bin of the negative values
                    else if (has && i0 == kValues / 2 && before - small < target && before >= target)
                        for (int r = 0; r < C; ++r) of(r)->above = before - small;
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
                each_group([&](int, const float (&l)[4]) {
                    if (!__any_sync(kFull, fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= lo)) return;
                    float e[4] = {0.f, 0.f, 0.f, 0.f};
                    if (kWeights) es_of(l, e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t bin = __float_as_uint(linear(l[i])) - 0x4b000000u;
                        if (l[i] >= lo) add(s.hist + bin, code_of(e[i]));
                    }
                });
            } else {
                each_group([&](int, const float (&l)[4]) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (l[i] >= lo && l[i] <= hi)
                            add(s.hist + bin_of(l[i]), kWeights ? weight(l[i]) : 0u);
                });
            }
            // The bins' sums over the cluster: each CTA takes 1 / C of the bins,
            // some a thread in order, and tells the others its total.
            const int per_cta = kBins / C, per_thread = max(1, per_cta / kThreads);
            if (C > 1) __syncthreads();
            const uint32_t *bins = send_bins(kWeights ? 2 * kBins : kBins, per_cta, 2 * per_cta);
            sync();
            auto bin_sum = [&](int at) -> u64 {
                if (C == 1) return s.hist[at] + ((u64)s.hist[kBins + at] << 16);
                u64 v = 0;
                for (int r = 0; r < C; ++r) {
                    v += bins[2 * r * per_cta + at];
                    if (kWeights) v += (u64)bins[(2 * r + 1) * per_cta + at] << 16;
                }
                return v;
            };
            u64 own = 0;
#pragma unroll 1
            for (int at = tid * per_thread, i = 0; i < per_thread && at < per_cta; ++i, ++at) own += bin_sum(at);
            u64 total;
            u64 before = scan(own, total);
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
            if (before < target && before + own >= target)
#pragma unroll 1
                for (int at = tid * per_thread;; ++at) {
                    const u64 v = bin_sum(at);
                    if (before + v >= target) {
                        for (int r = 0; r < C; ++r) {
                            Shared *o = of(r);
                            o->bin = rank * per_cta + at;
                            o->above = before;
                        }
                        break;
                    }
                    before += v;
                }
            sync();
            const uint32_t bin = (uint32_t)s.bin;
            above = s.above;
            // what is in the bin
            uint32_t kmin = kOne, kmax = 0, in_bin_n = 0;
            const float in_bin = (float)bin + 8388608.f;
            each_group([&](int, const float (&l)[4]) {
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
                if (!in) return;
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
            });
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
                for (int t0 = tid; t0 - lane < 4 * (int)n; t0 += kThreads) {  // four threads to an entry, each every fourth
                    const uint32_t key = s.all[min(t0 >> 2, (int)n - 1)].x;
                    u64 more = 0, equal = 0, count = 0;
#pragma unroll 4
                    for (int i = t0 & 3; i < (int)n; i += 4) {
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
    u64 kept_sum = 0;         // with top-p, the sum of what stays
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
            kept_sum = s.above + ties * w;
        } else {  // it ends among the tokens equal to the top-k cut
            ties = (s.target - s.sum + w_cut - 1) / w_cut;
            kept_sum = s.sum + ties * w_cut;
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

    if constexpr (RECORD) {
        // Top-p's search has left the sum, if min-p takes nothing from it: expf is off by two steps at
        // most, so no larger logit's e is below the floor if the cut's is well above.
        u64 total = kept_sum;
        const float e_cut = quick ? quick_e(at_cut) : plain_e(at_cut, m, T);
        if (!(p < 1.f && (floor_p <= 0.f || e_cut * (1.f - 0x1p-20f) >= floor_p))) {
            u64 sum = 0;
            each_group([&](int, const float (&l)[4]) {
                if (!(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= from)) return;
                uint32_t w[4];
                kept(l, w);
                sum += (wide(w[0]) + wide(w[1])) + (wide(w[2]) + wide(w[3]));
            });
            u64 here;
            scan(sum, here);
            const int t = exchange(here, 0, 0);
            total = part ? ties * wide(code_cut) : 0;
            for (int r = 0; r < C; ++r) total += s.xch[t][0][r];
        }
        if (!part) {
            if (rank == 0 && tid == 0) record(cut, ties ? 0x7fffffff : -1, total);
            return;
        }
        // the last kept one of those equal to the cut: of the candidates the one with ties - 1 before it,
        if (few) {
            for (int i = tid; i < n_cand; i += kThreads) {
                if (s.cand[i] != at_cut) continue;
                u64 before = 0;
                for (int r = 0; r < C; ++r) {
                    const Shared *o = of(r);
                    for (int j = 0; j < o->n_cand; ++j) before += o->cand[j] == at_cut && o->cand_at[j] < s.cand_at[i];
                }
                if (before + 1 == ties) record(cut, s.cand_at[i], total);
            }
            sync();  // no CTA leaves while another reads its candidates
            return;
        }
        // of the row by counts of its segments of 32 groups, a run of them to a warp, one to a lane
        static_assert(kMaxSegs <= 32 * kWarps);
        const int per = ((groups + 31) / 32 + kWarps - 1) / kWarps, g0 = warp * per * 32 + lane;
        uint32_t own = 0;
        const float which = infinite ? INFINITY : at_cut;
        constexpr int kBatch = BF16 ? 8 : 4;
        for (int j = 0; j < per; j += kBatch)
            batch(std::integral_constant<int, kBatch>(), g0 + j * 32, 32, min(groups, (warp + 1) * per * 32), [&](int g, const Vec &u) {
                float l[4];
                split(u, l);
                uint32_t n = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) n += l[i] == which;
                n = __reduce_add_sync(kFull, n);
                if (lane == (g - g0) / 32) own = n;
            });
        u64 here, before = scan(own, here);
        const int t = exchange(here, 0, 0);
        for (int r = 0; r < rank; ++r) before += s.xch[t][0][r];
        const unsigned found = __ballot_sync(kFull, before < ties && ties <= before + own);
        if (!found) return;
        const int seg = __ffs(found) - 1, g = g0 + 32 * seg;
        float l[4];
        load4(g, l);
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += l[i] == at_cut;
        u64 place = __shfl_sync(kFull, before, seg) + warp_scan(n) - n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (l[i] == at_cut && ++place == ties) record(cut, base + 4 * g + i - shift, total);
        return;
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
template <bool BF16, bool RECORD>
__global__ void __launch_bounds__(kLongThreads) long_row_kernel(const SampleArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ u64 sums[32];
    __shared__ u64 hist[256];
    __shared__ u64 s_sum;
    __shared__ int s_bin;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const size_t row = blockIdx.x;
    const Source src = source_of<RECORD>(a, row);
    const das_sampling &sampling = *src.sampling;
    const int b = src.b, V = a.vocab;
    auto key = [&](int i) {
        const size_t at = src.row * src.stride + i;
        return key_of(BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(src.logits)[at] << 16)
                           : static_cast<const float *>(src.logits)[at]);
    };
    float T = sampling.temperature ? sampling.temperature[b] : 1.f;
    long long k = sampling.top_k ? sampling.top_k[b] : 0;
    const float p = sampling.top_p ? sampling.top_p[b] : 1.f;
    float floor_p = sampling.min_p ? sampling.min_p[b] : 0.f;
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
            if constexpr (RECORD) {
                a.records[row] = RowRecord{};
            } else {
                accept_one(a, row, -1);
                a.tokens[row] = -1;
                if (a.logprobs) a.logprobs[row] = -INFINITY;
            }
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
    if constexpr (RECORD) {
        if (tid == 0) a.records[row] = record_of(top, cut, last, T, floor_p, total);
        return;
    }
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

// ---- proposals that were drawn by chance -------------------------------------------
// From the rows' records: the first proposal that is refused, and the draw in its place from
// what the target's row has more.  What bounds a call: of the 48.0 us of 64 proposals of 128257 bf16
// logits each, whose 33 MB take 4.8 us, the rows' first pass (largest logit and bins) takes about 12, the
// look for the cut 10, the count of the logits equal to it 6, and this kernel 13, of which 8 are the
// sweep over one row of target and drafter by 64 of the SMs; the rest is launches and barriers.  8 x 16
// proposals of 32000 take 28 to 30 us, one sequence's 8 of 32000 20 to 22 us, all latency.  A cluster to a sequence; each of its warps has a run of
// the row in 32 steps at most, whose sums stand in its lanes: the warp that the draw falls
// to finds the step in them and computes that alone again.
constexpr int kAcceptThreads = 1024;
template <bool BF16>
struct RowProbs {
    using Elem = std::conditional_t<BF16, uint16_t, float>;
    RowRecord r;
    const Elem *logits;
    float m, cut, rT;
    bool quick;
    __device__ __forceinline__ RowProbs(const SampleArgs &a, const RowRecord &record, size_t row, bool second) {
        r = record;
        logits = static_cast<const Elem *>(second ? a.second : a.logits) +
                 row * (size_t)(second ? a.second_stride : a.row_stride);
        const bool none = r.top == 0;  // (no logit above -inf)
        m = none ? 0.f : logit_of(r.top);
        cut = none ? INFINITY : logit_of(max(r.key, kKeyNone));
        if (none) r.last = -1;
        rT = none ? 1.f : __frcp_rn(r.T);
        quick = r.T > 1e-18f && r.T < 1e18f && (__float_as_uint(r.T) & 0x7fffffu) != 0x7fffffu;
    }
    __device__ __forceinline__ float logit(int v) const {
        float l;
        if constexpr (BF16) l = __uint_as_float((uint32_t)logits[v] << 16);
        else l = logits[v];
        return l == l ? l : -INFINITY;
    }
    __device__ __forceinline__ bool kept(float l, int v) const { return l > cut || (l == cut && v <= r.last); }
    __device__ __forceinline__ float floored(float e) const { return e >= r.floor ? e : 0.f; }
    // of a token alone
    __device__ __forceinline__ float p(int v) const {
        const float l = logit(v);
        if (!kept(l, v)) return 0.f;
        const float e = floored(e_of(key_of(l), r.top, m, r.T));
        return e > 0.f ? __fmul_rn(e, r.inv) : 0.f;
    }
    // e; where all T are `quick` the quotient by Markstein's steps as in sample_kernel, which differ
    // from the division below e^-100 alone, where no weight is left
    template <bool QUICK>
    __device__ __forceinline__ float e(float l) const {
        const float d = l - m;
        float y;
        if (QUICK) {
            const float q = fmaxf(d * rT, -100.f);
            y = expf(fmaf(fmaf(-q, r.T, d), rT, q));
        } else {
            y = plain_e(l, m, r.T);
        }
        return floored(l == m ? 1.f : y);
    }
};

template <bool BF16>
__global__ void __launch_bounds__(kAcceptThreads, 1) speculative_accept_kernel(const SpeculateArgs a) {
    constexpr int kWarps = kAcceptThreads / 32, kBatch = 2;
    __shared__ u64 s_sum[kWarps], s_cta[2][kMaxRowCtas];
    __shared__ RowRecord s_record[2];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int W = a.rows.W, V = a.rows.vocab;
    const size_t b = blockIdx.x / C;
    auto sync = [&] {
        if (C > 1) cluster.sync();
        else __syncthreads();
    };
    sync();  // every CTA of the cluster has started
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bool refused = false;
    if (tid < W) {  // (W <= 1024 = kAcceptThreads)
        const int y = a.draft[b * W + tid];
        const RowRecord *const at = a.rows.records + b * W + tid;
        const RowProbs<BF16> p(a.rows, at[0], b * W + tid, false), q(a.rows, at[(size_t)a.rows.B * W], b * W + tid, true);
        refused = y < 0 || y >= V || !((double)a.uniforms[b * W + tid] * (double)q.p(y) < (double)p.p(y));
    }
    const unsigned some = __ballot_sync(kFull, refused);
    if (lane == 0) s_sum[warp] = some ? warp * 32 + __ffs(some) - 1 : 0x7fffffff;
    __syncthreads();
    const int first = (int)min(__reduce_min_sync(kFull, (uint32_t)s_sum[lane]), (uint32_t)W);
    if (tid < 2 && first < W) s_record[tid] = a.rows.records[((size_t)tid * a.rows.B + b) * W + first];
    __syncthreads();
    if (rank == 0 && tid == 0) {
        a.accepted[b] = first;
        if (a.committed) a.committed[b] = min(first + 1, W);
        if (first == W) a.next_token[b] = a.draft[b * W + W - 1];
    }
    if (first == W) return;  // the same in the whole cluster

    const RowProbs<BF16> p(a.rows, s_record[0], b * W + first, false), q(a.rows, s_record[1], b * W + first, true);
    // the warp's run of `parts` times 32 tokens, 1 << log_step of them to a step
    const int parts = (int)(((long long)V + C * kWarps * 32 - 1) / (C * kWarps * 32));
    int log_step = 0;
    while (parts > 32 << log_step) ++log_step;
    const long long lo = (long long)(rank * kWarps + warp) * parts * 32;
    bool plain = false;  // rounding has left nothing: the target's own weights
    // x 2^40 rounded, x in [0, 1], as (the upper part of it) 2^20 + the lower: 64-bit conversions
    // are slow
    auto weight = [&](auto quick, long long v, float lp, float lq) -> uint2 {  // (past the row lp is -inf)
        if (!p.kept(lp, (int)v)) return make_uint2(0, 0);
        // (products and difference each rounded, never fused: equal probabilities leave 0)
        const float e = p.template e<quick.value>(lp);
        const float taken = q.kept(lq, (int)v) ? __fmul_rn(q.template e<quick.value>(lq), q.r.inv) : 0.f;
        float x = __fsub_rn(__fmul_rn(e, p.r.inv), taken);
        x = (plain ? e * 0x1p-8f : fmaxf(x, 0.f)) * 0x1p20f;
        const uint32_t up = __float2uint_rz(x);
        return make_uint2(up, __float2uint_rn((x - (float)up) * 0x1p20f));
    };
    auto sum_of = [](uint2 w) { return ((u64)w.x << 20) + w.y; };
    u64 total = 0, mine = 0, before = 0, step_sum = 0;
    auto sweep = [&](auto quick) {
        mine = step_sum = 0;
        for (int i0 = 0; i0 < parts; i0 += kBatch) {
            float lp[kBatch], lq[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const long long v = lo + (i0 + j) * 32 + lane;
                lp[j] = lq[j] = -INFINITY;
                if (i0 + j < parts && v < V) {
                    lp[j] = p.logit((int)v);
                    lq[j] = q.logit((int)v);
                }
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                uint2 w = weight(quick, lo + (i0 + j) * 32 + lane, lp[j], lq[j]);
                w = make_uint2(__reduce_add_sync(kFull, w.x), __reduce_add_sync(kFull, w.y));
                const u64 sum = sum_of(w);
                if (lane == (i0 + j) >> log_step) step_sum += sum;
                mine += sum;
            }
        }
    };
    const bool quick = p.quick && q.quick;
    for (int turn = 0; turn < 2; ++turn) {
        if (quick) sweep(std::true_type());
        else sweep(std::false_type());
        if (lane == 0) s_sum[warp] = mine;
        __syncthreads();
        u64 cta = s_sum[lane], up = lane < warp ? cta : 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            cta += __shfl_xor_sync(kFull, cta, d);
            up += __shfl_xor_sync(kFull, up, d);
        }
        if (tid < C) {
            u64(*to)[kMaxRowCtas] = C > 1 ? cluster.map_shared_rank(s_cta, tid) : s_cta;
            to[turn][rank] = cta;
        }
        sync();
        total = 0;
        before = up;
        for (int r = 0; r < C; ++r) {
            if (r < rank) before += s_cta[turn][r];
            total += s_cta[turn][r];
        }
        if (total > 0) break;
        plain = true;
    }
    if (total == 0) {
        if (rank == 0 && tid == 0) a.next_token[b] = -1;
        return;
    }
    if (tid == 0) {  // (one thread: doubles are slow)
        float u = a.resample[b];
        if (!(u >= 0.f)) u = 0.f;
        const u64 r = (u64)((double)u * (double)total);
        s_sum[0] = r < total ? r : total - 1;
    }
    __syncthreads();
    const u64 r = s_sum[0];
    if (r < before || r >= before + mine) return;
    auto scan = [&](u64 x) {  // inclusive, from `before` on
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const u64 o = __shfl_up_sync(kFull, x, d);
            if (lane >= d) x += o;
        }
        return x + before;
    };
    u64 x = scan(step_sum);
    const int step = __ffs(__ballot_sync(kFull, r < x)) - 1;
    before = __shfl_sync(kFull, x - step_sum, step);
    for (int i = step << log_step; i < (step + 1) << log_step; ++i) {
        const long long v = lo + i * 32 + lane;
        u64 w = 0;  // (as in the sweep, to the last bit)
        if (v < V) {
            const float lp = p.logit((int)v), lq = q.logit((int)v);
            w = sum_of(quick ? weight(std::true_type(), v, lp, lq) : weight(std::false_type(), v, lp, lq));
        }
        x = scan(w);
        if (r >= x - w && r < x) a.next_token[b] = (int)v;
        before = __shfl_sync(kFull, x, 31);
        if (before > r) break;
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

template <bool BF16, bool RECORD>
cudaError_t sample_launch_t(const SampleArgs &a, cudaStream_t stream) {
    const long long rows = (long long)a.B * a.W * (RECORD ? 2 : 1);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int sms = attn_grid_size(dev);
    if (sms <= 0) return cudaErrorInvalidDevice;
    // CTAs per row: enough to hold the row, and as many as fill the SMs
    constexpr int kMaxSlice = kSliceBytes<BF16> / (BF16 ? 2 : 4) - 4;  // (with the shift of a first group)
    const int hold = (int)(((long long)a.vocab + kMaxSlice - 1) / kMaxSlice);
    if (hold > kMaxRowCtas)
        return launch_pdl(long_row_kernel<BF16, RECORD>, dim3((unsigned)rows), dim3(kLongThreads), 1, 0,
                          stream, a);
    int C = 1;  // a power of two: the bins divide by it
    while (C < kMaxRowCtas && (C < hold || (rows * C * 2 <= sms && a.vocab > C * 4 * kDrawThreads)))
        C *= 2;
    const int slice = ((a.vocab + C - 1) / C + 3) / 4 * 4;
    const dim3 grid((unsigned)(rows * C)), block(RECORD ? kRecordThreads : kDrawThreads);
    size_t smem = RECORD ? 0 : (size_t)(slice + 4) * (BF16 ? 2 : 4);  // (a group more where rows begin within one)
    if (C > 1) smem = std::max(smem, 2 * kBins * sizeof(uint32_t));  // (bins may be sent there)
    static std::atomic<bool> configured[64];  // the shared-memory opt-in, once per device
    if (dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(sample_kernel<BF16, RECORD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSliceBytes<BF16>);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    return launch_pdl(sample_kernel<BF16, RECORD>, grid, block, C, smem, stream, a, slice);
}

}  // namespace

cudaError_t sample_launch(const SampleArgs &a, cudaStream_t stream) {
    if ((long long)a.B * a.W == 0) return cudaSuccess;
    return a.bf16 ? sample_launch_t<true, false>(a, stream) : sample_launch_t<false, false>(a, stream);
}

cudaError_t speculative_accept_launch(const SpeculateArgs &a, cudaStream_t stream) {
    if (a.rows.B == 0) return cudaSuccess;
    const cudaError_t e = a.rows.bf16 ? sample_launch_t<true, true>(a.rows, stream)
                                      : sample_launch_t<false, true>(a.rows, stream);
    if (e != cudaSuccess) return e;
    int C = 1;
    while (C < kMaxRowCtas && a.rows.vocab > C * 4 * kAcceptThreads) C *= 2;
    return launch_pdl(a.rows.bf16 ? speculative_accept_kernel<true> : speculative_accept_kernel<false>,
                      dim3((unsigned)(a.rows.B * C)), dim3(kAcceptThreads), C, 0, stream, a);
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
