// das_paged4_attention.cu -- depth-asynchronous attention (Eqs. 2-3) over the paged 4-bit
// cache, on the 5th-generation tensor cores of sm_103a with keys and values in
// tensor memory.
//
// The mathematics.  A stored value (c - 8) s has at most 8 significant bits, so it is a bf16
// number, and all products run in bf16: S^T = K Q^T and O^T = V^T P^T, with keys (or the
// elements of a value) as the 128 rows of the product and the query rows as its columns.
// The stored codes become A operands in tensor memory, which is where their widening
// ends, and a tile costs in proportion to the query rows there are (16, 32 or 64 columns).
// With x_j = s_j + off, off = -m - kBelow, m the score of one key of the segment,
//     p_j = 2^(x_j),  O = sum p_j v_j,  l = sum p_j,
// out = O / l and lse = ln 2 (m + kBelow + log2 l).  bf16 has fp32's exponents: p_j keeps its
// 8 bits from 2^-126 to 2, so m need not be the largest score: any key's will do that is within
// kBelow binary orders below it.  Only where a weight of a tile comes to 2 or more is the
// row's reference set again, to the tile's largest, and O and l are rescaled.  The output
// is divided by the sum of the rounded weights, taken by the tensor core with a row of
// ones, and is so a mean of the values with the very weights in use; the lse is from the
// unrounded ones.  Weights are rounded to bf16 as both operands of a product are of one type, and a second
// part of each would double P's stores and products: an output is off by 0.0018 to 0.0020 of its
// size (root mean square), by 0.0016 with weights in binary32, which is the output's own rounding.
//
// A word of eight codes gives four pairs (elements i and i + 4): or-ing four bits into bf16 128
// makes 128 + c, and (128 + c) s - 136 s is exact.  The order of elements (keys) that comes of it
// is undone in the other operand: in the queries, and in the places of P's rows.
//
// Work split: every (sequence, kv head) pair owns a tile for each 128 of its prefix (two
// pages) and one for the block's own keys.  All pairs' tiles are one list, of which CTA
// c takes the c-th of C ranges, cut into segments at pair boundaries.  A segment that is
// a whole pair writes the output, others a partial (O / l, lse); who comes last at the pair's counter
// joins them.  Lengths are read on the device, so the table's width does not matter.
//
// One CTA = two groups of four softmax warps, four warps that widen keys, four or eight that
// widen values, and one each for loads, S and P V.  With up to 32 rows the groups take turns at
// the tiles, with 64 each has half of every tile's rows; a thread has one key of a tile.
// Every wait is bounded (2 s); a time-out sets the status word and ends the CTA's waits.  Tensor
// memory is freed before the CTA exits.
//
// What bounds it: the warps' instructions, not the bytes.  4 x 32768 tokens with 32 query and 8 kv
// heads of 128 (143 MB, 21 us at the copy rate) take 44.4 us with one row a head, 3.2 TB/s, and 67.3 us
// with 16.  Of the 0.8 us that a tile takes with one row, 0.6 are left without the widening's
// arithmetic; with 16 the softmax groups are busy throughout, 2100 cycles a tile, of which almost a thousand
// are a tile's own waits, barrier and masks; the products take 540.  (Scores loaded a chunk ahead made
// it 70.7 us, as their registers spill.)  Scheduled instructions are half of the issue slots' number.  A call of one token
// (15.1 us) spends half of its time before the first tile and after the last.
#include <algorithm>
#include <atomic>

#include "das_internal.h"
#include "das_tcgen05.h"

namespace das {
namespace {

using namespace t5;

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kKeys = 128;  // of a tile: the rows of a product
constexpr int kPage = DAS_PAGE_TOKENS;
constexpr int kGroupWarps = 4, kSoftWarps = 8;
// The roles of a CTA's warps, for N columns.
template <int N>
struct Roles {
    // With few rows the two softmax groups take turns at the tiles, each with a reference, sums and an O
    // of its own; with 64 each has half of every tile's rows.
    static constexpr bool kTurns = N <= 32;
    // Sets of four warps that widen values: tile k is set k % the sets' number's.  (Keys have one.)
    // (A second one for values: 4 x 32768 tokens with one row 44.8 us, 46.8 without, a single token 15.2 and 14.7.
    // With 32 rows or 64 a thread has fewer registers for it than the softmax needs: 56.3 and 75.8 us, 54.1 and 72.1 without.)
    static constexpr int kValueSets = N == 16 ? 2 : 1;
    static constexpr int kKeyWarp0 = kSoftWarps, kValueWarp0 = kKeyWarp0 + 4;
    static constexpr int kProducerWarp = kValueWarp0 + 4 * kValueSets, kSWarp = kProducerWarp + 1;
    static constexpr int kPvWarp = kSWarp + 1, kThreads = (kPvWarp + 1) * 32;
};
constexpr float kBelow = 60.f, kMost = 1e38f;
// Tensor memory: keys [2], values [2], S [2], O, the sums of P.
constexpr int kKCol = 0, kVCol = 128, kSCol = 256, kOCol = 384, kSumCol = 448, kCols = 512;
constexpr int kInfos = 64;  // ring of the tiles' visible keys
// The end of a pair (its block tile, the read-out and what joins it) weighs kEnd tiles more.  (16 sequences of
// 1024 to 8192 tokens, 4 x 32768, both with 64 rows, as measured when it was chosen: 51.4 and 69.8 us; with 4
// 52.3 and 70.3, with 6 50.8 and 70.2.)
constexpr int kEnd = 5;
// Weight of a CTA's range, unless it is a pair.  (A pair of 1500 and one of 4000 tokens take 12.6 and 12.1 us,
// with 10 13.7 and 14.7; with 6 11.0 and 11.4, but 4 pairs of 256 tokens 8.1 us instead of 7.0, as they are split.)
constexpr int kLeast = 7;
constexpr int kFan = 8;     // partials that are joined at once
constexpr int kPrefetch = 8;  // pages pulled into L2 before the dependency wait

template <int D, int N>
struct Layout {
    static constexpr int kCodes = kPage * D / 2;               // of a page's keys, or values
    static constexpr int kScales = kPage * D / DAS_SCALE_GROUP;
    static constexpr int kVOff = 2 * kCodes, kKsOff = 4 * kCodes, kVsOff = kKsOff + 2 * kScales;
    static constexpr int kStage = (4 * kCodes + 4 * kScales + 1023) / 1024 * 1024;
    static constexpr int kStages = 8;
    static constexpr int kQ = N * D * 2, kP = kKeys * 128;
    static constexpr int kQOff = kStages * kStage;
    static constexpr int kPOff = kQOff + 2 * kQ;
    static constexpr int kOnesOff = kPOff + 2 * kP;            // an 8 x 16 operand of ones
    static constexpr int kBarOff = kOnesOff + 256;
    // full, empty [kStages], qready, qfree [2], kready, vready, sdone, pready, pvdone [2],
    // drain [2]
    static constexpr int kBars = 2 * kStages + 4 + 10 + 2;
    static constexpr int kInfoOff = (kBarOff + 8 * kBars + 15) / 16 * 16;
    static constexpr int kRowOff = kInfoOff + kInfos * 8;      // floats of the rows: 4 x [2][64], [64]
    static constexpr int kSumOff = kRowOff + 9 * 64 * 4;       // [8 warps][32]: sums or largest
    static constexpr int kVsxOff = kSumOff + 8 * 32 * 4;       // [8 warps][64]: the values' scales
    static constexpr int kNfOff = kVsxOff + 2 * 4 * 64 * 4;    // [4][128]: first key that is not finite
    static constexpr int kTableOff = kNfOff + 4 * 128 * 4;     // [256]: scale bytes' numbers, bf16 twice
    static constexpr int kJoinOff = kTableOff + 256 * 4;
    static constexpr int kMiscOff = kJoinOff + 64;
    static constexpr int kBytes = kMiscOff + 128 + 1024;       // + alignment slack
    static_assert(kBytes <= 232448, "shared memory per CTA");
};

// ---- the list of tiles ------------------------------------------------------------
__device__ __forceinline__ int clamp_to(int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); }
__device__ __forceinline__ int prefix_of(const Paged4AttnParams &p, int b) {
    return clamp_to(__ldcg(p.prefix_len + b), p.max_pages * kPage);
}
__device__ __forceinline__ int block_of(const Paged4AttnParams &p, int b) {
    return clamp_to(__ldcg(p.block_len + b), p.max_block);
}
// a sequence without rows has nothing but its outputs to clear
// (P may be 2^31 - 64)
__device__ __forceinline__ int tiles_of(int P, int T) { return T > 0 ? (int)((P + (unsigned)kKeys - 1) / kKeys) + 1 : 1; }

struct Walk {
    int b, h, t, nt, P, T;
};
__device__ __forceinline__ void walk_load(const Paged4AttnParams &p, Walk &w) {
    if (w.b < p.B) {
        w.P = prefix_of(p, w.b);
        w.T = block_of(p, w.b);
        w.nt = tiles_of(w.P, w.T);
    }
}
__device__ __forceinline__ void walk_pair(const Paged4AttnParams &p, Walk &w) {
    w.t = 0;
    if (++w.h == p.Hkv) {
        w.h = 0;
        ++w.b;
        walk_load(p, w);
    }
}

// What a CTA has of the list: tile t of the pair that begins at weighted position q has
// position q + t, and the range [c W / C, (c + 1) W / C) the tiles of positions in it.
struct Plan {
    Walk w;
    int ntiles, ctas;
    long long W, q;  // all weight; position of the first pair
};
__device__ __forceinline__ unsigned long long udiv(unsigned long long a, unsigned long long b) {
    return ((a | b) >> 32) == 0 ? (uint32_t)a / (uint32_t)b : a / b;
}
__device__ __forceinline__ int cta_of(const Plan &pl, long long q) {
    return (int)udiv((unsigned long long)(q + 1) * (unsigned)pl.ctas - 1, (unsigned long long)pl.W);
}
// (by one whole warp; P and T: the lane's sequence's lengths if there are no more than 32)
__device__ void make_plan(const Paged4AttnParams &p, Plan &pl, int P, int T) {
    const int lane = threadIdx.x & 31;
    auto weight = [&](int b) {
        if (b >= p.B) return 0;
        return (p.B <= 32 ? tiles_of(P, T) : tiles_of(prefix_of(p, b), block_of(p, b))) + kEnd;
    };
    long long W = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32)
        W += (long long)__reduce_add_sync(kFull, (unsigned)weight(b0 + lane)) * p.Hkv;
    const int ctas = (int)max(1ll, min((long long)p.num_ctas, max((long long)p.B * p.Hkv, W / kLeast)));
    pl.W = W;
    pl.ctas = ctas;
    pl.ntiles = 0;
    pl.w = {p.B, 0, 0, 1, 0, 0};
    pl.q = W;
    if ((int)blockIdx.x >= ctas) return;
    const long long at[2] = {(long long)udiv((unsigned long long)blockIdx.x * (unsigned long long)W, (unsigned)ctas),
                             (long long)udiv((unsigned long long)(blockIdx.x + 1) * (unsigned long long)W, (unsigned)ctas)};
    long long index[2] = {-1, -1};  // tiles before at[i]
    long long run = 0, tiles = 0;   // weight, tiles before the chunk
    for (int b0 = 0, found = 0; b0 < p.B && found < 2; b0 += 32) {
        const int wt = weight(b0 + lane);
        int inc = wt;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(kFull, inc, d);
            if (lane >= d) inc += u;
        }
        const int n = min(32, p.B - b0);
        while (found < 2) {
            const unsigned m = __ballot_sync(kFull, run + (long long)inc * p.Hkv > at[found]);
            if (!m) break;
            const int f = __ffs(m) - 1;
            const int wf = __shfl_sync(kFull, wt, f), before = __shfl_sync(kFull, inc, f) - wf;
            const long long q0 = run + (long long)before * p.Hkv, off = at[found] - q0;
            int h = (int)udiv((unsigned long long)off, (unsigned)wf), t = (int)(off - (long long)h * wf);
            const int nt = wf - kEnd;
            index[found] = tiles + ((long long)before - (long long)kEnd * f) * p.Hkv + (long long)h * nt + min(t, nt);
            if (found == 0) {
                pl.w.b = b0 + f;
                pl.w.h = h;
                pl.w.t = t;
                pl.q = q0 + (long long)h * wf;
                if (t >= nt) {  // past its last tile: the next pair
                    pl.q += wf;
                    pl.w.t = 0;
                    if (++pl.w.h == p.Hkv) {
                        pl.w.h = 0;
                        ++pl.w.b;
                    }
                }
            }
            ++found;
        }
        const int all = __shfl_sync(kFull, inc, 31);
        run += (long long)all * p.Hkv;
        tiles += ((long long)all - (long long)kEnd * n) * p.Hkv;
    }
    if (index[0] < 0) index[0] = tiles;
    if (index[1] < 0) index[1] = tiles;
    if (p.B <= 32) {
        pl.w.P = __shfl_sync(kFull, P, pl.w.b & 31);
        pl.w.T = __shfl_sync(kFull, T, pl.w.b & 31);
        pl.w.nt = tiles_of(pl.w.P, pl.w.T);
    } else {
        walk_load(p, pl.w);
    }
    pl.ntiles = (int)(index[1] - index[0]);
}

// A segment: tiles [w.t, end) of a pair.
struct Segment {
    int n, pre;  // tiles, those of them before the block's
};
__device__ __forceinline__ Segment segment_of(const Walk &w, int left) {
    const int n = min(left, w.nt - w.t);
    return {n, min(n, w.nt - 1 - w.t)};
}

__device__ __forceinline__ float unit_of(const float *unit, int h) {
    if (!unit) return 1.f;
    const uint32_t bits = __float_as_uint(unit[h]);
    const int e = bits >> 31 ? 0 : min(max((int)(bits >> 23) - 127, -40), 40);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}
// A scale byte's number, which is a bf16 number: its bits are those of the fp32 number 2^-112 times it.
__device__ __forceinline__ float scale_of(uint32_t byte) {
    return byte == 0xffu ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte << 20) * 5.192296858534828e33f;
}

// byte offset of 16-byte chunk c of row m, rows of 128 bytes, swizzled
__device__ __forceinline__ uint32_t chunk16(int m, int c) { return m * 128 + ((c ^ (m & 7)) << 4); }
// 16-byte chunk c of a token's keys: a page's are rows of 128 bytes
template <int D>
__device__ __forceinline__ uint32_t key_chunk(int t, int c) {
    constexpr int kTokens = 256 / D;  // tokens to a row
    return chunk16(t / kTokens, (t % kTokens) * (8 / kTokens) + c);
}
// Eight bf16 elements in the order that a word of eight codes is widened in.
__device__ __forceinline__ uint4 paired(uint4 x) {
    return make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632),
                      __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
}
// Four pairs 128 + c of a word's codes.  (The masks are registers, so that both take one
// instruction.)
struct Widen {
    uint32_t mask, base;
    __device__ __forceinline__ Widen() {
        asm volatile("mov.u32 %0, 0x000f000f;" : "=r"(mask));
        asm volatile("mov.u32 %0, 0x43004300;" : "=r"(base));
    }
    __device__ __forceinline__ void operator()(uint32_t w, uint32_t (&h)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(h[i]) : "r"(w >> (4 * i)), "r"(mask), "r"(base));
    }
};
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
    return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u);
}

// A bounded wait (as t5::wait) that sleeps between its tries: what the many warps that wait would
// poll away are issue slots of those that work.
static __device__ __noinline__ bool sleep_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag,
                                               int32_t *status) {
    const unsigned long long t0 = globaltimer();
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        __nanosleep(20);
        if ((it & 15u) == 0) {
            if (*abort_flag) return false;
            if (globaltimer() - t0 > kWaitNs) {
                *abort_flag = 1;
                atomicOr(status, kStatusWaitTimeout);
                return false;
            }
        }
    }
}

// A run of a pair's partials to be joined: run r0 / run of n segments, CTA c0's first.
struct Join {
    int pair, rows, c0, n, run, r0;
};
// Partials at places first, first + step, ... of rows to the output, or into the first one.
// out = sum_s 2^(lse_s - M) O_s / sum_s 2^(lse_s - M), lse = M + log2 of that sum.  (The whole CTA.)
template <int D>
__device__ void join(const Paged4AttnParams &p, const Join &jn, size_t first, int step, int count, bool final,
                     float *lses) {
    constexpr int kPer = D / 4;  // threads to a row
    const int b = jn.pair / p.Hkv, h = jn.pair % p.Hkv;
    const int all = final ? p.rows_max : jn.rows;
    for (int u = threadIdx.x; u < all * kPer; u += blockDim.x) {
        const int r = u / kPer, c = u % kPer * 4;
        float M = -INFINITY, L = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kLoads = 4;
        for (int s0 = 0; s0 < (r < jn.rows ? count : 0); s0 += kLoads) {
            float ls[kLoads];
            float4 x[kLoads];
#pragma unroll
            for (int s = 0; s < kLoads; ++s) {
                ls[s] = -INFINITY;
                x[s] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s0 + s < count) {
                    const size_t at = (first + (size_t)(s0 + s) * step) * p.rows_max + r;
                    ls[s] = __ldcg(p.part_lse + at);
                    x[s] = __ldcg(reinterpret_cast<const float4 *>(p.part_o + at * D + c));
                }
            }
            float m = M;
#pragma unroll
            for (int s = 0; s < kLoads; ++s) m = fmaxf(m, ls[s]);  // (NaN goes into the sums alone)
            const float f = M == m ? 1.f : ex2(M - m);
            M = m;
            L *= f;
            acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
#pragma unroll
            for (int s = 0; s < kLoads; ++s) {
                const float g = ls[s] == -INFINITY ? 0.f : ex2(ls[s] - m);
                L += g;
                acc = make_float4(acc.x + x[s].x * g, acc.y + x[s].y * g, acc.z + x[s].z * g, acc.w + x[s].w * g);
            }
        }
        const float inv = L == 0.f ? 0.f : 1.f / L, lse = L == 0.f ? -INFINITY : M + log2f(L);
        if (final) {
            const int hq = h * p.G + r % p.G, i = r / p.G;
            *reinterpret_cast<uint2 *>(p.out + (((size_t)b * p.max_block + i) * p.Hq + hq) * D + c) =
                make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (c == 0) p.lse[((size_t)b * p.Hq + hq) * p.max_block + i] = lse * kLn2;
        } else {
            *reinterpret_cast<float4 *>(p.part_o + (first * p.rows_max + r) * D + c) =
                make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            if (c == 0) lses[r] = lse;
        }
    }
    if (final) return;
    __syncthreads();  // all have read the first one's lse
    for (int r = threadIdx.x; r < jn.rows; r += blockDim.x) p.part_lse[first * p.rows_max + r] = lses[r];
}

template <int D, int N>
__global__ void __launch_bounds__(Roles<N>::kThreads, 1)
    paged4_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const Paged4AttnParams p) {
    using Lt = Layout<D, N>;
    using Ro = Roles<N>;
    constexpr bool kTurns = Ro::kTurns;
    constexpr int kValueSets = Ro::kValueSets, kKeyWarp0 = Ro::kKeyWarp0, kValueWarp0 = Ro::kValueWarp0,
                  kProducerWarp = Ro::kProducerWarp, kSWarp = Ro::kSWarp, kPvWarp = Ro::kPvWarp,
                  kThreads = Ro::kThreads;
    constexpr int kStages = Lt::kStages, R = kTurns ? N : N / 2;  // rows of a group
    constexpr int kStep = kTurns ? 2 : 1;                         // from one tile of a group to its next
    // rows whose scores a softmax thread has at once (with 16 for all 16 ragged sequences take 56.9 us, 52.2 with
    // 8, and 4 x 32768 with 64 rows 72.1 and 70.1; with 8 for all 4 x 32768 with one row 46.1, 45.1 with 16)
    constexpr int kChunk = N == 16 ? 16 : 8;
    static_assert(R % kChunk == 0, "rows in chunks");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const sm = smem_raw + (-smem_u32(smem_raw) & 1023u);
    const uint32_t sbase = smem_u32(sm);
    const uint32_t b_full = sbase + Lt::kBarOff, b_empty = b_full + 8 * kStages,
                   b_qready = b_empty + 8 * kStages, b_qfree = b_qready + 16, b_kready = b_qfree + 16,
                   b_vready = b_kready + 16, b_sdone = b_vready + 16,
                   b_pready = b_sdone + 16, b_pvdone = b_pready + 16, b_drain = b_pvdone + 16;
    int2 *const infos = reinterpret_cast<int2 *>(sm + Lt::kInfoOff);
    volatile uint32_t *const misc = reinterpret_cast<volatile uint32_t *>(sm + Lt::kMiscOff);
    volatile int *const abort_flag = reinterpret_cast<volatile int *>(sm + Lt::kMiscOff + 4);
    int *const s_nf = reinterpret_cast<int *>(sm + Lt::kNfOff);
    // of each group's rows: minus the reference, a factor or the rounded weights' sum, the weights' sum,
    // the factor of the group's O; lse
    float *const s_off = reinterpret_cast<float *>(sm + Lt::kRowOff), *const s_alpha = s_off + 128,
                 *const s_total = s_off + 256, *const s_factor = s_off + 384, *const s_lse = s_off + 512;
    Join *const s_joins = reinterpret_cast<Join *>(sm + Lt::kJoinOff);  // [2]: cut pairs of a CTA
    Plan *s_plan = reinterpret_cast<Plan *>(sm + Lt::kMiscOff + 16);
    static_assert(sizeof(Plan) <= 112, "plan");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(b_full + 8 * s, 1);
            mbar_init(b_empty + 8 * s, 8);  // the warps that widen
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_qready + 8 * i, 4);
            mbar_init(b_qfree + 8 * i, 1);
            mbar_init(b_kready + 8 * i, 4);
            mbar_init(b_vready + 8 * i, 4);
            mbar_init(b_sdone + 8 * i, 1);
            mbar_init(b_pready + 8 * i, kTurns ? kGroupWarps : kSoftWarps);
            mbar_init(b_pvdone + 8 * i, 1);
            mbar_init(b_drain + 8 * i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *abort_flag = 0;
    }
    if (warp == kSWarp) {
        asm volatile(
            "tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                sbase + Lt::kMiscOff),
            "n"(kCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (warp == kProducerWarp && elect_one())
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_k)) : "memory");
    for (int i = threadIdx.x; i < 256 / 16; i += kThreads)
        sts4(sbase + Lt::kOnesOff + 16 * i, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
    uint32_t *const table = reinterpret_cast<uint32_t *>(sm + Lt::kTableOff);
    for (int i = threadIdx.x; i < 256; i += kThreads) table[i] = pack_bf16(scale_of(i), scale_of(i));
    fence_async_smem();
    // The plan, from lengths that the kernel before may yet write: they are compared below.  Into L2 in the
    // meantime: the first pages (for nothing if the table then says others), the first queries.
    int P0 = 0, T0 = 0;
    if (warp == 0 && p.B <= 32) {
        if (lane < p.B) {
            P0 = prefix_of(p, lane);
            T0 = block_of(p, lane);
        }
        Plan pl;
        make_plan(p, pl, P0, T0);
        if (lane == 0) *s_plan = pl;
        const int page0 = 2 * pl.w.t + lane;
        if (lane < kPrefetch && pl.ntiles > 0 && page0 < (pl.w.P + kPage - 1) / kPage && page0 < 2 * (pl.w.t + pl.ntiles)) {
            const int pg = __ldcg(p.table + (size_t)pl.w.b * p.max_pages + page0);
            if (pg >= 0 && pg < p.pages) {
                const size_t tile = (size_t)pg * p.Hkv + pl.w.h;
                prefetch_bulk(p.k + tile * Lt::kCodes, Lt::kCodes);
                prefetch_bulk(p.v + tile * Lt::kCodes, Lt::kCodes);
                prefetch_bulk(p.k_scale + tile * Lt::kScales, Lt::kScales);
                prefetch_bulk(p.v_scale + tile * Lt::kScales, Lt::kScales);
            }
        }
        for (int r = lane; r < (pl.ntiles > 0 ? p.G * pl.w.T : 0); r += 32)
            for (int c = 0; c < D; c += 64)
                prefetch_line(p.q + (((size_t)pl.w.b * p.max_block + r / p.G) * p.Hq + pl.w.h * p.G + r % p.G) * D + c);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 0) {
        int P1 = 0, T1 = 0;
        if (p.B <= 32 && lane < p.B) {
            P1 = prefix_of(p, lane);
            T1 = block_of(p, lane);
        }
        if (p.B > 32 || !__all_sync(kFull, P0 == P1 && T0 == T1)) {
            Plan pl;
            make_plan(p, pl, P1, T1);
            if (lane == 0) *s_plan = pl;
        }
    }
    if (blockIdx.x == 0 && warp == 1)
        for (int b = lane; b < p.B; b += 32)
            if (__ldcg(p.prefix_len + b) != prefix_of(p, b) || __ldcg(p.block_len + b) != block_of(p, b))
                atomicOr(p.status, kStatusClamped);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = misc[0];
    Walk w = s_plan->w;
    const int ntiles = s_plan->ntiles;

    auto waits = [&](uint32_t bar, uint32_t parity) {
        return mbar_try_wait(bar, parity) || sleep_wait(bar, parity, abort_flag, p.status);
    };
    // Tile k of the range has buffers k % 2; of its prefix tiles, the kp-th has stage kp % kStages.
    auto half_of = [](int k) { return (uint32_t)(k >> 1) & 1; };
    int loaded = 0;  // (the producer's)
    if (warp == kProducerWarp) {
        // ================================ loads ==================================
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        bool ok = true;
        for (int left = ntiles; left > 0 && ok; walk_pair(p, w)) {
            const Segment s = segment_of(w, left);
            const int pages = (w.P + kPage - 1) / kPage;
            for (int i0 = 0; i0 < s.pre && ok; i0 += 16) {  // 32 pages at a time, one a lane
                const int at = 2 * (w.t + i0) + lane, n_here = min(16, s.pre - i0);
                int page = -1, n = 0;
                if (at < pages && lane < 2 * n_here) {
                    page = __ldcg(p.table + (size_t)w.b * p.max_pages + at);
                    if (page < 0 || page >= p.pages) {
                        atomicOr(p.status, kStatusBadPage);
                        page = -1;
                    } else {
                        n = min(kPage, w.P - at * kPage);
                    }
                }
                for (int i = 0; i < n_here; ++i) {
                    const int p0 = __shfl_sync(kFull, page, 2 * i), p1 = __shfl_sync(kFull, page, 2 * i + 1);
                    const int n0 = __shfl_sync(kFull, n, 2 * i), n1 = __shfl_sync(kFull, n, 2 * i + 1);
                    const int st = loaded % kStages;
                    if (loaded >= kStages)
                        ok = waits(b_empty + 8 * st, (uint32_t)(loaded / kStages - 1) & 1);
                    if (!ok) break;
                    if (elect_one()) {
                        infos[loaded % kInfos] = make_int2(n0, n1);
                        const uint32_t full = b_full + 8 * st, dst = sbase + st * Lt::kStage;
                        mbar_arrive_expect_tx(full, ((p0 >= 0) + (p1 >= 0)) * 2 * (Lt::kCodes + Lt::kScales));
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int pg = j ? p1 : p0;
                            if (pg < 0) continue;
                            const int tile = pg * p.Hkv + w.h;
                            tma_3d(dst + j * Lt::kCodes, &tm_k, full, 0, 0, tile, policy);
                            bulk_load(dst + Lt::kVOff + j * Lt::kCodes, p.v + (size_t)tile * Lt::kCodes, Lt::kCodes,
                                      full, policy);
                            bulk_load(dst + Lt::kKsOff + j * Lt::kScales, p.k_scale + (size_t)tile * Lt::kScales,
                                      Lt::kScales, full, policy);
                            bulk_load(dst + Lt::kVsOff + j * Lt::kScales, p.v_scale + (size_t)tile * Lt::kScales,
                                      Lt::kScales, full, policy);
                        }
                    }
                    __syncwarp();
                    ++loaded;
                }
            }
            left -= s.n;
        }
    } else if (warp == kSWarp) {
        // ============================= S^T = K Q^T ===============================
        constexpr uint32_t id = idesc_bf16(kKeys, N, 0, 0);
        bool ok = true;
        int k = 0;
        for (int seg = 0; k < ntiles && ok; ++seg, walk_pair(p, w)) {
            const int end = k + segment_of(w, ntiles - k).n;
            const uint64_t dq = sdesc(sbase + Lt::kQOff + (seg & 1) * Lt::kQ, 16, 1024, 2);
            ok = waits(b_qready + 8 * (seg & 1), half_of(seg));
            for (; k < end && ok; ++k) {
                const int s = k & 1;
                // S is free when P has been made of it.  Where the groups share the tiles, its product is waited for
                // instead, with time to spare: S being done then says that P's buffer is free.
                ok = waits(b_kready + 8 * s, half_of(k)) &&
                     (k < 2 || waits((kTurns ? b_pready : b_pvdone) + 8 * s, half_of(k) ^ 1));
                if (!ok) break;
                fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        mma_bf16_ta(tmem + kSCol + 64 * s, tmem + kKCol + 64 * s + 8 * kk,
                                    dq + (((kk >> 2) * (N * 128) + (kk & 3) * 32) >> 4), id, kk > 0);
                    mma_commit(b_sdone + 8 * s);
                    if (k + 1 == end) mma_commit(b_qfree + 8 * (seg & 1));
                }
                __syncwarp();
            }
        }
    } else if (warp == kPvWarp) {
        // ============================ O^T += V^T P^T =============================
        constexpr uint32_t id = idesc_bf16(kKeys, N, 0, 1), id_sum = idesc_bf16(64, 8, 1, 0);
        const uint64_t ones = sdesc(sbase + Lt::kOnesOff, 128, 256, 0);
        bool ok = true;
        int k = 0;
        for (; k < ntiles && ok; walk_pair(p, w)) {
            const Segment sg = segment_of(w, ntiles - k);
            for (int i = 0; i < sg.n && ok; ++i, ++k) {
                const int s = k & 1;
                ok = waits(b_vready + 8 * s, half_of(k)) && waits(b_pready + 8 * s, half_of(k));
                if (!ok) break;
                fence_after();
                if (elect_one()) {
                    const uint64_t dp = sdesc(sbase + Lt::kPOff + s * Lt::kP, Lt::kP, 1024, 2);
                    const int steps = i < sg.pre ? 8 : 4;  // (the block has 64 keys at most)
                    const uint32_t dO = tmem + kOCol + (kTurns ? 32 * s : 0), d_sum = tmem + kSumCol + (kTurns ? 8 * s : 0);
                    for (int kk = 0; kk < steps; ++kk)
                        mma_bf16_ta(dO, tmem + kVCol + 64 * s + 8 * kk, dp + ((kk * 2048) >> 4), id,
                                    i >= kStep || kk > 0);
                    for (int kk = 0; kk < steps; ++kk)
                        mma_bf16(d_sum, dp + ((kk * 2048) >> 4), ones, id_sum, i >= kStep || kk > 0);
                    mma_commit(b_pvdone + 8 * s);
                }
                __syncwarp();
            }
        }
    } else if (warp >= kValueWarp0) {
        // ============================ values, widened ============================
        // Thread (warp, lane): element d of a value; 32 elements share a scale.
        const int quad = warp % 4, set = (warp - kValueWarp0) / 4, d = quad * 32 + lane;
        const uint32_t dst = tmem + kVCol + ((uint32_t)(quad * 32) << 16);
        const bool mine = d < D;  // (a whole warp's)
        // the warp's scales of a tile, in pairs of keys: columns 2 lane and 2 lane + 1 are keys 8 o + q and
        // 8 o + q + 4, q = 2 (lane % 2) and one more
        uint2 *const scales = reinterpret_cast<uint2 *>(sm + Lt::kVsxOff) + (warp - kValueWarp0) * 32;
        const int at_o = lane >> 1, at_pg = at_o >> 3, at_q = 16 * (lane & 1);
        const Widen widen;
        const uint32_t m8 = 0xc308c308u;  // -136
        int k = 0, kp = 0;
        bool ok = true;
        for (; k < ntiles && ok; walk_pair(p, w)) {
            const Segment sg = segment_of(w, ntiles - k);
            for (int i = 0; i < sg.n && ok; ++i, ++k) {
                const int s = k & 1;
                if (kValueSets == 2 && s != set) {
                    kp += i < sg.pre;
                    continue;
                }
                if (i < sg.pre) {
                    const int st = kp % kStages;
                    const uint8_t *const stage = sm + st * Lt::kStage;
                    ok = waits(b_full + 8 * st, (uint32_t)(kp / kStages) & 1);
                    if (!ok) break;
                    if (mine) {
                        const int2 n = infos[kp % kInfos];
                        const int left = (at_pg ? n.y : n.x) - (at_o & 7) * 8;
                        uint2 by = *reinterpret_cast<const uint2 *>(stage + Lt::kVsOff + at_pg * Lt::kScales +
                                                                    quad * kPage + (at_o & 7) * 8);
                        if (left < 8) {  // places past the last token may hold anything
                            const unsigned long long keep = left <= 0 ? 0 : (1ull << 8 * left) - 1;
                            by.x &= (uint32_t)keep;
                            by.y &= (uint32_t)(keep >> 32);
                        }
                        __syncwarp();
                        const uint32_t b0 = by.x >> at_q, b1 = by.y >> at_q;
                        scales[lane] = make_uint2(__byte_perm(table[b0 & 0xffu], table[b1 & 0xffu], 0x5410),
                                                  __byte_perm(table[b0 >> 8 & 0xffu], table[b1 >> 8 & 0xffu], 0x5410));
                        __syncwarp();
                    }
                    if (k >= 2) ok = waits(b_pvdone + 8 * s, half_of(k) ^ 1);
                    if (!ok) break;
                    fence_after();
                    if (mine) {
                        const uint32_t *words = reinterpret_cast<const uint32_t *>(stage + Lt::kVOff) + d;
                        const uint4 *f = reinterpret_cast<const uint4 *>(scales);
                        uint32_t word[4];
                        uint4 sc[4];
                        auto load = [&] {
#pragma unroll
                            for (int o = 0; o < 4; ++o) {
                                word[o] = words[o * D];
                                sc[o] = f[o];
                            }
                            words += 4 * D;
                            f += 4;
                        };
                        load();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {  // half a page's keys: 16 columns
                            uint32_t r[16];
#pragma unroll
                            for (int o = 0; o < 4; ++o) {
                                uint32_t h[4];
                                widen(word[o], h);
                                r[4 * o] = bf16_mul2(bf16_add2(h[0], m8), sc[o].x);
                                r[4 * o + 1] = bf16_mul2(bf16_add2(h[1], m8), sc[o].y);
                                r[4 * o + 2] = bf16_mul2(bf16_add2(h[2], m8), sc[o].z);
                                r[4 * o + 3] = bf16_mul2(bf16_add2(h[3], m8), sc[o].w);
                            }
                            if (c < 3) load();  // (no load is moved over a store)
                            st_lanes(dst + 64 * s + 16 * c, r);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_empty + 8 * st);
                    ++kp;
                } else {  // the block's own, in units of the stored ones' (exact, but for what is past bf16's range)
                    if (k >= 2) ok = waits(b_pvdone + 8 * s, half_of(k) ^ 1);
                    if (!ok) break;
                    fence_after();
                    if (mine) {
                        const float unit = 1.f / unit_of(p.v_unit, w.h);
                        const uint16_t *src = p.v_blk + ((size_t)w.b * p.max_block * p.Hkv + w.h) * D + d;
                        int nf = kKeys;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {  // 16 keys: 8 columns
                            uint32_t r[8];
#pragma unroll
                            for (int o = 0; o < 2; ++o) {
                                const int key = 16 * c + 8 * o;
                                float x[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    x[j] = key + j < w.T ? __uint_as_float((uint32_t)src[(size_t)(key + j) * p.Hkv * D] << 16)
                                                         : 0.f;
#pragma unroll
                                for (int j = 7; j >= 0; --j)
                                    if (!(fabsf(x[j]) < INFINITY)) {
                                        nf = min(nf, key + j);
                                        x[j] = 0.f;
                                    }
#pragma unroll
                                for (int j = 0; j < 4; ++j) r[4 * o + j] = pack_bf16_finite(x[j] * unit, x[j + 4] * unit);
                            }
                            st_lanes(dst + 64 * s + 8 * c, r);
                        }
                        s_nf[(k & 3) * kKeys + d] = nf;
                    }
                }
                st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_vready + 8 * s);
            }
        }
    } else if (warp >= kKeyWarp0) {
        // ======================== queries; keys, widened =========================
        // Thread (warp, lane): a key of the tile.
        const int quad = warp % 4, key = quad * 32 + lane;
        const Widen widen;
        const uint32_t dst = tmem + kKCol + ((uint32_t)(quad * 32) << 16);
        int k = 0, kp = 0;
        bool ok = true;
        for (int seg = 0; k < ntiles && ok; ++seg, walk_pair(p, w)) {
            const Segment sg = segment_of(w, ntiles - k);
            // the queries
            if (seg >= 2) ok = waits(b_qfree + 8 * (seg & 1), half_of(seg) ^ 1);
            if (!ok) break;
            const uint32_t q = sbase + Lt::kQOff + (seg & 1) * Lt::kQ;
            constexpr int kPerRow = D / 8;
            const int rows = p.G * w.T;
#pragma unroll 4
            for (int i = key; i < N * kPerRow; i += kKeys) {
                const int r = i / kPerRow, c = i % kPerRow;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (r < rows)
                    x = *reinterpret_cast<const uint4 *>(
                        p.q + (((size_t)w.b * p.max_block + r / p.G) * p.Hq + w.h * p.G + r % p.G) * D + c * 8);
                x = paired(x);
                sts4(q + (c >> 3) * (N * 128) + chunk16(r, c & 7), x.x, x.y, x.z, x.w);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_qready + 8 * (seg & 1));
            for (int i = 0; i < sg.n && ok; ++i, ++k) {
                const int s = k & 1;
                if (k >= 2) ok = waits(b_sdone + 8 * s, half_of(k) ^ 1);
                if (!ok) break;
                if (i < sg.pre) {
                    const int st = kp % kStages;
                    const uint8_t *const stage = sm + st * Lt::kStage;
                    ok = waits(b_full + 8 * st, (uint32_t)(kp / kStages) & 1);
                    if (!ok) break;
                    fence_after();
                    const int pg = key / kPage, t = key % kPage;
                    const uint8_t *const at_scale = stage + Lt::kKsOff + pg * Lt::kScales + t * (D / 32);
                    const uint32_t by = D == 128 ? *reinterpret_cast<const uint32_t *>(at_scale)
                                           : *reinterpret_cast<const uint16_t *>(at_scale);
                    uint4 codes[D / 32];
                    uint32_t scs[D / 32];
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) scs[c] = table[by >> 8 * c & 0xffu];
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
                        codes[c] = *reinterpret_cast<const uint4 *>(stage + pg * Lt::kCodes + key_chunk<D>(t, c));
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {  // 32 elements under a scale
                        const uint4 x = codes[c];
                        const uint32_t sc = scs[c], m8 = bf16_mul2(sc, 0xc308c308u);  // -136
                        const uint32_t word[4] = {x.x, x.y, x.z, x.w};
                        uint32_t r[16];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t h[4];
                            widen(word[j], h);
#pragma unroll
                            for (int e = 0; e < 4; ++e) r[4 * j + e] = bf16_fma2(h[e], sc, m8);
                        }
                        st_lanes(dst + 64 * s + 16 * c, r);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_empty + 8 * st);
                    ++kp;
                } else {  // the block's own (S of keys past it is not looked at)
                    fence_after();
                    if (quad < 2) {
                        const uint4 *src = reinterpret_cast<const uint4 *>(
                            p.k_blk + (((size_t)w.b * p.max_block + key) * p.Hkv + w.h) * D);
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t r[16];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint4 x = make_uint4(0, 0, 0, 0);
                                if (key < w.T) x = src[4 * c + j];
                                x = paired(x);
                                r[4 * j] = x.x;
                                r[4 * j + 1] = x.y;
                                r[4 * j + 2] = x.z;
                                r[4 * j + 3] = x.w;
                            }
                            st_lanes(dst + 64 * s + 16 * c, r);
                        }
                    }
                }
                st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_kready + 8 * s);
            }
        }
    } else {
        // ================================ softmax ================================
        // Thread (warp, lane): a key of a tile; rows [row0, row0 + R).
        const int group = warp / kGroupWarps, quad = warp % kGroupWarps, key = quad * 32 + lane;
        const int bar = 1 + group, row0 = kTurns ? 0 : group * R;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t o_col = lanes + kOCol + (kTurns ? 32 * group : row0);
        // the row whose rounded weights' sum this lane has, in the group's one of the equal columns
        const uint32_t sum_col = lanes + kSumCol + (kTurns ? 8 * group : group);
        const int sum_row = 16 * quad + lane;
        const bool sum_mine = lane < 16 && sum_row >= row0 && sum_row < row0 + R;
        const int place = (key & ~7) | (key & 3) << 1 | (key >> 2 & 1);  // of the key among P's rows
        float *const off = s_off + 64 * group, *const alpha = s_alpha + 64 * group;
        float *const group_sums = reinterpret_cast<float *>(sm + Lt::kSumOff) + group * (kGroupWarps * 32),
                     *const sums = group_sums + quad * 32;
        auto group_sync = [&] { asm volatile("bar.sync %0, 128;" ::"r"(bar) : "memory"); };
        auto all_sync = [&] { asm volatile("bar.sync 3, 256;" ::: "memory"); };
        long long q_pair = s_plan->q;
        int k_seg = 0, kp_seg = 0;
        int joins = 0;  // (thread 0's)
        for (; k_seg < ntiles; q_pair += w.nt + kEnd, walk_pair(p, w)) {
            const Segment sg = segment_of(w, ntiles - k_seg);
            const int rows = p.G * w.T;
            const float sc_page = fmaxf(p.scale_log2 * unit_of(p.k_unit, w.h), 1.2e-38f);
            const float v_unit = unit_of(p.v_unit, w.h);
            float l[R];
#pragma unroll
            for (int j = 0; j < R; ++j) l[j] = 0.f;
            bool has_ref = false;  // the same in the whole group
#pragma unroll 1
            for (int i = kTurns ? (k_seg ^ group) & 1 : 0; i < sg.n; i += kStep) {
                const int k = k_seg + i, s = kTurns ? group : k & 1;
                const bool blk = i >= sg.pre;
                const bool ok = waits(b_sdone + 8 * s, half_of(k));
                fence_after();
                const float sc = blk ? p.scale_log2 : sc_page;
                int2 n = make_int2(kPage, kPage);
                if (!blk) n = infos[(kp_seg + i) % kInfos];
                // hidden keys: of pages past the prefix, of the block past it or the row (key i is seen by the
                // rows from i G on)
                const bool some_hidden = blk || n.x + n.y < kKeys || !ok;
                int from = 0, until = N;
                if (some_hidden) {
                    from = !ok ? N : blk ? (key < w.T ? key * p.G : N) : key % kPage < (key < kPage ? n.x : n.y) ? 0 : N;
                    if (blk) until = rows;
                }
                const uint32_t s_col = lanes + kSCol + 64 * s + row0;
                auto scores = [&](int c, uint32_t(&a)[kChunk]) {
                    ld_lanes(s_col + c, a);
                    ld_wait(a);
                    if (some_hidden)
#pragma unroll
                        for (int j = 0; j < kChunk; ++j)
                            if (row0 + c + j < from || row0 + c + j >= until) a[j] = 0xff800000u;
                };
                if (!has_ref) {
                    // the segment's first key that is seen, if this tile has one
                    const int first = n.x > 0 ? 0 : n.y > 0 ? kPage : -1;
#pragma unroll 1
                    for (int c = 0; c < R; c += kChunk) {
                        uint32_t a[kChunk];
                        scores(c, a);
                        if (key == max(first, 0))
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) {
                                const float m = __uint_as_float(a[j]) * sc;
                                // (of one of -inf, below all others, so that the reference moves)
                                off[row0 + c + j] = fmaxf(fminf(-m, kMost), -kMost) - kBelow;
                            }
                    }
                    group_sync();
                    has_ref = first >= 0;
                }
                if (kTurns && k >= 2) waits(b_pvdone + 8 * s, half_of(k) ^ 1);  // P's buffer is free
                const uint32_t dst = sbase + Lt::kPOff + s * Lt::kP + place * 128, turn = (place & 7) << 4;
                // (all exponentials of a chunk first, so that their chains overlap)
                auto weights = [&](int c, uint32_t(&a)[kChunk]) {
#pragma unroll
                    for (int j = 0; j < kChunk; j += 4) {
                        const float4 o = *reinterpret_cast<const float4 *>(off + row0 + c + j);
                        float e[4];
                        axpy2(e[0], e[1], sc, __uint_as_float(a[j]), __uint_as_float(a[j + 1]), o.x, o.y);
                        axpy2(e[2], e[3], sc, __uint_as_float(a[j + 2]), __uint_as_float(a[j + 3]), o.z, o.w);
#pragma unroll
                        for (int t = 0; t < 4; ++t) a[j + t] = __float_as_uint(ex2(e[t]));
                    }
                    uint32_t big = 0;
#pragma unroll
                    for (int j = 0; j < kChunk; j += 8) {
                        uint32_t pk[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            pk[t] = pack_bf16(__uint_as_float(a[j + 2 * t]), __uint_as_float(a[j + 2 * t + 1]));
                        big |= pk[0] | pk[1] | pk[2] | pk[3];
                        sts4(dst + ((uint32_t)((row0 + c + j) / 8 * 16) ^ turn), pk[0], pk[1], pk[2], pk[3]);
                    }
                    return big;
                };
                uint32_t big = 0;
#pragma unroll
                for (int c = 0; c < R; c += kChunk) {
                    uint32_t a[kChunk];
                    scores(c, a);
                    big |= weights(c, a);
#pragma unroll
                    for (int j = 0; j < kChunk; j += 2)
                        add2(l[c + j], l[c + j + 1], l[c + j], l[c + j + 1], __uint_as_float(a[j]), __uint_as_float(a[j + 1]));
                }
                fence_async_smem();
                uint32_t over;
                asm volatile(
                    "{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n"
                    " barrier.cta.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}"
                    : "=r"(over)
                    : "r"(big & 0x40004000u), "r"(bar)
                    : "memory");
                if (over) {
                    // A weight of 2 or more: its row's reference is set to the tile's largest score, and O and the
                    // sums are rescaled, by two factors as one could be 0 where the product is not.  (l has the
                    // tile's weights under the old reference already; where one made it infinite, what it was
                    // before counts nothing.)
#pragma unroll 1
                    for (int c = 0; c < R; c += kChunk) {
                        uint32_t a[kChunk];
                        scores(c, a);
#pragma unroll
                        for (int j = 0; j < kChunk; ++j) {
                            const float x = __uint_as_float(a[j]) * sc;
                            const uint32_t m = __reduce_max_sync(kFull, ordered(x == x ? x : -INFINITY));
                            if (lane == 0) sums[c + j] = unordered(m);
                        }
                    }
                    group_sync();
                    if (quad == 0 && lane < R) {
                        float m = -INFINITY;
                        for (int v = 0; v < kGroupWarps; ++v) m = fmaxf(m, group_sums[v * 32 + lane]);
                        const float was = off[row0 + lane];
                        const bool jump = m + was >= 1.f && m < INFINITY;
                        if (jump) off[row0 + lane] = -m - kBelow;
                        alpha[row0 + lane] = jump ? ex2(0.5f * (-m - kBelow - was)) : 1.f;
                    }
                    group_sync();
                    if (i >= kStep) {
                        waits(b_pvdone + 8 * (k - kStep & 1), half_of(k - kStep));
                        fence_after();
#pragma unroll 1
                        for (int c = 0; c < R; c += 8) {
                            uint32_t o[8];
                            ld_lanes(o_col + c, o);
                            ld_wait(o);
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha[row0 + c + j] * alpha[row0 + c + j]);
                            st_lanes(o_col + c, o);
                        }
                        uint32_t o[1];
                        ld_lanes(sum_col, o);
                        ld_wait(o);
                        if (sum_mine) o[0] = __float_as_uint(__uint_as_float(o[0]) * alpha[sum_row] * alpha[sum_row]);
                        st_lanes(sum_col, o);
                        st_wait();
                    }
#pragma unroll
                    for (int c = 0; c < R; c += kChunk) {
                        uint32_t a[kChunk];
                        scores(c, a);
                        weights(c, a);
#pragma unroll
                        for (int j = 0; j < kChunk; ++j)
                            {
                            const float f = alpha[row0 + c + j];
                            l[c + j] = l[c + j] == INFINITY ? __uint_as_float(a[j]) : l[c + j] * f * f;
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                }
                fence_before();
                if (lane == 0) mbar_arrive(b_pready + 8 * s);
            }

            // ---- the end of a segment: O / l and lse, as output or as a partial ----
            // l of row j over the warp's keys, in lane j (R lanes)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                if (2 * d > R) {
#pragma unroll
                    for (int j = 0; j < R; ++j) l[j] += __shfl_xor_sync(kFull, l[j], d);
                } else {
#pragma unroll
                    for (int j = 0; j < R / 2; ++j)
                        if (j < d) {
                            const bool up = lane & d;
                            const float give = up ? l[j] : l[j + d], keep = up ? l[j + d] : l[j];
                            l[j] = keep + __shfl_xor_sync(kFull, give, d);
                        }
                }
            }
            if (lane < R) sums[lane] = l[0];
            // with turns, a group may have none of the segment's tiles
            const bool had = !kTurns || sg.n > 1 || (k_seg & 1) == group;
            const int last = k_seg + sg.n - 1;
            if (had) {
                const int mine = kTurns && (last & 1) != group ? last - 1 : last;
                waits(b_pvdone + 8 * (mine & 1), half_of(mine));
                fence_after();
                uint32_t o[1];
                ld_lanes(sum_col, o);
                ld_wait(o);
                if (sum_mine) alpha[sum_row] = __uint_as_float(o[0]);
            }
            group_sync();
            if (quad == 0 && lane < R) {
                float sum = 0.f;
                for (int v = 0; v < kGroupWarps; ++v) sum += group_sums[v * 32 + lane];
                s_total[64 * group + row0 + lane] = had ? sum : 0.f;
                if (!has_ref) off[row0 + lane] = INFINITY;
                if (!had) alpha[row0 + lane] = 0.f;
            }
            // from here a group has the rows [orow0, orow0 + kOut) of the output
            constexpr int kOut = N / 2;
            const int orow0 = group * kOut;
            if (kTurns) {
                all_sync();
                // Both groups read both O below: each thread sees the last products of either complete itself, as the
                // barrier does not order tensor memory.  (After it, as the phase before those has then ended.)
                waits(b_pvdone + 8 * (last & 1), half_of(last));
                if (sg.n > 1) waits(b_pvdone + 8 * (last - 1 & 1), half_of(last - 1));
                fence_after();
            } else {
                group_sync();
            }
            const bool has_blk = sg.n > sg.pre, whole = w.t == 0 && has_blk;
            if (quad == 0 && lane < kOut) {
                const int r = orow0 + lane;
                float f[2] = {0.f, 0.f}, total = 0.f, sum = 0.f, least;
                if (kTurns) {  // both groups' under the larger reference
                    least = fminf(s_off[r], s_off[64 + r]);
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const float mine = s_off[64 * g + r];
                        f[g] = mine == INFINITY ? 0.f : ex2(least - mine);
                        total += f[g] * s_total[64 * g + r];
                        sum += f[g] * s_alpha[64 * g + r];
                    }
                } else {
                    least = off[r];
                    f[0] = 1.f;
                    total = s_total[64 * group + r];
                    sum = alpha[r];
                }
                // no visible key: 0 and -inf; NaN stays NaN
                const float inv = total == 0.f ? 0.f : v_unit / sum;
                s_factor[r] = f[0] * inv;
                s_factor[64 + r] = f[1] * inv;
                s_lse[r] = total == 0.f ? -INFINITY : log2f(total) - least;
            }
            group_sync();
            const size_t pair = (size_t)w.b * p.Hkv + w.h;
            const size_t slot = pair + blockIdx.x;
            if (quad * 32 < D) {
                const int k_last = k_seg + sg.n - 1;
                const int nf = has_blk ? s_nf[(k_last & 3) * kKeys + key] : kKeys;  // (key: the element d here)
                const bool two = kTurns && sg.n > 1, second = kTurns && (k_seg & 1);  // whose O the first tile's is
                const float *const f0 = s_factor + (second ? 64 : 0), *const f1 = s_factor + (second ? 0 : 64);
                const uint32_t o0 = lanes + kOCol + orow0 + (second ? 32 : 0), o1 = lanes + kOCol + orow0 + (second ? 0 : 32);
#pragma unroll 1
                for (int c = 0; c < kOut && orow0 + c < p.rows_max; c += 8) {
                    uint32_t o[8];
                    float x[8];
                    ld_lanes(o0 + c, o);
                    ld_wait(o);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(o[j]) * f0[orow0 + c + j];
                    if (two) {
                        ld_lanes(o1 + c, o);
                        ld_wait(o);
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[j] += __uint_as_float(o[j]) * f1[orow0 + c + j];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (orow0 + c + j >= nf * p.G) x[j] = __uint_as_float(0x7fffffffu);
                    if (whole) {
                        // lane d has rows r and r + 1 of element d: an even lane stores row r's two elements, an
                        // odd one row r + 1's
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const bool odd = lane & 1;
                            const float got = __shfl_xor_sync(kFull, odd ? x[j] : x[j + 1], 1);
                            const int r = orow0 + c + j + odd, i = r / p.G;
                            if (r < p.rows_max)
                                *reinterpret_cast<uint32_t *>(
                                    p.out + (((size_t)w.b * p.max_block + i) * p.Hq + w.h * p.G + r % p.G) * D + (key & ~1)) =
                                    r < rows ? (odd ? pack_bf16(got, x[j + 1]) : pack_bf16(x[j], got)) : 0u;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int r = orow0 + c + j;
                            if (r < rows) p.part_o[(slot * p.rows_max + r) * D + key] = x[j];
                        }
                    }
                }
            }
            fence_before();
            if (quad == 3 && lane < kOut && orow0 + lane < p.rows_max) {
                const int r = orow0 + lane;
                if (whole)
                    p.lse[((size_t)w.b * p.Hq + w.h * p.G + r % p.G) * p.max_block + r / p.G] =
                        r < rows ? s_lse[r] * kLn2 : -INFINITY;
                else
                    p.part_lse[slot * p.rows_max + r] = r < rows ? s_lse[r] : -INFINITY;
            }
            all_sync();  // (the rows' arrays, and with turns the other group's O, may be written again)
            if (!whole && threadIdx.x == 0) {
                // Whoever comes last at its run's counter joins the run when its tiles are done.
                // With more than kFan partials a pair's are cut into runs of about as many as there are runs.
                const Plan &pl = *s_plan;
                const int c0 = cta_of(pl, q_pair), n = cta_of(pl, q_pair + w.nt - 1) - c0 + 1;
                int run = n;
                if (n > kFan) {
                    run = 2;
                    while (run * run < n) ++run;
                }
                const int r0 = ((int)blockIdx.x - c0) / run * run, count = min(run, n - r0);
                __threadfence();  // (for the other threads' stores too, which the barrier puts before)
                int32_t *const counter = p.counts + (r0 == 0 ? c0 : p.num_ctas + c0 + r0);
                if (atomicAdd(counter, 1) == count - 1) {
                    *counter = 0;
                    __threadfence();
                    s_joins[joins++] = {(int)pair, rows, c0, n, run, r0};
                }
            }
            k_seg += sg.n;
            kp_seg += sg.pre;
        }
        if (threadIdx.x == 0) misc[2] = joins;
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*abort_flag) {  // a timed-out run: products and copies may be in flight yet
        if (warp == kSWarp || warp == kPvWarp) {
            const uint32_t drain = b_drain + (warp == kSWarp ? 8 : 0);
            if (elect_one()) mma_commit(drain);
            __syncwarp();
            drain_wait(drain, 0);
        }
        if (warp == kProducerWarp && elect_one())
            for (int j = loaded - 1; j >= 0 && j >= loaded - kStages; --j)
                drain_wait(b_full + 8 * (j % kStages), (uint32_t)(j / kStages) & 1);
        __syncwarp();
        fence_before();
        __syncthreads();
        fence_after();
    }
    // (else the softmax warps have seen every product's completion)
    if (warp == kSWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols));
    // ---- partials joined, by all of the CTA ----
    for (int j = 0, n = misc[2]; j < n; ++j) {
        const Join jn = s_joins[j];
        const size_t first = (size_t)jn.pair + jn.c0;
        const int runs = (jn.n + jn.run - 1) / jn.run;
        join<D>(p, jn, first + jn.r0, 1, min(jn.run, jn.n - jn.r0), runs == 1, s_lse);
        if (runs == 1) continue;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            int32_t *const counter = p.counts + 2 * p.num_ctas + jn.c0;
            const bool last = atomicAdd(counter, 1) == runs - 1;
            if (last) *counter = 0;
            __threadfence();
            misc[3] = last;
        }
        __syncthreads();
        if (misc[3]) join<D>(p, jn, first, jn.run, runs, true, s_lse);
    }
}

size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

template <int D, int N>
cudaError_t launch(const Paged4AttnParams &p, const CUtensorMap &tm_k, cudaStream_t stream) {
    constexpr int smem = Layout<D, N>::kBytes;
    static std::atomic<bool> configured[64];  // the shared-memory opt-in, once per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(paged4_attn_kernel<D, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.num_ctas);
    cfg.blockDim = dim3(Roles<N>::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, paged4_attn_kernel<D, N>, tm_k, p);
}

template <int D>
cudaError_t launch_d(const Paged4AttnParams &p, const CUtensorMap &tm_k, cudaStream_t stream) {
    return p.rows_max <= 16   ? launch<D, 16>(p, tm_k, stream)
           : p.rows_max <= 32 ? launch<D, 32>(p, tm_k, stream)
                              : launch<D, 64>(p, tm_k, stream);
}

}  // namespace

// header | counters [3][C] | part_lse [slots][rows_max] | part_o [slots][rows_max][D], slots = pairs + C (a
// segment's slot is its pair + its CTA).
// Counters are 0 between calls, and lie in the same place for every shape, so that no call's partials lie over
// another's.  They go by CTAs: a pair of several segments has tiles on both sides of the border after its first CTA c0
// and of that before each other, and no two pairs lie across one border.  So [0][c0] is the run of segments
// that begins with the pair's first, [1][c] a run that begins with a later CTA c, and [2][c0] the pair's runs.
constexpr int kCounters = 3;

size_t paged4_workspace_bytes(int device, int batch, int kv_heads, int rows_max, int head_dim) {
    const int C = attn_grid_size(device);
    if (C <= 0) return 0;
    const size_t slots = (size_t)batch * kv_heads + (size_t)C;
    return kWorkspaceHeader + round256(kCounters * C * sizeof(int32_t)) + round256(slots * rows_max * sizeof(float)) +
           round256(slots * rows_max * head_dim * sizeof(float));
}

cudaError_t paged4_attn_launch(Paged4AttnParams &p, int head_dim, const CUtensorMap &tm_k, void *workspace,
                               cudaStream_t stream) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    p.num_ctas = attn_grid_size(dev);
    if (p.num_ctas <= 0) return cudaErrorInvalidDevice;
    const size_t slots = (size_t)p.B * p.Hkv + (size_t)p.num_ctas;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    p.status = reinterpret_cast<int32_t *>(ws);
    ws += kWorkspaceHeader;
    p.counts = reinterpret_cast<int32_t *>(ws);
    ws += round256(kCounters * p.num_ctas * sizeof(int32_t));
    p.part_lse = reinterpret_cast<float *>(ws);
    p.part_o = reinterpret_cast<float *>(ws + round256(slots * p.rows_max * sizeof(float)));
    return head_dim == 128 ? launch_d<128>(p, tm_k, stream) : launch_d<64>(p, tm_k, stream);
}

}  // namespace das
