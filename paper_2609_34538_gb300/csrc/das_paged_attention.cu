// das_paged_attention.cu -- depth-asynchronous attention (Eqs. 2-3) over the
// paged e4m3 cache with a scale per (page, kv head), on the 5th-generation
// tensor cores of sm_103a with the codes as they are stored.
//
// The mathematics.  With s_j = scale ks(page) q . kc_j (base 2) and values
// vs(page) vc_j, a running reference m over x_j = s_j + log2 vs and
//     p_j = 2^(x_j - m + kHead),
// O = sum_j p_j vc_j and l = sum_j p_j / vs give o = O / l and
// lse = ln 2 (m - kHead + log2 l): a page's value scale is part of the weight
// that its codes are multiplied with, so the products run on the codes alone.
// m moves (O and l are rescaled) only when a thread's weights of a tile sum to
// more than kMost = 2^13, so that no weight is above 2^13 and all parts of one fit
// their types; it is then set to where the row's weights of the tile sum to 2^7 to 2^8.
//
// The operands of an 8-bit product have 3 or 4 significant bits, which is too few
// for queries and weights, so each is split into parts:
//   queries  2^e q = hi + lo / 16, both e4m3, two rows of one M = 128 product,
//            exact for elements down to about 2^-13 of the row's largest (a
//            bf16 value has 8 significant bits); S = S_hi + S_lo / 16, added
//            where the scores are read;
//   weights  p = a + (b + c) / 64, all e5m2 (which A may be beside an e4m3 B): a
//            and b two rows of one product, c a second product into b's rows;
//            O = O_hi + O_lo / 64, added at the end of a segment.  Off by 2^-9 of
//            p, as bf16 weights are, down to p = 2^-14, which is 2^-21 of the tile's
//            sum, and below by 2^-6 of p or 2^-30 of that sum: what one dominant key
//            leaves to thousands of others is kept.  Two e4m3 parts, whose range ended
//            2^-17 below the reference, lost most of that; they took 53.3 us where
//            three take 55.4 (4 x 32768 tokens).  Values widened to f16 in shared
//            memory, 16 KB more written and 8 more read a tile, took 60.7.
// Row r of the pair (r = i * G + g) has its hi (a) part in TMEM lane
// 32 (r / 16) + r % 16 and its lo (b, c) parts 16 lanes on, in the same warp's reach.
//
// Work split: every (sequence, kv head) pair owns one tile for each of its
// ceil(P / 64) pages plus one for the block's own keys.  There are two ways:
//   clusters  a cluster of 1 to 8 CTAs to a pair, a CTA to a share of its tiles;
//             the partials (O / l, lse) go into the shared memory of the CTA that
//             joins their row;
//   the list  of all pairs' tiles, of which CTA c of a persistent grid (one per
//             SM) takes the c-th of C equal ranges, cut into segments at pair
//             boundaries; a segment that is a whole pair writes the output, others a
//             partial, which paged_merge_kernel (or paged_merge_many_kernel) joins.
//             Many short pairs are split into ranges of whole pairs instead.
// log_cluster_of and launch_d say which, with both measured.
//
// What bounds it: 4 sequences of 32768 tokens, 32 / 8 heads of 128 and blocks of 16
// take 55.4 us, 4.8 TB/s of codes (bare TMA reads of the same tiles: 48.8 us); a tile
// of 16 KB takes a CTA 0.39 us, the pace of the softmax groups below.  One
// sequence of 4096 tokens with 32 heads takes 14.2 us (blocks of 1) and 14.6 us (8),
// of which the tiles take 6 to 7; the smallest calls 5.9 us.
//
// One CTA = two groups of four softmax warps, which take turns at the tiles
// (one warp per sub-partition left its latencies bare), + one TMA warp + two
// MMA warps + four warps that prepare each segment's queries (split) and block
// keys and values (bf16, with rows past the block zero).  The block tile runs
// bf16 products: S with M = 64 (the hi lanes), P V with P split into two bf16 parts.
// The kernel is launched as a programmatic dependent: barrier set-up, the
// tensor-memory allocation, the plan (from lengths read before the dependency
// wait, read again after it) and L2 prefetches of the first tiles and queries
// overlap the previous kernel's tail; nothing read before the wait is used
// unchecked.  Every wait is bounded (2 s); a time-out sets the status word and
// ends the CTA's waits.  Tensor memory is freed before the CTA exits.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "das_internal.h"
#include "das_tcgen05.h"

namespace das {
namespace {

using namespace t5;

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kGroupWarps = 4;     // softmax warps of one group, a TMEM quadrant each
constexpr int kGroups = 2;         // group g takes the tiles k with k % 2 = g
constexpr int kSoftWarps = kGroups * kGroupWarps;
constexpr int kProducerWarp = kSoftWarps;
constexpr int kPvWarp = kProducerWarp + 1;
constexpr int kSWarp = kPvWarp + 1;
constexpr int kQueryWarp0 = kSWarp + 1;
constexpr int kQueryWarps = 4;
constexpr int kThreads = (kQueryWarp0 + kQueryWarps) * 32;
constexpr int kRows = 64;          // query rows per pair
constexpr int kSBufs = 3;          // S buffers in tensor memory
constexpr int kTmemCols = 512;     // S [0, 192), each group's O, each group's P (2 x 16 columns)
constexpr int kOCol = kSBufs * kTileKeys;
constexpr int kOStep = 128;
constexpr int kPCol = kOCol + kGroups * kOStep;
constexpr int kPStep = 32;
static_assert(kPCol + kGroups * kPStep == kTmemCols, "tensor memory");
// A new reference leaves the row of the tile a sum of 2^kSumLog to twice that, which 64
// equal weights of 2^kHead have.  The lower, the more the sums may grow before the
// next one; the higher, the more of small weights is kept (kSumLog 6, 7, 8, 10, kHead
// 6 less: 54.3, 55.4, 57.7, 63.9 us for 4 x 32768 tokens whose pages' scores and
// values differ in size by a factor of 4).
constexpr int kSumLog = 7;
constexpr float kHead = 1.f, kMost = 8192.f;
constexpr float kQLoInv = 1.f / 16.f, kPLo = 64.f, kPLoInv = 1.f / kPLo;
constexpr uint32_t kPLo2 = 0x54005400u;   // f16x2 of kPLo
constexpr uint32_t kLoLanes = 16u << 16;
constexpr int kPrefetch = 4;       // pages pulled into L2 before the dependency wait

// Four weights, f16 pairs x and y (0 to kMost), as three e5m2 parts each: p = a +
// (b + c) / kPLo.  Each part leaves 2^-3 at most of what it rounds, so p is off by 2^-9 of
// itself down to 2^-14, where a ends, and below by 2^-6 of itself or 2^-23 (a multiple of
// b's least number).  kPLo times what a leaves is 2^15 at most.  The differences are exact.
struct Parts {
    uint32_t a, b, c;
};
__device__ __forceinline__ Parts parts_of(uint32_t x, uint32_t y) {
    Parts r;
    uint32_t u, v;
    r.a = e5m2x4_f16(x, y);
    f16_e5m2x4(r.a, u, v);
    x = hmul2(hsub2(x, u), kPLo2);
    y = hmul2(hsub2(y, v), kPLo2);
    r.b = e5m2x4_f16(x, y);
    f16_e5m2x4(r.b, u, v);
    r.c = e5m2x4_f16(hsub2(x, u), hsub2(y, v));
    return r;
}

// ---- tile list --------------------------------------------------------------------
__device__ __forceinline__ int clamp_to(int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); }
__device__ __forceinline__ int prefix_of(const PagedAttnParams &p, int b) {
    return clamp_to(__ldcg(p.prefix_len + b), p.max_pages * kTileKeys);
}
__device__ __forceinline__ int block_of(const PagedAttnParams &p, int b) {
    return clamp_to(__ldcg(p.block_len + b), p.max_block);
}
__device__ __forceinline__ int tiles_of(int P) { return (P + kTileKeys - 1) / kTileKeys + 1; }

// The lengths of up to kLens sequences are kept in shared memory (prefixes,
// then blocks); with more sequences, they are read where they are needed.
constexpr int kLens = 32;

struct Walk {
    int b, h, t, nt, P, T;
    const int *lens;  // shared memory, or null
};
__device__ __forceinline__ void walk_load(const PagedAttnParams &p, Walk &w) {
    if (w.b < p.B) {
        w.P = w.lens ? w.lens[w.b] : prefix_of(p, w.b);
        w.T = w.lens ? w.lens[kLens + w.b] : block_of(p, w.b);
        w.nt = tiles_of(w.P);
    }
}
__device__ __forceinline__ void walk_pair(const PagedAttnParams &p, Walk &w) {
    w.t = 0;
    if (++w.h == p.Hkv) {
        w.h = 0;
        ++w.b;
        walk_load(p, w);
    }
}
// Tile x of pair n has weighted position x + beta n; CTA c takes the tiles at
// [c W / C, (c + 1) W / C).  The end of a pair (its block tile, the joining of
// the groups, the next pair's start) costs a CTA about as much as nine pages, so
// a range that holds one takes beta tiles fewer (weights 3, 5, 7, 9, 12: 57.6,
// 56.9, 56.4, 55.7, 56.2 us for 4 x 32768 tokens, 49.9, 45.7, 46.1, 45.4, 44.9
// for 16 ragged sequences); beta = 0 with more pairs than CTAs (nearly every
// range then holds one) or where a CTA could stay empty.
constexpr int kBlockWeight = 9;
struct Split {
    long long N, W;
    int beta;
};
__device__ __forceinline__ Split split_of(const PagedAttnParams &p, long long tiles) {
    const long long pairs = (long long)p.B * p.Hkv;
    Split s;
    s.N = tiles;
    s.beta = pairs <= p.num_ctas &&
                     tiles + kBlockWeight * pairs >= (long long)(2 + kBlockWeight) * p.num_ctas
                 ? kBlockWeight
                 : 0;
    s.W = tiles + s.beta * pairs;
    return s;
}
__device__ __forceinline__ long long udiv(long long a, long long b) {
    if ((((unsigned long long)a | (unsigned long long)b) >> 32) == 0)
        return (long long)((uint32_t)a / (uint32_t)b);
    return a / b;
}
// the CTA whose range holds weighted position q
__device__ __forceinline__ int cta_of(long long q, const Split &s, int C) {
    return (int)udiv((q + 1) * C - 1, s.W);
}
__device__ __forceinline__ int seq_tiles(const PagedAttnParams &p, int b) {
    return b < p.B ? tiles_of(prefix_of(p, b)) : 0;
}

// This CTA's number of tiles and its first one (a whole warp executes this).
__device__ int plan(const PagedAttnParams &p, const int *lens, Walk &w) {
    const int lane = threadIdx.x & 31;
    auto tiles = [&](int b) {
        return lens ? (b < p.B ? tiles_of(lens[b]) : 0) : seq_tiles(p, b);
    };
    long long all = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32)
        all += (long long)__reduce_add_sync(kFull, (unsigned)tiles(b0 + lane)) * p.Hkv;
    const Split sp = split_of(p, all);
    const long long q[2] = {udiv((long long)blockIdx.x * sp.W, p.num_ctas),
                            udiv(((long long)blockIdx.x + 1) * sp.W, p.num_ctas)};
    long long at[2] = {sp.N, sp.N};
    w = {0, 0, 0, 1, 0, 0, lens};
    int found = 0;
    long long run_w = 0, run_t = 0;  // weighted positions / tiles before the chunk
    for (int b0 = 0; b0 < p.B && found < 2; b0 += 32) {
        const int nt = tiles(b0 + lane), nseq = min(32, p.B - b0);
        int inc = nt;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(kFull, inc, d);
            if (lane >= d) inc += u;
        }
        const long long after =
            run_w + ((long long)inc + (long long)sp.beta * min(lane + 1, nseq)) * p.Hkv;
        while (found < 2) {
            const unsigned m = __ballot_sync(kFull, after > q[found]);
            if (!m) break;
            const int f = __ffs(m) - 1;
            const int ntf = __shfl_sync(kFull, nt, f), before = __shfl_sync(kFull, inc, f) - ntf;
            const long long off =
                q[found] - run_w - ((long long)before + (long long)sp.beta * f) * p.Hkv;
            int h = (int)udiv(off, ntf + sp.beta);
            int t = (int)(off - (long long)h * (ntf + sp.beta));
            if (t >= ntf) {  // in a block tile's extra weight: the next pair
                t = 0;
                ++h;
            }
            at[found] = run_t + (long long)before * p.Hkv + (long long)h * ntf + t;
            if (found == 0) {
                w.b = b0 + f;
                w.h = h;
                w.t = t;
                if (h == p.Hkv) {
                    w.h = 0;
                    ++w.b;
                }
                walk_load(p, w);
            }
            ++found;
        }
        const int chunk = __shfl_sync(kFull, inc, 31);
        run_w += ((long long)chunk + (long long)sp.beta * nseq) * p.Hkv;
        run_t += (long long)chunk * p.Hkv;
    }
    return (int)max(0ll, at[1] - at[0]);  // the host admits no more than 2^30 a CTA
}

// The same where every range is to be whole pairs, as many as another CTA's.
__device__ int plan_whole(const PagedAttnParams &p, const int *lens, Walk &w) {
    const long long pairs = (long long)p.B * p.Hkv;
    const int first = (int)(blockIdx.x * pairs / p.num_ctas),
              last = (int)((blockIdx.x + 1) * pairs / p.num_ctas);
    w = {first / p.Hkv, first % p.Hkv, 0, 1, 0, 0, lens};
    walk_load(p, w);
    Walk v = w;
    int n = 0;
    for (int i = first; i < last; ++i, walk_pair(p, v)) n += v.nt;
    return n;
}

// In clusters: the tiles of a pair that CTA `rank` of 1 << log_c takes, [lo, hi).  The block
// tile, the last one, weighs kLastWeight pages where there are several to a CTA.
constexpr int kLastWeight = 2;
struct Share {
    int lo, hi;
};
__device__ __forceinline__ Share share_of(int nt, int log_c, int rank) {  // (nt < 2^26)
    const int W = nt + (nt >= 4 << log_c ? kLastWeight : 0);
    return {min(nt, rank * W >> log_c), min(nt, (rank + 1) * W >> log_c)};
}
__device__ int plan_pair(const PagedAttnParams &p, const int *lens, Walk &w) {
    const int pair = blockIdx.x >> p.log_cluster;
    w = {pair / p.Hkv, pair % p.Hkv, 0, 1, 0, 0, lens};
    walk_load(p, w);
    const Share s = share_of(w.nt, p.log_cluster, blockIdx.x & ((1 << p.log_cluster) - 1));
    w.t = s.lo;
    return s.hi - s.lo;
}

// A place in a ring of N and the parity of its present phase, kept by counting
// (a 64-bit remainder is a long dependent sequence).
template <int N>
struct Ring {
    int i = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++i == N) {
            i = 0;
            phase ^= 1;
        }
    }
};

// ---- shared memory ------------------------------------------------------------------
struct TileInfo {
    float ks, lv, ivs;  // key scale, log2 and reciprocal of the value scale
    int n;              // visible keys
};
constexpr int kInfos = 64;  // ring of the pages' numbers: 32 looked up, and those in the stages

template <int D, bool CLUSTER>
struct Layout {
    // in clusters the last stage and the second buffer of queries, side by side, take
    // the cluster's partials: a CTA has one segment there
    static constexpr int kAllStages = 8, kStages = CLUSTER ? 7 : 8;
    static constexpr int kTile = kTileKeys * D;         // an e4m3 tile
    static constexpr int kStage = 2 * kTile;            // keys, values
    static constexpr int kQ8 = 2 * kRows * D;           // split queries [128 rows][D]
    static constexpr int kBf = kTileKeys * D * 2;       // a bf16 tile or the bf16 queries
    static constexpr int kPb = 2 * kRows * kTileKeys * 2;  // P of the block tile
    static constexpr int kQ8Off = kAllStages * kStage;
    static constexpr int kQbOff = kQ8Off + 2 * kQ8;
    // the block tile's P takes the place of its queries, which S is done with
    static constexpr int kPbOff = kQbOff;
    static constexpr int kKbOff = kQbOff + (kBf > kPb ? kBf : kPb);
    static constexpr int kVbOff = kKbOff + kBf;
    static constexpr int kBarOff = kVbOff + kBf;
    // full, empty [kStages], qready, qfree [2], bready, bfree, sready, sfree
    // [kSBufs], pready, pvdone [2], drain [2]
    static constexpr int kBars = 2 * kAllStages + 4 + 2 + 2 * kSBufs + 4 + 2;
    static constexpr int kInfoOff = (kBarOff + kBars * 8 + 15) / 16 * 16;
    static constexpr int kExpOff = kInfoOff + kInfos * 16;
    static constexpr int kMlOff = kExpOff + 2 * kRows * 4;  // (m, l) of each group's rows
    static constexpr int kLenOff = kMlOff + kGroups * kRows * 8;
    static constexpr int kMiscOff = kLenOff + 2 * kLens * 4;
    static constexpr int kBytes = kMiscOff + 64 + 1024;  // + alignment slack
    static constexpr uint32_t kSwizzle = D == 128 ? 2 : 4;  // 128- or 64-byte rows
    static_assert(kTile % 1024 == 0 && kQ8Off % 1024 == 0 && kPbOff % 1024 == 0, "alignment");
    static_assert(kInfos >= 32 + kStages + 1, "tile numbers in use are not written over");
    static constexpr int kPartOff = kQ8Off - kStage;  // [kRows][D] floats, and [kRows] of lse:
    static constexpr int kPartLseOff = kExpOff;       // the exponents' first half
    static_assert(kBytes <= 232448, "shared memory per CTA");
    static_assert(kStage + kQ8 == kRows * D * 4, "partials take a stage and a buffer of queries");
};

// byte offset of 16-byte chunk c of row m: rows of D bytes, swizzled
template <int D>
__device__ __forceinline__ uint32_t chunk8(int m, int c) {
    return m * D + ((D == 128 ? c ^ (m & 7) : c ^ ((m >> 1) & 3)) << 4);
}
// the same for 128-byte rows (bf16 panels of 64 columns)
__device__ __forceinline__ uint32_t chunk16(int m, int c) { return m * 128 + ((c ^ (m & 7)) << 4); }
__device__ __forceinline__ void st_shared(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

// One segment's queries: thread ct of 128 takes half of row ct / 2, finds the
// row's e = 7 - floor(log2 max |q|) (its largest element then scales into
// [128, 256)), and writes 2^e q = hi + lo / 16 as two e4m3 rows.
template <int D>
__device__ __forceinline__ void split_queries(const PagedAttnParams &p, const Walk &w, uint32_t q8,
                                              int *qexp, int ct) {
    const int row = ct >> 1, half = ct & 1;
    const bool live = row < p.G * w.T;
    constexpr int kChunks = D / 16;  // 16-byte loads of half a row
    uint4 x[kChunks];
    if (live) {
        const uint4 *src = reinterpret_cast<const uint4 *>(
            p.q + (((size_t)w.b * p.max_block + row / p.G) * p.Hq + w.h * p.G + row % p.G) * D +
            half * (D / 2));
#pragma unroll
        for (int i = 0; i < kChunks; ++i) x[i] = src[i];
    } else {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) x[i] = make_uint4(0, 0, 0, 0);
    }
    uint32_t u[4 * kChunks];
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        u[4 * i] = x[i].x;
        u[4 * i + 1] = x[i].y;
        u[4 * i + 2] = x[i].z;
        u[4 * i + 3] = x[i].w;
    }
#pragma unroll
    for (int i = 0; i < 4 * kChunks; ++i)
        mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(u[i] << 16)),
                             fabsf(__uint_as_float(u[i] & 0xffff0000u))));
    mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, 1));
    int e = 0;
    if (mx > 0.f && mx <= 3.4e38f) {
        e = 7 - ((int)((__float_as_uint(mx) >> 23) & 0xffu) - 127);
        e = e < -120 ? -120 : (e > 120 ? 120 : e);
    }
    const float sc = __uint_as_float((uint32_t)(127 + e) << 23);
    const int m = 32 * (row >> 4) + (row & 15);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {  // 16 elements: 8 words in, 4 + 4 words out
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = u[8 * c + j];
            const float a = __uint_as_float(v << 16) * sc, b = __uint_as_float(v & 0xffff0000u) * sc;
            const uint32_t hi = e4m3_f32(a, b);
            float ha, hb;
            unpack_f16(f16_e4m3(hi), ha, hb);
            const uint32_t lo = e4m3_f32((a - ha) * 16.f, (b - hb) * 16.f);
            h[j >> 1] = j & 1 ? h[j >> 1] | hi << 16 : hi;
            l[j >> 1] = j & 1 ? l[j >> 1] | lo << 16 : lo;
        }
        const int chunk = half * (D / 32) + c;
        st_shared(q8 + chunk8<D>(m, chunk), h[0], h[1], h[2], h[3]);
        st_shared(q8 + chunk8<D>(m + 16, chunk), l[0], l[1], l[2], l[3]);
    }
    if (half == 0) qexp[row] = e;
}

// A pair's bf16 queries, block keys and block values: [64 rows][D] as D / 64
// swizzled panels, rows past the block zero.
template <int D>
__device__ __forceinline__ void load_block(const PagedAttnParams &p, const Walk &w, uint32_t qb,
                                           uint32_t kb, uint32_t vb, int ct) {
    constexpr int kPerRow = D / 8;
    const int rows = p.G * w.T;
    for (int i = ct; i < kRows * kPerRow; i += kQueryWarps * 32) {
        const int r = i / kPerRow, c = i % kPerRow;
        const uint32_t at = (c >> 3) * (kRows * 128) + chunk16(r, c & 7);
        uint4 q = make_uint4(0, 0, 0, 0), k = q, v = q;
        if (r < rows)
            q = *reinterpret_cast<const uint4 *>(
                p.q + (((size_t)w.b * p.max_block + r / p.G) * p.Hq + w.h * p.G + r % p.G) * D +
                c * 8);
        if (r < w.T) {
            const size_t s = (((size_t)w.b * p.max_block + r) * p.Hkv + w.h) * D + c * 8;
            k = *reinterpret_cast<const uint4 *>(p.k_blk + s);
            v = *reinterpret_cast<const uint4 *>(p.v_blk + s);
        }
        st_shared(qb + at, q.x, q.y, q.z, q.w);
        st_shared(kb + at, k.x, k.y, k.z, k.w);
        st_shared(vb + at, v.x, v.y, v.z, v.w);
    }
}

__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float x) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory");
}
__device__ __forceinline__ void st_cluster4(uint32_t addr, float x, float y, float z, float w) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(x), "f"(y),
                 "f"(z), "f"(w)
                 : "memory");
}

// CLUSTER: a cluster of 1 << p.log_cluster CTAs to a pair, which join their partials through
// their shared memory; else the list of all pairs' tiles, and paged_merge_kernel.
template <int D, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 1)
    paged_attn_kernel(const __grid_constant__ CUtensorMap tm_k,
                      const __grid_constant__ CUtensorMap tm_v, const PagedAttnParams p) {
    using Lt = Layout<D, CLUSTER>;
    constexpr int kStages = Lt::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                              ~uintptr_t(1023));
    const uint32_t sbase = smem_u32(sm);
    const uint32_t b_full = sbase + Lt::kBarOff, b_empty = b_full + 8 * kStages,
                   b_qready = b_empty + 8 * kStages, b_qfree = b_qready + 16,
                   b_bready = b_qfree + 16, b_bfree = b_bready + 8, b_sready = b_bfree + 8,
                   b_sfree = b_sready + 8 * kSBufs, b_pready = b_sfree + 8 * kSBufs,
                   b_pvdone = b_pready + 16, b_drain = b_pvdone + 16;
    TileInfo *info = reinterpret_cast<TileInfo *>(sm + Lt::kInfoOff);
    int *qexp = reinterpret_cast<int *>(sm + Lt::kExpOff);  // [2][kRows]
    constexpr int kFirstQ = CLUSTER;  // the buffer of the first segment's queries
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(sm + Lt::kMiscOff);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + Lt::kMiscOff + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(b_full + 8 * s, 1);
            mbar_init(b_empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_qready + 8 * i, kQueryWarps);
            // the segment's last S, and every softmax warp once it has read e
            mbar_init(b_qfree + 8 * i, 1 + kSoftWarps);
            mbar_init(b_pready + 8 * i, kGroupWarps);
            mbar_init(b_pvdone + 8 * i, 1);
            mbar_init(b_drain + 8 * i, 1);
        }
        mbar_init(b_bready, kQueryWarps);
        mbar_init(b_bfree, 1);
        for (int i = 0; i < kSBufs; ++i) {
            mbar_init(b_sready + 8 * i, 1);
            mbar_init(b_sfree + 8 * i, kGroupWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *abort_flag = 0;
    }
    if (warp == 0) {
        asm volatile(
            "tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                smem_u32(const_cast<uint32_t *>(tmem_slot))),
            "n"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if constexpr (CLUSTER)  // waited for before the first store to another CTA: it has begun
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    bool begun = false;
    int *len_sm = reinterpret_cast<int *>(sm + Lt::kLenOff);
    const bool early = p.B <= kLens;
    if (early && warp == kProducerWarp) {
        len_sm[lane] = lane < p.B ? prefix_of(p, lane) : 0;
        len_sm[kLens + lane] = lane < p.B ? block_of(p, lane) : 0;
    }
    if (warp == kProducerWarp && elect_one()) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_k)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_v)) : "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;

    Walk w0 = {0, 0, 0, 1, 0, 0, nullptr};
    int ntiles = 0;
    if (early) {
        ntiles = CLUSTER ? plan_pair(p, len_sm, w0) : p.whole ? plan_whole(p, len_sm, w0) : plan(p, len_sm, w0);
        // Into L2 while the kernels before this one finish: the range's first pages
        // (if the table still says other pages after the wait, these were for
        // nothing), their scales, and the first queries.
        if (warp == kProducerWarp) {
            if (lane < min(ntiles, w0.nt - 1 - w0.t) && lane < kPrefetch) {
                const int pg = __ldcg(p.table + (size_t)w0.b * p.max_pages + w0.t + lane);
                if (pg >= 0 && pg < p.pages) {
                    const size_t tile = (size_t)pg * p.Hkv + w0.h;
                    prefetch_bulk(p.k + tile * Lt::kTile, Lt::kTile);
                    prefetch_bulk(p.v + tile * Lt::kTile, Lt::kTile);
                    prefetch_line(p.k_scale + tile);
                    prefetch_line(p.v_scale + tile);
                }
            }
        } else if (warp >= kQueryWarp0 && ntiles > 0) {
            const int r = threadIdx.x - kQueryWarp0 * 32;  // half a row of the first pair
            if ((r >> 1) < p.G * w0.T)
                prefetch_line(p.q + (((size_t)w0.b * p.max_block + (r >> 1) / p.G) * p.Hq +
                                     w0.h * p.G + (r >> 1) % p.G) * D + (r & 1) * (D / 2));
        }
    }
    // every input (and the workspace) may be written by the previous kernel
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // (the producer's first look-up is on its way while the lengths are read again)
    int page_early = 0;
    const int n_early = early ? min(ntiles, w0.nt - 1 - w0.t) : 0;
    if (warp == kProducerWarp && lane < n_early)
        page_early = __ldcg(p.table + (size_t)w0.b * p.max_pages + w0.t + lane);
    bool kept = false;  // whether the plan holds; the same in every warp
    if (early) {
        const int P1 = lane < p.B ? prefix_of(p, lane) : 0, T1 = lane < p.B ? block_of(p, lane) : 0;
        kept = __all_sync(kFull, P1 == len_sm[lane] && T1 == len_sm[kLens + lane]);
        if (!kept) {
            __syncthreads();  // every warp has compared
            if (warp == kProducerWarp) {
                len_sm[lane] = P1;
                len_sm[kLens + lane] = T1;
            }
            __syncthreads();
        }
    }
    if (!kept) {
        const int *const lens = early ? len_sm : nullptr;
        ntiles = CLUSTER ? plan_pair(p, lens, w0) : p.whole ? plan_whole(p, lens, w0) : plan(p, lens, w0);
    }
    if (blockIdx.x == 0 && warp == 0)
        for (int b = lane; b < p.B; b += 32)
            if (p.prefix_len[b] != prefix_of(p, b) || p.block_len[b] != block_of(p, b))
                atomicOr(p.status, kStatusClamped);

    auto waits = [&](uint32_t bar, uint32_t parity) {
        return wait(bar, parity, abort_flag, p.status);
    };
    int issued = 0;  // tiles whose loads were issued (the producer's)
    // The roles below walk the same segments: a run of pages of one pair, and the
    // pair's block tile if the range reaches it.
    if (warp == kProducerWarp) {
        // ================================ producer ===============================
        // Stage s is reused once the P V that read it has completed.  32 pages at a
        // time, lane i looks up the i-th and writes its numbers to their ring; the
        // next 32 are asked for when these are begun.
        uint64_t policy;
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        Ring<kStages> st;
        bool ok = true;
        struct Chunk {
            Walk w;         // the segment: its pair and first page
            int left;       // tiles of the range from there on
            int i0, n;      // the chunk's first page in the segment, the segment's pages
            int page;       // lane i: page i0 + i, -1 if it is none
            float ks, vs;   // its scales
        };
        auto begin = [&](Chunk &c) {  // at the next segment with pages, if there is one
            c.i0 = 0;
            for (;;) {
                c.n = min(c.left, c.w.nt - 1 - c.w.t);
                if (c.n > 0 || c.left <= 0) return;
                c.left -= c.w.nt - c.w.t;
                walk_pair(p, c.w);
            }
        };
        auto look_up = [&](Chunk &c, bool have) {
            const int i = c.i0 + lane;
            if (!have)
                c.page = i < c.n
                             ? __ldcg(p.table + (size_t)c.w.b * p.max_pages + c.w.t + i)
                             : 0;
            if (c.page < 0 || c.page >= p.pages) {
                atomicOr(p.status, kStatusBadPage);
                c.page = -1;
            }
            const size_t tile = (size_t)max(c.page, 0) * p.Hkv + c.w.h;
            c.ks = p.k_scale[tile];
            c.vs = p.v_scale[tile];
        };
        auto load = [&](int tile) {
            const uint32_t full = b_full + 8 * st.i, dst = sbase + st.i * Lt::kStage;
            tma_3d(dst, &tm_k, full, 0, 0, tile, policy);
            tma_3d(dst + Lt::kTile, &tm_v, full, 0, 0, tile, policy);
        };
        Chunk c = {w0, ntiles, 0, 0, page_early, 0.f, 0.f};
        begin(c);
        if (c.left > 0) look_up(c, kept && c.n == n_early && c.left == ntiles);
        while (c.left > 0 && ok) {
            const int tile0 = max(c.page, 0) * p.Hkv + c.w.h, end = min(32, c.n - c.i0);
            // the range's first loads go before the scales are there (their bytes are
            // announced below: a barrier's phase waits for that)
            const int ahead = issued == 0 ? min(end, kStages) : 0;
            for (int i = 0; i < ahead; ++i) {
                const int tile = __shfl_sync(kFull, tile0, i);
                if (elect_one()) load(tile);
                __syncwarp();
                st.next();
            }
            Chunk next = c;
            next.i0 += 32;
            if (next.i0 >= next.n) {
                next.left -= next.w.nt - next.w.t;
                walk_pair(p, next.w);
                begin(next);
            }
            if (next.left > 0) look_up(next, false);
            {
                const float v = fmaxf(c.vs, 8.6736174e-19f);  // 2^-60: codes under a 0 scale vanish
                TileInfo ti;
                ti.ks = c.ks;
                ti.lv = log2f(v);
                ti.ivs = 1.f / v;
                ti.n = c.page < 0 ? 0 : min(kTileKeys, c.w.P - (c.w.t + c.i0 + lane) * kTileKeys);
                if (lane < end) info[(issued + lane) % kInfos] = ti;
            }
            __syncwarp();
            if (lane < ahead) mbar_arrive_expect_tx(b_full + 8 * lane, Lt::kStage);
            __syncwarp();
            issued += ahead;
            for (int i = ahead; i < end; ++i) {
                const int tile = __shfl_sync(kFull, tile0, i);
                if (issued >= kStages) ok = waits(b_empty + 8 * st.i, st.phase ^ 1);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(b_full + 8 * st.i, Lt::kStage);
                    load(tile);
                }
                __syncwarp();
                ++issued;
                st.next();
            }
            c = next;
        }
    } else if (warp == kSWarp) {
        // =============================== S = Q K^T ===============================
        const uint32_t id8 = idesc_e4m3(2 * kRows, kTileKeys, 0, 0);
        const uint32_t idb = idesc_bf16(kRows, kTileKeys, 0, 0);
        const uint64_t dk8 = sdesc(sbase, 16, 8 * D, Lt::kSwizzle);
        Walk w = w0;
        Ring<kStages> st;
        Ring<kSBufs> sb;
        uint32_t blk_phase = 0;
        int k = 0;
        bool ok = true;
        auto buffer = [&] {  // the next S buffer is free
            if (k >= kSBufs) ok = ok && waits(b_sfree + 8 * sb.i, sb.phase ^ 1);
            fence_after();
        };
        for (int seg = 0; k < ntiles && ok; ++seg, walk_pair(p, w)) {
            const int k_end = min(ntiles, k + w.nt - w.t);
            const bool has_blk = w.t + (k_end - k) == w.nt;
            const uint64_t dq8 =
                sdesc(sbase + Lt::kQ8Off + ((seg + kFirstQ) & 1) * Lt::kQ8, 16, 8 * D, Lt::kSwizzle);
            ok = waits(b_qready + 8 * (seg & 1), (uint32_t)((seg >> 1) & 1));
            for (const int k_blk = has_blk ? k_end - 1 : k_end; k < k_blk && ok; ++k) {
                ok = waits(b_full + 8 * st.i, st.phase);
                buffer();
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t dS = tmem + (uint32_t)(sb.i * kTileKeys);
                    const uint64_t b0 = dk8 + (uint64_t)((st.i * Lt::kStage) >> 4);
#pragma unroll
                    for (int kk = 0; kk < D / 32; ++kk)
                        mma_e4m3(dS, dq8 + kk * 2, b0 + kk * 2, id8, kk > 0);
                    mma_commit(b_sready + 8 * sb.i);
                    if (k + 1 == k_end) mma_commit(b_qfree + 8 * (seg & 1));
                }
                __syncwarp();
                st.next();
                sb.next();
            }
            if (has_blk && ok) {
                ok = waits(b_bready, blk_phase);
                blk_phase ^= 1;
                buffer();
                if (!ok) break;
                if (elect_one()) {
                    const uint64_t dqb = sdesc(sbase + Lt::kQbOff, 16, 1024, 2);
                    const uint64_t dkb = sdesc(sbase + Lt::kKbOff, 16, 1024, 2);
                    const uint32_t dS = tmem + (uint32_t)(sb.i * kTileKeys);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t off = ((kk >> 2) * (kRows * 128) + (kk & 3) * 32) >> 4;
                        mma_bf16(dS, dqb + off, dkb + off, idb, kk > 0);
                    }
                    mma_commit(b_sready + 8 * sb.i);
                    mma_commit(b_qfree + 8 * (seg & 1));
                }
                __syncwarp();
                sb.next();
                ++k;
            }
        }
    } else if (warp == kPvWarp) {
        // ================================ O += P V ===============================
        const uint32_t id8 = idesc_e5m2_e4m3(2 * kRows, D, 0, 1);
        const uint32_t idb = idesc_bf16(2 * kRows, D, 0, 1);
        const uint64_t dv8 = sdesc(sbase + Lt::kTile, 8 * D, 8 * D, Lt::kSwizzle);
        Walk w = w0;
        Ring<kStages> st;
        int k = 0;
        bool ok = true;
        for (; k < ntiles && ok; walk_pair(p, w)) {
            const int k_seg = k, k_end = min(ntiles, k + w.nt - w.t);
            const bool has_blk = w.t + (k_end - k) == w.nt;
            for (const int k_blk = has_blk ? k_end - 1 : k_end; k < k_blk && ok; ++k) {
                ok = waits(b_pready + 8 * (k & 1), (uint32_t)(k >> 1) & 1) &&
                     waits(b_full + 8 * st.i, st.phase);
                if (!ok) break;
                fence_after();
                if (elect_one()) {
                    const uint32_t dO = tmem + kOCol + (uint32_t)((k & 1) * kOStep);
                    const uint32_t a0 = tmem + kPCol + (uint32_t)((k & 1) * kPStep);
                    const uint64_t b0 = dv8 + (uint64_t)((st.i * Lt::kStage) >> 4);
                    // (the group's first tile of the segment begins its O)
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)  // parts a and b, then c, each of 2 x 32 keys
                        mma_f8_ta(dO, a0 + 8 * kk, b0 + (uint64_t)(((kk & 1) * 32 * D) >> 4), id8,
                                  k - k_seg >= kGroups || kk > 0);
                    mma_commit(b_empty + 8 * st.i);
                    mma_commit(b_pvdone + 8 * (k & 1));
                }
                __syncwarp();
                st.next();
            }
            if (has_blk && ok) {
                ok = waits(b_pready + 8 * (k & 1), (uint32_t)(k >> 1) & 1);
                if (!ok) break;
                fence_after();
                if (elect_one()) {
                    const uint64_t dpb = sdesc(sbase + Lt::kPbOff, 16, 1024, 2);
                    const uint64_t dvb = sdesc(sbase + Lt::kVbOff, kRows * 128, 1024, 2);
                    const uint32_t dO = tmem + kOCol + (uint32_t)((k & 1) * kOStep);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_bf16(dO, dpb + kk * 2, dvb + (uint64_t)((kk * 2048) >> 4), idb,
                                 k - k_seg >= kGroups || kk > 0);
                    mma_commit(b_pvdone + 8 * (k & 1));
                    mma_commit(b_bfree);
                }
                __syncwarp();
                ++k;
            }
        }
    } else if (warp >= kQueryWarp0) {
        // ====================== queries, block keys and values ===================
        const int ct = threadIdx.x - kQueryWarp0 * 32;
        Walk w = w0;
        int left = ntiles, nblk = 0;
        for (int seg = 0; left > 0; ++seg) {
            const int q = seg & 1;
            if (seg >= 2 && !waits(b_qfree + 8 * q, (uint32_t)(((seg >> 1) - 1) & 1))) break;
            const int buf = (seg + kFirstQ) & 1;
            split_queries<D>(p, w, sbase + Lt::kQ8Off + buf * Lt::kQ8, qexp + buf * kRows, ct);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_qready + 8 * q);
            if (left >= w.nt - w.t) {  // the segment reaches the pair's block tile
                if (nblk >= 1 && !waits(b_bfree, (uint32_t)((nblk - 1) & 1))) break;
                load_block<D>(p, w, sbase + Lt::kQbOff, sbase + Lt::kKbOff, sbase + Lt::kVbOff, ct);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_bready);
                ++nblk;
            }
            left -= w.nt - w.t;
            walk_pair(p, w);
        }
    } else {
        // ================================ softmax ================================
        // Group g takes every second tile, with a reference, sums and an O of
        // its own; the groups meet at the end of a segment.  Thread (warp,
        // lane): row 16 (warp % 4) + lane % 16, 32 of a tile's keys.
        const int group = warp / kGroupWarps, quad = warp % kGroupWarps;
        const int row = quad * 16 + (lane & 15), half = lane >> 4;
        const int key0 = 32 * half;
        const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t o_col = lanes + kOCol + (uint32_t)(group * kOStep);
        float2 *ml = reinterpret_cast<float2 *>(sm + Lt::kMlOff);
        const uint32_t p_col = lanes + kPCol + (uint32_t)(group * kPStep);
        {  // beside c there is no fourth part
            const uint32_t zero[8] = {};
            st_half(p_col + kPStep / 2, zero);
        }
        Walk w = w0;
        float m_ref = -INFINITY, l_sum = 0.f, row_scale = 1.f;
        int k = 0, kp = 0;  // the next tile, and the pages before it
        for (int seg = 0; k < ntiles; ++seg, walk_pair(p, w)) {
            const int k_seg = k, k_end = min(ntiles, k + w.nt - w.t);
            const bool has_blk = w.t + (k_end - k_seg) == w.nt;
            const int rows_active = p.G * w.T, irow = row / p.G, seg_t = w.t;
            const bool live = row < rows_active;
            m_ref = -INFINITY;
            l_sum = 0.f;
            {
                const int q = seg & 1;
                waits(b_qready + 8 * q, (uint32_t)((seg >> 1) & 1));
                row_scale = p.scale_log2 *
                            __uint_as_float((uint32_t)(127 - qexp[((q + kFirstQ) & 1) * kRows + row]) << 23);
                __syncwarp();
                if (lane == 0) mbar_arrive(b_qfree + 8 * q);
            }
            const int k_blk = has_blk ? k_end - 1 : k_end;  // pages are the tiles before it
            // Weights of a tile from its scores v (hidden ones -inf), in e, and their
            // sum.  They are taken under the present reference; a thread whose 32
            // weights sum to no more than kMost has none above it, and only where
            // that fails, or there is no reference yet, is the row's maximum found and the
            // reference set by it (O and l rescaled) and the weights taken again.
            auto weights_of = [&](float (&v)[32], float (&e)[32], float scale, float lv, bool hidden) {
                auto exps = [&] {
                    const float off = lv + kHead - (m_ref == -INFINITY ? 0.f : m_ref);
                    if (hidden) {  // a hidden score stays -inf under a scale of 0
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            e[j] = v[j] == -INFINITY ? -INFINITY : v[j] * scale + off;
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 2)
                            fma2(e[j], e[j + 1], v[j], v[j + 1], scale, off);
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) e[j] = ex2(e[j]);
                    float x[16];
#pragma unroll
                    for (int j = 0; j < 16; j += 2)
                        add2(x[j], x[j + 1], e[j], e[j + 1], e[j + 16], e[j + 17]);
#pragma unroll
                    for (int d = 8; d > 1; d >>= 1)
#pragma unroll
                        for (int j = 0; j < d; j += 2)
                            add2(x[j], x[j + 1], x[j], x[j + 1], x[j + d], x[j + d + 1]);
                    return x[0] + x[1];
                };
                const bool fresh = k - k_seg < kGroups;  // the segment's first tile of the group
                float sum = exps();
                if (__any_sync(kFull, live && (m_ref == -INFINITY || !(sum <= kMost)))) {
                    float x[11];
#pragma unroll
                    for (int j = 0; j < 10; ++j) x[j] = max3(v[3 * j], v[3 * j + 1], v[3 * j + 2]);
                    x[10] = fmaxf(v[30], v[31]);
                    float mt = fmaxf(max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]),
                                          max3(x[6], x[7], x[8])),
                                     fmaxf(x[9], x[10]));
                    mt = fmaxf(mt, __shfl_xor_sync(kFull, mt, 16));
                    mt = mt == -INFINITY ? -INFINITY : mt * scale + lv;
                    const bool over = !(sum <= kMost);
                    const bool over_row = __shfl_xor_sync(kFull, over, 16) || over;
                    const bool jump = live && mt > -INFINITY && (m_ref == -INFINITY || over_row);
                    if (__any_sync(kFull, jump)) {
                        const float old = m_ref;
                        if (jump) m_ref = mt;
                        sum = exps();
                        const float row_sum = sum + __shfl_xor_sync(kFull, sum, 16);
                        float alpha = 1.f;
                        if (jump) {  // by the row's sum: what is far below one large weight is kept
                            const int log_sum = (int)(__float_as_uint(row_sum) >> 23 & 0xffu) - 127;
                            const int up = max(0, min(kSumLog - log_sum, kSumLog - (int)kHead));
                            const float f = __uint_as_float((uint32_t)(127 + up) << 23);
                            m_ref -= (float)up;
                            sum *= f;
#pragma unroll
                            for (int j = 0; j < 32; ++j) e[j] *= f;
                            alpha = ex2(old - m_ref);  // from -inf: 0
                            l_sum *= alpha;
                        }
                        if (!fresh) {  // the group has an O here
                            waits(b_pvdone + 8 * group, (uint32_t)((k / kGroups - 1) & 1));
                            fence_after();
                            // thread t holds lane t: row t % 16's hi or lo part, the same alpha
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                uint32_t o[32];
                                ld_lanes32(o_col + c, o);
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                                st_lanes32(o_col + c, o);
                            }
                            st_wait();
                        }
                    }
                }
                return sum;
            };
            // the group's P and O are its own again once P V of tile k - 2 is done
            auto wait_pv = [&] {
                if (k >= kGroups) waits(b_pvdone + 8 * group, (uint32_t)((k / kGroups - 1) & 1));
                fence_after();
            };

            for (k = k_seg + ((k_seg ^ group) & 1); k < k_blk; k += kGroups) {
                const int kq = kp + (k - k_seg), s = kq % kStages;
                // (a buffer's phase before this one, the other group's, is over: S
                // are issued and committed in order, and this group has had tile k - 2)
                const bool ok_s = waits(b_sready + 8 * (k % kSBufs), (uint32_t)(k / kSBufs) & 1);
                fence_after();
                const uint32_t s_addr = lanes + (uint32_t)((k % kSBufs) * kTileKeys);
                uint32_t a[32], c[32];
                ld_half(s_addr, a);
                ld_half(s_addr + kLoLanes, c);
                // while the loads are on their way: the tile's numbers, and whether the
                // group's P and O are its own again (once P V of tile k - 2 is done)
                waits(b_full + 8 * s, (uint32_t)(kq / kStages) & 1);
                const bool pv_early =
                    k < kGroups ||
                    mbar_try_wait(b_pvdone + 8 * group, (uint32_t)((k / kGroups - 1) & 1));
                const TileInfo ti = info[kq % kInfos];
                const float scale = row_scale * ti.ks;
                const int n = ti.n;
                ld_wait(a);
                ld_wait(c);
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_sfree + 8 * (k % kSBufs));
                float v[32], e[32];
#pragma unroll
                for (int j = 0; j < 32; j += 2)
                    axpy2(v[j], v[j + 1], kQLoInv, __uint_as_float(c[j]), __uint_as_float(c[j + 1]),
                          __uint_as_float(a[j]), __uint_as_float(a[j + 1]));
                if (n < kTileKeys || !ok_s) {
                    const int lim = ok_s ? n : 0;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (key0 + j >= lim) v[j] = -INFINITY;
                }
                const float sum = weights_of(v, e, scale, ti.lv, n < kTileKeys || !ok_s);
                uint32_t pa[8], pb[8], pc[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const Parts r = parts_of(pack_f16(e[4 * j], e[4 * j + 1]),
                                             pack_f16(e[4 * j + 2], e[4 * j + 3]));
                    pa[j] = r.a;
                    pb[j] = r.b;
                    pc[j] = r.c;
                }
                if (!pv_early) wait_pv();
                st_half(p_col, pa);
                st_half(p_col + kLoLanes, pb);
                st_half(p_col + kPStep / 2 + kLoLanes, pc);
                // keys past the page's last token may hold anything: zero their value rows
                if (n < kTileKeys) {
                    const uint32_t vt = sbase + s * Lt::kStage + Lt::kTile + n * D;
                    for (int i = threadIdx.x % (kGroupWarps * 32); i < (kTileKeys - n) * (D / 16);
                         i += kGroupWarps * 32)
                        st_shared(vt + i * 16, 0, 0, 0, 0);
                    fence_async_smem();
                }
                st_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_pready + 8 * group);
                l_sum += sum * ti.ivs;
            }
            if (has_blk && k == k_blk) {  // the block's own keys, bf16
                const bool ok_s = waits(b_sready + 8 * (k % kSBufs), (uint32_t)(k / kSBufs) & 1);
                fence_after();
                uint32_t a[32];
                ld_half(lanes + (uint32_t)((k % kSBufs) * kTileKeys), a);
                ld_wait(a);
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_sfree + 8 * (k % kSBufs));
                const int lim = live && ok_s ? min(w.T, irow + 1) : 0;  // the causal mask
                float v[32], e[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = key0 + j < lim ? __uint_as_float(a[j]) : -INFINITY;
                l_sum += weights_of(v, e, p.scale_log2, 0.f, true);
                wait_pv();
                const uint32_t pb = sbase + Lt::kPbOff;
                const int m = 32 * quad + (lane & 15);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t h[4], l[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = e[8 * c + 2 * i], y = e[8 * c + 2 * i + 1];
                        h[i] = pack_bf16(x, y);
                        l[i] = pack_bf16((x - __uint_as_float(h[i] << 16)) * kPLo,
                                         (y - __uint_as_float(h[i] & 0xffff0000u)) * kPLo);
                    }
                    st_shared(pb + chunk16(m, key0 / 8 + c), h[0], h[1], h[2], h[3]);
                    st_shared(pb + chunk16(m + 16, key0 / 8 + c), l[0], l[1], l[2], l[3]);
                }
                fence_async_smem();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_pready + 8 * group);
            }

            {
                // ---- end of a segment: the groups' sums joined, O / l and lse ----
                // group g's last tile here is the last one of its parity, if any
                const int k_last = k_end - 1, kl = (k_last & 1) == group ? k_last : k_last - 1;
                const bool any = kl >= k_seg;
                if (any) waits(b_pvdone + 8 * group, (uint32_t)((kl / kGroups) & 1));
                fence_after();
                const float lg = l_sum + __shfl_xor_sync(kFull, l_sum, 16);
                if (half == 0) ml[group * kRows + row] = make_float2(any ? m_ref : -INFINITY, lg);
                asm volatile("bar.sync 1, 256;" ::: "memory");
                fence_after();
                const float2 ml0 = ml[row], ml1 = ml[kRows + row];
                const float M = fmaxf(ml0.x, ml1.x), M0 = M == -INFINITY ? 0.f : M;
                const float s0 = ex2(ml0.x - M0), s1 = ex2(ml1.x - M0);  // 0 for a group without tiles
                const float l = s0 * ml0.y + s1 * ml1.y;
                // 0: no visible key; NaN (a code that is none) stays NaN
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const float lse = l == 0.f ? -INFINITY : (M - kHead + log2f(l)) * kLn2;
                const bool whole = seg_t == 0 && has_blk;
                const bool two = k_last > k_seg;  // both groups hold an O
                const int gq = w.h * p.G + row % p.G;
                const size_t slot =
                    ((size_t)(w.b * p.Hkv + w.h) + blockIdx.x) * p.rows_max + row;
                uint16_t *orow = p.out + (((size_t)w.b * p.max_block + irow) * p.Hq + gq) * D;
                float *prow = p.part_o + slot * D;
                // in a cluster row r is joined by CTA r % C, where the partial of CTA c has
                // place c * kRows / C + r / C, its 16-byte chunks xored with the row
                const int log_c = p.log_cluster, C = 1 << log_c, to = row & (C - 1);
                const int place = ((blockIdx.x & (C - 1)) << 6 >> log_c) + (row >> log_c);
                const uint32_t far = CLUSTER ? at_rank(sbase + Lt::kPartOff + place * (D * 4), to) : 0;
                // group g writes columns [g D / 2, (g + 1) D / 2), 32 at a time
                float x[D / 64][16];
                const uint32_t o0 = lanes + kOCol + (uint32_t)((k_seg & 1) * kOStep);
                const uint32_t o1 = lanes + kOCol + (uint32_t)((~k_seg & 1) * kOStep);
                const float f0 = (k_seg & 1 ? s1 : s0) * inv, f1 = (k_seg & 1 ? s0 : s1) * inv;
#pragma unroll
                for (int c = 0; c < D / 64; ++c) {
                    const uint32_t col = (uint32_t)(group * (D / 2) + 32 * c);
                    uint32_t a[16], e[16];
                    ld_half(o0 + col, a);
                    ld_half(o0 + col + kLoLanes, e);
                    ld_wait(a);
                    ld_wait(e);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        x[c][j] = (__uint_as_float(a[j]) + kPLoInv * __uint_as_float(e[j])) * f0;
                    if (two) {
                        ld_half(o1 + col, a);
                        ld_half(o1 + col + kLoLanes, e);
                        ld_wait(a);
                        ld_wait(e);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            x[c][j] += (__uint_as_float(a[j]) + kPLoInv * __uint_as_float(e[j])) * f1;
                    }
                }
                if constexpr (CLUSTER) {
                    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
                    begun = true;
                } else {  // both groups have read both O and ml: the next segment may write them
                    fence_before();
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                }
                if (live) {
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) {
                        const int d0 = group * (D / 2) + 32 * c + 16 * half;
                        if (whole) {
#pragma unroll
                            for (int j = 0; j < 16; j += 8)
                                *reinterpret_cast<uint4 *>(orow + d0 + j) = make_uint4(
                                    pack_bf16(x[c][j], x[c][j + 1]),
                                    pack_bf16(x[c][j + 2], x[c][j + 3]),
                                    pack_bf16(x[c][j + 4], x[c][j + 5]),
                                    pack_bf16(x[c][j + 6], x[c][j + 7]));
                        } else if (CLUSTER) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                st_cluster4(far + (((d0 + j) / 4 ^ (place & (D / 4 - 1))) << 4), x[c][j],
                                            x[c][j + 1], x[c][j + 2], x[c][j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<float4 *>(prow + d0 + j) = make_float4(
                                    x[c][j], x[c][j + 1], x[c][j + 2], x[c][j + 3]);
                        }
                    }
                    if (half == 0 && group == 0) {
                        if (whole)
                            p.lse[((size_t)w.b * p.Hq + gq) * p.max_block + irow] = lse;
                        else if (CLUSTER)
                            st_cluster(at_rank(sbase + Lt::kPartLseOff + place * 4, to), lse);
                        else
                            p.part_lse[slot] = lse;
                    }
                }
                if (whole)  // rows past the block: 0 and lse -inf
                    for (int i = threadIdx.x; i < (p.rows_max - rows_active) * (D / 8);
                         i += kSoftWarps * 32) {
                        const int r = rows_active + i / (D / 8), c = (i % (D / 8)) * 8;
                        const int ii = r / p.G, gg = w.h * p.G + r % p.G;
                        *reinterpret_cast<uint4 *>(
                            p.out + (((size_t)w.b * p.max_block + ii) * p.Hq + gg) * D + c) =
                            make_uint4(0, 0, 0, 0);
                        if (c == 0) p.lse[((size_t)w.b * p.Hq + gg) * p.max_block + ii] = -INFINITY;
                    }
            }
            kp += k_blk - k_seg;
            k = k_end;
        }
    }
    if constexpr (CLUSTER) {  // this CTA's partials are where they belong
        __syncwarp();
        if (!begun) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (*abort_flag) {  // a timed-out run: MMAs and copies may be in flight yet
        if (warp == kSWarp || warp == kPvWarp) {
            const uint32_t drain = b_drain + (warp == kSWarp ? 8 : 0);
            if (elect_one()) mma_commit(drain);
            __syncwarp();
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(drain, 0) && globaltimer() - t0 < kWaitNs) {
            }
        }
        if (warp == kProducerWarp && elect_one())
            for (int j = issued - 1; j >= 0 && j >= issued - kStages; --j)
                drain_wait(b_full + 8 * (j % kStages), (uint32_t)(j / kStages) & 1);
        __syncwarp();
        fence_before();
        __syncthreads();
        fence_after();
    }
    // (else the softmax warps have seen every product's completion)
    if (warp == kThreads / 32 - 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "n"(kTmemCols));
    if constexpr (CLUSTER) {
        // ---- the cluster's partials joined: every C-th row by one of its CTAs ----
        // (formulas as in paged_merge_kernel)
        constexpr int V = D / 32, kMaxC = 8;
        const int C = 1 << p.log_cluster, rank = blockIdx.x & (C - 1);
        bool held[kMaxC];  // whether CTA r has a partial
        int n = 0;
#pragma unroll
        for (int r = 0; r < kMaxC; ++r) {
            const Share s = share_of(w0.nt, p.log_cluster, min(r, C - 1));
            held[r] = r < C && s.hi > s.lo;
            n += held[r];
        }
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (n <= 1) return;  // one CTA had the pair
        const float *const part_o = reinterpret_cast<const float *>(sm + Lt::kPartOff);
        const float *const part_lse = reinterpret_cast<const float *>(sm + Lt::kPartLseOff);
        for (int row = rank + C * warp; row < p.rows_max; row += C * (kThreads / 32)) {
            const int i = row / p.G, g = w0.h * p.G + row % p.G;
            float ls[kMaxC], o[kMaxC][V], M = -INFINITY, L = 0.f, acc[V];
#pragma unroll
            for (int r = 0; r < kMaxC; ++r) {
                ls[r] = -INFINITY;
#pragma unroll
                for (int v = 0; v < V; ++v) o[r][v] = 0.f;
                if (held[r] && row < p.G * w0.T) {
                    const int place = (r << 6 >> p.log_cluster) + (row >> p.log_cluster);
                    const int chunk = (V * lane / 4) ^ (place & (D / 4 - 1));
                    ls[r] = part_lse[place];
#pragma unroll
                    for (int v = 0; v < V; v += 2) {
                        const float2 x = *reinterpret_cast<const float2 *>(
                            part_o + place * D + chunk * 4 + (V * lane & 3) + v);
                        o[r][v] = x.x;
                        o[r][v + 1] = x.y;
                    }
                }
            }
            bool nan = false;
#pragma unroll
            for (int r = 0; r < kMaxC; ++r) {
                M = fmaxf(M, ls[r]);
                nan = nan || ls[r] != ls[r];
            }
            const float m = M == -INFINITY && !nan ? 0.f : M;
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = 0.f;
#pragma unroll
            for (int r = 0; r < kMaxC; ++r) {
                const float x = __expf(ls[r] - m);
                L += x;
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += x * o[r][v];
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            uint16_t *orow = p.out + (((size_t)w0.b * p.max_block + i) * p.Hq + g) * D + V * lane;
#pragma unroll
            for (int v = 0; v < V; v += 2)
                *reinterpret_cast<uint32_t *>(orow + v) = pack_bf16(acc[v] * inv, acc[v + 1] * inv);
            if (lane == 0)
                p.lse[((size_t)w0.b * p.Hq + g) * p.max_block + i] =
                    L == 0.f ? -INFINITY : m + __logf(L);
        }
    }
}

// ---- merge ------------------------------------------------------------------------
// One warp per query row of a pair that was cut: with partials O_s / l_s and
// lse_s, out = sum_s e^(lse_s - M) O_s / l_s / sum_s e^(lse_s - M) and
// lse = M + ln of that sum.
// Two warps a CTA: its registers then fit beside an attention CTA's, so that
// it waits for the attention grid on the SM and has the plan by then.
constexpr int kMergeWarps = 2;
constexpr int kMergeLoads = 4;

struct Cut {  // a pair's segments: of CTAs c0, c0 + 1, ... if dense
    Split sp;
    long long q0;
    int c0, n;
    bool dense;
};
__device__ __forceinline__ Cut cut_of(const PagedAttnParams &p, int b, int h) {
    const int lane = threadIdx.x & 31;
    long long total = 0, before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        const int nt = seq_tiles(p, b0 + lane);
        total += (long long)__reduce_add_sync(kFull, (unsigned)nt) * p.Hkv;
        before += (long long)__reduce_add_sync(kFull, b0 + lane < b ? (unsigned)nt : 0u) * p.Hkv;
    }
    Cut c;
    c.sp = split_of(p, total);
    const int nt = tiles_of(prefix_of(p, b));
    c.q0 = before + (long long)h * nt + (long long)c.sp.beta * (b * p.Hkv + h);
    c.c0 = cta_of(c.q0, c.sp, p.num_ctas);
    // with fewer tiles than CTAs a tile is a CTA's own and the CTAs between are empty
    c.dense = c.sp.beta > 0 || c.sp.N >= p.num_ctas;
    c.n = c.dense ? cta_of(c.q0 + nt - 1, c.sp, p.num_ctas) - c.c0 + 1 : nt;
    return c;
}
// where a row's partial of segment s is
__device__ __forceinline__ size_t slot_of(const PagedAttnParams &p, const Cut &c, int pair, int s, int row) {
    const int cta = c.dense ? c.c0 + s : cta_of(c.q0 + s, c.sp, p.num_ctas);
    return ((size_t)pair + cta) * p.rows_max + row;
}

template <int D>
__global__ void __launch_bounds__(kMergeWarps * 32) paged_merge_kernel(const PagedAttnParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // (the lengths may be read before the wait: the attention grid lets this one
    // begin only after its own wait)
    constexpr int V = D / 32;
    const int rblocks = (p.rows_max + kMergeWarps - 1) / kMergeWarps;
    const int pair = blockIdx.x / rblocks, lane = threadIdx.x & 31;
    const int row = (blockIdx.x % rblocks) * kMergeWarps + (threadIdx.x >> 5);
    const int b = pair / p.Hkv, h = pair % p.Hkv;
    const Cut cut = cut_of(p, b, h);
    const int nseg = cut.n, rows_active = p.G * block_of(p, b);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (nseg <= 1 || row >= p.rows_max) return;
    const int i = row / p.G, g = h * p.G + row % p.G;
    uint16_t *orow = p.out + (((size_t)b * p.max_block + i) * p.Hq + g) * D + V * lane;
    float *lrow = p.lse + ((size_t)b * p.Hq + g) * p.max_block + i;
    float M = -INFINITY, L = 0.f, acc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] = 0.f;
    if (row < rows_active) {
        for (int s0 = 0; s0 < nseg; s0 += kMergeLoads) {
            float ls[kMergeLoads], o[kMergeLoads][V];
#pragma unroll
            for (int u = 0; u < kMergeLoads; ++u) {
                ls[u] = -INFINITY;
#pragma unroll
                for (int v = 0; v < V; ++v) o[u][v] = 0.f;
                if (s0 + u < nseg) {
                    const size_t slot = slot_of(p, cut, pair, s0 + u, row);
                    ls[u] = __ldcg(p.part_lse + slot);
                    const float *src = p.part_o + slot * D + V * lane;
#pragma unroll
                    for (int v = 0; v < V; v += 2) {
                        const float2 x = __ldcg(reinterpret_cast<const float2 *>(src + v));
                        o[u][v] = x.x;
                        o[u][v + 1] = x.y;
                    }
                }
            }
            float m = M;
#pragma unroll
            for (int u = 0; u < kMergeLoads; ++u) m = fmaxf(m, ls[u]);
            float any = 0.f;  // NaN where a partial is
#pragma unroll
            for (int u = 0; u < kMergeLoads; ++u) any += ls[u] == ls[u] ? 0.f : ls[u];
            if (m == -INFINITY && any == 0.f) continue;
            const float a = __expf(M - m);
            L *= a;
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] *= a;
#pragma unroll
            for (int u = 0; u < kMergeLoads; ++u) {
                const float x = __expf(ls[u] - m);
                L += x;
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += x * o[u][v];
            }
            M = m;
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
    for (int v = 0; v < V; v += 2)
        *reinterpret_cast<uint32_t *>(orow + v) = pack_bf16(acc[v] * inv, acc[v + 1] * inv);
    if (lane == 0) *lrow = L == 0.f ? -INFINITY : M + __logf(L);
}

// The same where pairs have many segments: a row by both warps of a CTA.  A warp's
// four groups of eight lanes take every fourth segment, two at a time, with a
// reference and sums of their own, so that sixteen segments of a row are on their
// way at once.  2 kv heads of 32768 tokens, the whole call: 16.2 us, 25.3 with a warp
// to a row and four at once.
struct Part {  // sums under the reference M
    float M, L;
};
// the factors of two parts under their common reference, for which a becomes their sum
__device__ __forceinline__ float2 join(Part &a, Part b) {
    const float m = fmaxf(a.M, b.M);
    const float2 f = {a.M == m ? 1.f : __expf(a.M - m), b.M == m ? 1.f : __expf(b.M - m)};
    a = {m, a.L * f.x + b.L * f.y};
    return f;
}

template <int D>
__global__ void __launch_bounds__(kMergeWarps * 32) paged_merge_many_kernel(const PagedAttnParams p) {
    __shared__ float4 s_acc[32];
    __shared__ Part s_part;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int kChunks = D / 32;  // of 8 lanes x 4 floats
    constexpr int kGroups = 4, kLoads = 2, kStep = 2 * kGroups;
    const int pair = blockIdx.x / p.rows_max, row = blockIdx.x % p.rows_max;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = lane >> 3, col = 4 * (lane & 7);
    const int b = pair / p.Hkv, h = pair % p.Hkv;
    const Cut cut = cut_of(p, b, h);
    const int rows_active = p.G * block_of(p, b);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (cut.n <= 1) return;  // (the same in both warps)
    Part part = {-INFINITY, 0.f};
    float acc[4 * kChunks];
#pragma unroll
    for (int v = 0; v < 4 * kChunks; ++v) acc[v] = 0.f;
    if (row < rows_active) {
        for (int s0 = warp * kGroups + group; s0 < cut.n; s0 += kLoads * kStep) {
            float ls[kLoads];
            float4 o[kLoads][kChunks];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                ls[u] = -INFINITY;
#pragma unroll
                for (int c = 0; c < kChunks; ++c) o[u][c] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s0 + u * kStep < cut.n) {
                    const size_t slot = slot_of(p, cut, pair, s0 + u * kStep, row);
                    ls[u] = __ldcg(p.part_lse + slot);
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
                        o[u][c] = __ldcg(reinterpret_cast<const float4 *>(p.part_o + slot * D + 32 * c + col));
                }
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                if (ls[u] == -INFINITY) continue;
                // (a NaN goes into the sums, not into the reference)
                const float2 f = join(part, {ls[u] == ls[u] ? ls[u] : part.M, ls[u] == ls[u] ? 1.f : ls[u]});
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    acc[4 * c] = acc[4 * c] * f.x + o[u][c].x * f.y;
                    acc[4 * c + 1] = acc[4 * c + 1] * f.x + o[u][c].y * f.y;
                    acc[4 * c + 2] = acc[4 * c + 2] * f.x + o[u][c].z * f.y;
                    acc[4 * c + 3] = acc[4 * c + 3] * f.x + o[u][c].w * f.y;
                }
            }
        }
    }
    // the groups' sums, the lower lane's first in both lanes; then group c has chunk c
#pragma unroll
    for (int d = 8; d < 32; d *= 2) {
        const Part other = {__shfl_xor_sync(kFull, part.M, d), __shfl_xor_sync(kFull, part.L, d)};
        Part low = lane & d ? other : part;
        const float2 f = join(low, lane & d ? part : other);
        part = low;
#pragma unroll
        for (int v = 0; v < 4 * kChunks; ++v) {
            const float y = __shfl_xor_sync(kFull, acc[v], d);
            acc[v] = lane & d ? y * f.x + acc[v] * f.y : acc[v] * f.x + y * f.y;
        }
    }
    float4 x = make_float4(acc[0], acc[1], acc[2], acc[3]);
#pragma unroll
    for (int c = 1; c < kChunks; ++c)
        if (group == c) x = make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
    if (warp == 1) {
        s_acc[lane] = x;
        if (lane == 0) s_part = part;
    }
    __syncthreads();
    if (warp == 1) return;
    const float4 y = s_acc[lane];
    const float2 f = join(part, s_part);
    const int i = row / p.G, g = h * p.G + row % p.G;
    const float inv = part.L == 0.f ? 0.f : 1.f / part.L, fx = f.x * inv, fy = f.y * inv;
    if (group < kChunks)
        *reinterpret_cast<uint2 *>(p.out + (((size_t)b * p.max_block + i) * p.Hq + g) * D + 32 * group + col) =
            make_uint2(pack_bf16(x.x * fx + y.x * fy, x.y * fx + y.y * fy),
                       pack_bf16(x.z * fx + y.z * fy, x.w * fx + y.w * fy));
    if (lane == 0)
        p.lse[((size_t)b * p.Hq + g) * p.max_block + i] =
            part.L == 0.f ? -INFINITY : part.M + __logf(part.L);
}

size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

// The logarithm of the CTAs to a pair where clusters are used, else -1.
// Measured at 38 shapes, in tiles of 0.34 us: a cluster's CTA takes its own tiles and
// 23; in the list a CTA takes an equal share of all tiles and 32, 0.25 for each of a
// pair's segments, and 9 for each pair that ends in its range.  One sequence of
// 4096 tokens with 32, 8 and 2 kv heads takes 14.2, 10.1 and 9.5 us in clusters,
// 17.4, 12.7 and 15.3 in the list; of 32768 tokens 58.3, 32.3 and 31.4, and 53.8,
// 22.8 and 16.2.
// Lengths are not known here: the list's time is taken as the least it can be with x
// pairs as long as the table allows and the others empty, x from a sequence's kv
// heads to all pairs, which is at x = CTAs sqrt(0.25 / nt).
template <int D>
int log_cluster_of(const PagedAttnParams &p, int dev) {
    static std::atomic<int> most[64][4];  // 1 + the clusters of 1 << i CTAs that fit the device
    if (dev >= 64) return -1;
    const long long pairs = (long long)p.B * p.Hkv, nt = (long long)p.max_pages + 1;
    const double ctas = p.num_ctas,
                 x = std::min(std::max(ctas * std::sqrt(0.25 / (double)nt), (double)p.Hkv), (double)pairs);
    const double list = 9.0 + x * (double)nt / ctas + 0.25 * ctas / x + 9.0 * (double)pairs / ctas;
    for (int i = 3; i >= 0; --i) {
        const int C = 1 << i;
        if (pairs * C > p.num_ctas) continue;
        if ((double)((nt + C - 1) / C) > list) return -1;  // (smaller clusters cost more)
        if (i == 0) return 0;
        int fit = most[dev][i].load(std::memory_order_relaxed);
        if (fit == 0) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(p.num_ctas / C * C));
            cfg.blockDim = dim3(kThreads);
            cfg.dynamicSmemBytes = Layout<D, true>::kBytes;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = C;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, paged_attn_kernel<D, true>, &cfg) != cudaSuccess)
                n = 0;
            fit = 1 + n;
            most[dev][i].store(fit, std::memory_order_relaxed);
        }
        if (pairs <= fit - 1) return i;
    }
    return -1;
}

template <int D>
cudaError_t launch_d(PagedAttnParams &p, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                     cudaStream_t stream) {
    constexpr int smem = Layout<D, false>::kBytes;
    static_assert(smem == Layout<D, true>::kBytes, "one size for both");
    static std::atomic<bool> configured[64];  // the shared-memory opt-in, once per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        for (const auto kernel : {paged_attn_kernel<D, false>, paged_attn_kernel<D, true>}) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
            if (e != cudaSuccess) return e;
        }
        if (dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    p.log_cluster = log_cluster_of<D>(p, dev);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.num_ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (p.log_cluster >= 0) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = 1 << p.log_cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
        cfg.gridDim = dim3((unsigned)(p.B * p.Hkv << p.log_cluster));
        return cudaLaunchKernelEx(&cfg, paged_attn_kernel<D, true>, tm_k, tm_v, p);
    }
    // Many short pairs: ranges of whole pairs need no merge kernel, whose time grows with
    // the pairs, and no segments of cut ones.  12 sequences of 91 tokens with 32 heads
    // take 19.5 us, 26.1 in equal ranges, of 832 31.4 and 36.6; 200 sequences of 190
    // tokens with 8 heads 67.5 and 96.9.  They cost what some CTAs' share of pairs is
    // above the mean, and with one long sequence among empty ones nearly that CTA's whole
    // share (11 of 10 tokens and one of 832: 33.3 and 31.6).  The rule's four constants
    // are fitted to 21 shapes of 12 to 1000 sequences.
    const long long pairs = (long long)p.B * p.Hkv, nt = p.max_pages + 1LL;
    const long long each = (pairs + p.num_ctas - 1) / p.num_ctas;
    p.whole = pairs > p.num_ctas && each * nt <= 26 + pairs / 24 &&
              (each * p.num_ctas - pairs) * nt <= (8 + pairs / 40) * p.num_ctas;
    e = cudaLaunchKernelEx(&cfg, paged_attn_kernel<D, false>, tm_k, tm_v, p);
    if (e != cudaSuccess || p.whole) return e;
    // With more than two rounds of segments to a pair (16 pairs: 19.5 us, 20.6 with a
    // warp to a row; 32: 17.4 and 17.4; 128: 55.1 and 42.8)
    const bool many = pairs * 2 * kMergeLoads < p.num_ctas;
    const long long rblocks = many ? p.rows_max : (p.rows_max + kMergeWarps - 1) / kMergeWarps;
    cfg.gridDim = dim3((unsigned)(pairs * rblocks));
    cfg.blockDim = dim3(kMergeWarps * 32);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, many ? paged_merge_many_kernel<D> : paged_merge_kernel<D>, p);
}

}  // namespace

// header | part_o [slots][rows_max][D] | part_lse [slots][rows_max], slots =
// B * Hkv + C (a segment's slot is its pair + its CTA).
size_t paged_workspace_bytes(int device, int batch, int kv_heads, int rows_max, int head_dim) {
    const int C = attn_grid_size(device);
    if (C <= 0) return 0;
    const size_t slots = (size_t)batch * kv_heads + (size_t)C;
    return kWorkspaceHeader + round256(slots * rows_max * head_dim * sizeof(float)) +
           round256(slots * rows_max * sizeof(float));
}

cudaError_t paged_attn_launch(PagedAttnParams &p, int head_dim, const CUtensorMap &tm_k,
                              const CUtensorMap &tm_v, void *workspace, cudaStream_t stream) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    p.num_ctas = attn_grid_size(dev);
    if (p.num_ctas <= 0) return cudaErrorInvalidDevice;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const size_t slots = (size_t)p.B * p.Hkv + (size_t)p.num_ctas;
    p.status = reinterpret_cast<int32_t *>(ws);
    p.part_o = reinterpret_cast<float *>(ws + kWorkspaceHeader);
    p.part_lse = reinterpret_cast<float *>(
        ws + kWorkspaceHeader + round256(slots * p.rows_max * head_dim * sizeof(float)));
    return head_dim == 128 ? launch_d<128>(p, tm_k, tm_v, stream)
                           : launch_d<64>(p, tm_k, tm_v, stream);
}

}  // namespace das
