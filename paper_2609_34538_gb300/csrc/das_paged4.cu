// das_paged4.cu -- the commit into the paged 4-bit cache: codes of 4 bits under a scale of
// a byte for every 32 elements of a token's head.
//
// The mathematics.  A scale has 4 significant bits and a bf16 element 8, so a quotient x / s
// comes within 2^-9 of a half only if it is one: x times the rounded reciprocal, rounded once
// more to multiples of 2^-11 (by adding 6144), decides a code as the quotient does.
//
// A warp to a (sequence, page of it, slab, keys or values, kv head).  D / 8 lanes have a
// token's row, 8 elements each, so that a scale is a matter of four lanes.  Keys lie token by
// token and go straight out.  Of the values eight tokens share a word: a lane collects its
// elements' bits over eight tokens, the lanes of the other rows add theirs, and
// each stores a part.  Words and scales that older tokens share are read first and
// keep their bits.
//
// The kernel is launched as a programmatic dependent of the previous kernel in the
// stream: it reads nothing before griddepcontrol.wait, and every CTA executes that wait.
#include <algorithm>

#include "das_internal.h"

namespace das {
namespace {

constexpr int kPage = DAS_PAGE_TOKENS;
constexpr uint32_t kFull = 0xffffffffu;
constexpr int kWarps = 4;

struct Append4Args {
    const uint16_t *fresh[2];  // staged keys, values
    uint8_t *codes[2], *scales[2];
    const float *unit[2];
    const int32_t *slots, *slot_start;
    int32_t *error_flag;
    int batch, W, pages, kv_heads, max_slots, pieces;
    unsigned jobs;
};

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {  // of sizes: NaN loses
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The exponent of the power of two that a unit stands for, -40 to 40.
__device__ __forceinline__ int unit_log(const float *unit, size_t at) {
    if (!unit) return 0;
    const uint32_t bits = __float_as_uint(unit[at]);
    return bits >> 31 ? 0 : min(max((int)(bits >> 23) - 127, -40), 40);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Eight elements of a row as codes (in the lowest bits of c), and the scale byte of the
// 32 that this and the three lanes beside it have.  Full warps.
struct Codes {
    uint32_t c[8];
    uint32_t byte;
};
__device__ __forceinline__ Codes quantise(uint4 x, int unit) {
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max_bf16x2(m, w[j] & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        nan = nan || (w[j] & 0x7fffu) > 0x7f80u || (w[j] >> 16 & 0x7fffu) > 0x7f80u;
    if (nan || m >= 0x7f80u) {  // the largest finite one; NaN as 0
        m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if ((w[j] & 0x7fffu) > 0x7f80u) w[j] &= 0xffff0000u;
            if ((w[j] >> 16 & 0x7fffu) > 0x7f80u) w[j] &= 0xffffu;
            if ((w[j] & 0x7fffu) < 0x7f80u) m = max(m, w[j] & 0x7fffu);
            if ((w[j] >> 16 & 0x7fffu) < 0x7f80u) m = max(m, w[j] >> 16 & 0x7fffu);
        }
    }
    m |= (uint32_t)nan << 16;
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        const uint32_t o = __shfl_xor_sync(kFull, m, d);
        m = max(m & 0xffffu, o & 0xffffu) | ((m | o) & 0x10000u);
    }
    const float t = __uint_as_float(m << 16) * exp2i(-unit) * (1.f / 7.f);
    uint32_t bits = __float_as_uint(t);
    Codes r;
    float s;
    if (t < 6.103515625e-05f) {  // 2^-14: multiples of 2^-17
        s = rintf(t * 131072.f);
        r.byte = (uint32_t)s;
        s *= 7.62939453125e-06f;
    } else {
        bits = (bits + 0x7ffffu + (bits >> 20 & 1u)) & 0xfff00000u;
        bits = min(bits, 0x42700000u);  // 60
        s = __uint_as_float(bits);
        r.byte = (bits >> 20) - (112u << 3);
    }
    const float inv = s > 0.f ? __frcp_rn(s) * exp2i(-unit) : 0.f, lim = s > 0.f ? 7.f : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float v = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
        const float q = fminf(fmaxf(fmaf(v, inv, 6144.f), 6144.f - lim), 6144.f + lim);
        r.c[j] = __float_as_uint(q + (12582912.f + 8.f - 6144.f)) & 15u;
    }
    if (m >> 16) r.byte = 0xffu;
    return r;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32) append_paged4_kernel(const Append4Args a) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kGroups = D / DAS_SCALE_GROUP;
    const int lane = threadIdx.x & 31, row = lane / kLanes, l = lane % kLanes, warp = threadIdx.x >> 5;
    unsigned x = blockIdx.x;
    const int job = (int)(x / a.jobs) * kWarps + warp;
    const int which = job >= a.kv_heads, h = job - (which ? a.kv_heads : 0);
    x %= a.jobs;
    const int piece = x % a.pieces;
    x /= a.pieces;
    const int b = x % a.batch;
    const size_t slab = x / a.batch;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (job >= 2 * a.kv_heads) return;

    const int s0 = a.slot_start[b];
    const long long n_all = (long long)a.slot_start[b + 1] - s0;
    if (n_all < 0 || n_all > a.W || s0 < 0 || s0 + n_all > a.max_slots) {
        if (lane == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    if (n_all == 0) return;
    int slot = a.slots[s0], begin = 0, end = (int)n_all;
    if (slot < 0) {
        if (lane == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    {  // the piece-th page that the tokens lie on
        const int t = piece * kPage - slot % kPage;  // the token at the page's first place
        if (t >= end) return;
        begin = max(t, 0);
        end = min(t + kPage, end);
        if (piece) slot = a.slots[s0 + begin];
    }
    const int page = slot / kPage, first = slot % kPage;
    if (slot < 0 || page >= a.pages || (piece && first)) {
        if (lane == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    const size_t tile = (slab * a.pages + page) * a.kv_heads + h;
    const size_t stride = (size_t)a.kv_heads * D;
    const int unit = unit_log(a.unit[which], slab * a.kv_heads + h);
    const uint4 *src = reinterpret_cast<const uint4 *>(a.fresh[which] + ((slab * a.batch + b) * a.W) * stride + h * D) + l;
    auto load = [&](int t) {  // token t's part, or zeros
        return t >= begin && t < end ? __ldcs(src + t * (stride / 8)) : make_uint4(0, 0, 0, 0);
    };
    uint8_t *const scales = a.scales[which] + tile * (kPage * kGroups);
    if (which == 0) {
        uint32_t *const codes = reinterpret_cast<uint32_t *>(a.codes[0] + tile * (kPage * D / 2)) + l;
#pragma unroll 4
        for (int t0 = begin; t0 < end; t0 += kRows) {
            const int t = t0 + row, place = first + t - begin;
            const Codes q = quantise(load(t), unit);
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) w |= q.c[j] << (4 * j);
            if (t < end) {
                codes[place * (D / 8)] = w;
                if (l % 4 == 0) scales[place * kGroups + l / 4] = (uint8_t)q.byte;
            }
        }
    } else {
        uint32_t *const codes = reinterpret_cast<uint32_t *>(a.codes[1] + tile * (kPage * D / 2));
        const int last = first + end - begin;  // the place past the last
        for (int o = first / 8; o * 8 < last; ++o) {  // eight places that share words
            const int t0 = begin + o * 8 - first;     // the token at the first of them
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 0;
            unsigned long long bytes = 0;
#pragma unroll
            for (int i = 0; i < 8 / kRows; ++i) {
                const int at = i * kRows + row;
                const Codes q = quantise(load(t0 + at), unit);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] |= q.c[j] << (4 * at);
                bytes |= (unsigned long long)q.byte << (8 * at);
            }
            // the other rows' bits: lane (row, l) is to store its elements [row 8 / kRows, ...)
#pragma unroll
            for (int d = kLanes; d < 32; d <<= 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] |= __shfl_xor_sync(kFull, w[j], d);
                bytes |= __shfl_xor_sync(kFull, bytes, d);
            }
            const int lo = max(first - o * 8, 0), hi = min(last - o * 8, 8);  // the new ones of the eight
            const uint32_t keep = ~(uint32_t)(((1ull << 4 * hi) - 1) & ~((1ull << 4 * lo) - 1));
            constexpr int kMine = 8 / kRows;
            uint32_t *const dst = codes + o * D + 8 * l + kMine * row;
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                uint32_t v = w[j];
#pragma unroll
                for (int r = 1; r < kRows; ++r)
                    if (row == r) v = w[r * kMine + j];
                if (keep) v = (v & ~keep) | (dst[j] & keep);
                dst[j] = v;
            }
            if (row == 0 && l % 4 == 0) {
                uint8_t *const at = scales + (l / 4) * kPage + o * 8;
                if (!keep) *reinterpret_cast<unsigned long long *>(at) = bytes;
                else
                    for (int i = lo; i < hi; ++i) at[i] = (uint8_t)(bytes >> 8 * i);
            }
        }
    }
}

}  // namespace

cudaError_t append_paged4_launch(const das_kv_cache_paged4 &c, const void *k_new, const void *v_new,
                                 int batch, int W, const int32_t *slots, int max_slots,
                                 const int32_t *slot_start, int32_t *error_flag, cudaStream_t stream) {
    Append4Args a = {};
    a.fresh[0] = static_cast<const uint16_t *>(k_new);
    a.fresh[1] = static_cast<const uint16_t *>(v_new);
    a.codes[0] = static_cast<uint8_t *>(c.k);
    a.codes[1] = static_cast<uint8_t *>(c.v);
    a.scales[0] = static_cast<uint8_t *>(c.k_scale);
    a.scales[1] = static_cast<uint8_t *>(c.v_scale);
    a.unit[0] = c.k_unit;
    a.unit[1] = c.v_unit;
    a.slots = slots;
    a.slot_start = slot_start;
    a.error_flag = error_flag;
    a.batch = batch;
    a.W = W;
    a.pages = c.pages;
    a.kv_heads = c.kv_heads;
    a.max_slots = max_slots;
    a.pieces = (W + 2 * kPage - 2) / kPage;
    const long long jobs = (long long)c.depths * c.layers * batch * a.pieces;
    const long long ctas = jobs * ((2LL * c.kv_heads + kWarps - 1) / kWarps);
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
    a.jobs = (unsigned)jobs;
    if (ctas == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, c.head_dim == 128 ? append_paged4_kernel<128> : append_paged4_kernel<64>, a);
}

}  // namespace das
