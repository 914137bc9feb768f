// das_paged4.cu -- the commit into the paged 4-bit cache: codes of 4 bits under a scale of
// a byte for every 32 elements of a token's head.
//
// The mathematics.  A scale has 4 significant bits and a bf16 element 8, so a quotient x / s
// is a half or no nearer to one than 1/255 of itself: x times a reciprocal that is off by 2^-22,
// rounded once more to multiples of 2^-11 (by adding 6144), decides a code as the quotient does.
// A scale is rounded down by 1/17 of itself at most, so the largest quotient is below 7.5 and needs
// no bound but where a scale is below 2^-14 (multiples of 2^-17), is cut at 60, or a group has an
// infinity or NaN: such a warp takes the general way (quantise), token by token.
//
// A warp to the tokens on a page of (sequence, slab, keys or values, kv head).  D / 8 lanes have a token's row, 8 elements each, so that a scale is a matter
// of four lanes; each of them has four tokens at once and makes the scale of one.
// A code is the low bits of a sum with 1.5 2^23, and codes are put together by
// multiply-adds of such sums, whose high parts a constant takes away.  Keys lie token by
// token and go straight out.  Of the values eight tokens share a word: a lane collects its
// elements' bits over its tokens and changes half of the words for the same half of the lanes
// that have the other tokens.  Words that older tokens share are read first and keep their bits.
//
// Bound by memory for long appends: 4 sequences of 501 to 1001 tokens at 8 depths and 4 layers,
// 8 heads of 128, take 96.8 us, 5.5 TB/s (81% of the copy rate); 8 of 8 to 16 tokens at 32 depths
// 23.6 us, instructions of passes of eight tokens that are partly there and the chain of
// look-ups before them.  64 registers and 32 warps to an SM are the best of both: with 80
// the long one takes 102 us.  Loads of the next pass ahead of this one's work made that 95 us, but the
// short one 25; several pieces of work to a warp in turn 98 and 23.
//
// The kernel is launched as a programmatic dependent of the previous kernel in the
// stream: it reads nothing before griddepcontrol.wait, and every CTA executes that wait.
#include <algorithm>
#include <type_traits>

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
    int jobs, splits;  // (slab, keys or values, head)s, and the CTAs that they take
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
__device__ __noinline__ Codes quantise(uint4 x, int unit) {
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

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 8) append_paged4_kernel(const Append4Args a) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kGroups = D / DAS_SCALE_GROUP;
    constexpr int kPass = 4 * kRows, kOcts = kPass / 8;  // tokens at once, and eights of them
    constexpr uint32_t kMagic = 0x4b400000u;             // 1.5 2^23
    const int lane = threadIdx.x & 31, row = lane / kLanes, l = lane % kLanes, warp = threadIdx.x >> 5;
    const int quarter = lane & 3;
    const int part = blockIdx.x % a.splits, piece = blockIdx.x / a.splits % a.pieces;
    const int b = blockIdx.x / a.splits / a.pieces;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int s0 = a.slot_start[b];
    const long long n_all = (long long)a.slot_start[b + 1] - s0;
    if (n_all < 0 || n_all > a.W || s0 < 0 || s0 + n_all > a.max_slots) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    if (n_all == 0) return;
    int slot = a.slots[s0], begin = 0, end = (int)n_all;
    if (slot < 0) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    {  // the piece-th page that the tokens lie on
        const int t = piece * kPage - slot % kPage;  // the token at the page's first place
        if (t >= end) return;
        begin = max(t, 0);
        end = min(t + kPage, end);
        if (piece) slot = a.slots[s0 + begin];
    }
    const int page = slot / kPage, first = slot % kPage, last = first + end - begin;
    if (slot < 0 || page >= a.pages || (piece && first)) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    const size_t stride = (size_t)a.kv_heads * D;
    const int job = part * kWarps + warp;
    if (job >= a.jobs) return;
    const int h = job % a.kv_heads, which = job / a.kv_heads & 1;
    const size_t slab = job / a.kv_heads / 2;
    const size_t tile = (slab * a.pages + page) * a.kv_heads + h;
    const int unit = unit_log(a.unit[which], slab * a.kv_heads + h);
    const float per_unit = exp2i(-unit);
    // of the token at place 0 of the page (not read before `first`)
    const uint16_t *src = a.fresh[which] + ((long long)((slab * a.batch + b) * a.W) + begin - first) * (long long)stride +
                          h * D + 8 * l;
    uint8_t *const scales = a.scales[which] + tile * (kPage * kGroups);
    uint32_t *const codes = reinterpret_cast<uint32_t *>(a.codes[which] + tile * (kPage * D / 2));
    // (values by whole words; keys have no need to)
    for (int p0 = which ? first / 8 * 8 : first; p0 < last; p0 += kPass) {
        auto place = [&](int i) { return p0 + i * kRows + row; };
        auto fresh = [&](int p) { return p >= first && p < last; };
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            if (fresh(place(i))) x[i] = __ldcs(reinterpret_cast<const uint4 *>(src + place(i) * (long long)stride));
        }
        // the largest sizes of four tokens, two to a word, and of this lane's one of them
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = max_u16x2(max_u16x2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                             max_u16x2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
            if (!fresh(place(i))) m[i] = 0x3f80u;  // (any that needs no care)
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m[i] = max_u16x2(__byte_perm(m[i], m[i + 2], 0x5410), __byte_perm(m[i], m[i + 2], 0x7632));
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) m[i] = max_u16x2(m[i], __shfl_xor_sync(kFull, m[i], d));
        }
        const uint32_t both = quarter & 1 ? m[1] : m[0], most = quarter & 2 ? both >> 16 : both & 0xffffu;
        const float t = __uint_as_float(most << 16) * per_unit * (1.f / 7.f);
        uint32_t bits = __float_as_uint(t);
        bits = (bits + 0x7ffffu + (bits >> 20 & 1u)) & 0xfff00000u;
        uint32_t byte = (bits >> 20) - (112u << 3);
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__uint_as_float(bits)));
        inv *= per_unit;
        uint32_t w[4][8];  // 0x4b400000 + code
        if (__any_sync(kFull, most >= 0x7f80u || t < 6.103515625e-05f || bits > 0x42700000u)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Codes q = quantise(x[i], unit);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[i][j] = kMagic + q.c[j];
                if (quarter == i) byte = q.byte;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = __shfl_sync(kFull, inv, (lane & ~3) + i);
                const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    w[i][j] = __float_as_uint(fmaf(__uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16), f,
                                                   6144.f) + (12582912.f + 8.f - 6144.f));
            }
        }
        {
            const int p = p0 + quarter * kRows + row;
            if (fresh(p)) scales[which ? l / 4 * kPage + p : p * kGroups + l / 4] = (uint8_t)byte;
        }
        if (which == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t c = -(kMagic * 0x11111111u);
#pragma unroll
                for (int j = 0; j < 8; ++j) c += w[i][j] << (4 * j);
                if (fresh(place(i))) codes[place(i) * (D / 8) + l] = c;
            }
            continue;
        }
        const uint32_t at_row = 1u << 4 * row;  // (the token's place in the word)
#pragma unroll
        for (int o = 0; o < kOcts; ++o) {
            constexpr int kEach = 4 / kOcts;  // a lane's tokens of the eight
            uint32_t c[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t sum = -(kMagic * (kEach == 4 ? 0x01010101u : 0x00010001u));
#pragma unroll
                for (int i = 0; i < kEach; ++i) sum += w[o * kEach + i][j] << (4 * kRows * i);
                c[j] = sum * at_row;
            }
            // half of the words for the other half of the lanes' tokens, until all eight are in
#pragma unroll
            for (int d = 16, n = 4; d >= kLanes; d >>= 1, n >>= 1) {
                const bool up = lane & d;
#pragma unroll
                for (int j = 0; j < n; ++j) {
                    const uint32_t give = up ? c[j] : c[j + n], mine = up ? c[j + n] : c[j];
                    c[j] = mine | __shfl_xor_sync(kFull, give, d);
                }
            }
            constexpr int kMine = 8 / kRows;
            const int p = p0 + o * 8;  // the place of the first of the eight
            const int lo = max(first - p, 0), hi = min(last - p, 8);  // the new ones
            if (lo >= hi) continue;
            const uint32_t keep = ~(uint32_t)(((1ull << 4 * hi) - 1) & ~((1ull << 4 * lo) - 1));
            using Out = std::conditional_t<kMine == 4, uint4, uint2>;
            // the first of the words that are left here: those of half the lanes' elements, halved
            const int j0 = kMine == 4 ? (lane & 16 ? 4 : 0) : (lane & 16 ? 4 : 0) + (lane & 8 ? 2 : 0);
            Out *const dst = reinterpret_cast<Out *>(codes + p / 8 * D + 8 * l + j0);
            if (keep) {
                const Out old = *dst;
                const uint32_t *const was = reinterpret_cast<const uint32_t *>(&old);
#pragma unroll
                for (int j = 0; j < kMine; ++j) c[j] = (c[j] & ~keep) | (was[j] & keep);
            }
            if constexpr (kMine == 4) *dst = make_uint4(c[0], c[1], c[2], c[3]);
            else *dst = make_uint2(c[0], c[1]);
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
    if (batch == 0 || W == 0) return cudaSuccess;
    const long long jobs = 2LL * c.depths * c.layers * c.kv_heads;
    if (jobs > 0x7fffffffLL / 2) return cudaErrorInvalidValue;
    a.jobs = (int)jobs;
    a.splits = (int)((jobs + kWarps - 1) / kWarps);
    const long long ctas = (long long)a.splits * a.pieces * batch;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
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
