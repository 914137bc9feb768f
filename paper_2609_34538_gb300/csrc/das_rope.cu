// das_rope.cu -- norms of queries and keys per head, their rotation by position, and the
// copy of values, from a projection's rows into the attention calls' tensors.
//
// A warp takes one token's heads, or a part of them.  D / 8 lanes have a head's row, a
// lane 8 of its elements: the two elements of every rotated pair are the same lane's, so
// rows need no exchange but the sum of squares, and any output may overwrite its
// input.  The angle n f_j is taken in turns as a 64-bit fraction: n times f_j / (2 pi)
// modulo 1 is an integer product whose overflow is what is not wanted.  (f_j / (2 pi) is
// cut to 2^-64, 1 / (2 pi) to 2^-66, so n f_j is off by n (f_j 2^-66 + 2^-64) turns at most.)
// The lane's four angles serve all of the token's heads.
//
// Bound by memory, reads and writes of 2 bytes an element each.  4 x 2001 tokens of prompts of 500
// to 2001, 48 heads of 128, take 25.3 us, 69% of the measured copy rate, 16 x 16 tokens with half of the
// head rotated 4.4 us, a single token 3.2 us.  As measured when they were chosen, in a loop on the same rows:
// 23.8 us, without two steps' loads before the first use 28.1, with four steps' 22.6, but then 16 x 16 tokens
// took 5.7 us instead of 5.3; with 40 warps to an SM instead of 32, whose registers spill, 30 and more.
// Angles in doubles took 13 us more, as doubles are slow.  The choice of what is not rotated takes 0.2 us.
#include <algorithm>

#include "das_internal.h"

namespace das {
namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kWarps = 4;

struct RopeParams {
    RopeArgs a;
    int heads, part, parts;  // all heads of a token, of one warp, warps to a token
};

__device__ __forceinline__ void unpack(uint2 u, float *x) {
    x[0] = __uint_as_float(u.x << 16);
    x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16);
    x[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void weights(const void *w, bool bf16, int unit, float *x) {
    if (!w) {
        x[0] = x[1] = x[2] = x[3] = 1.f;
    } else if (bf16) {
        unpack(__ldg(static_cast<const uint2 *>(w) + unit), x);
    } else {
        const float4 f = __ldg(static_cast<const float4 *>(w) + unit);
        x[0] = f.x;
        x[1] = f.y;
        x[2] = f.z;
        x[3] = f.w;
    }
}

// f / (2 pi) modulo 1 in steps of 2^-64: the significand times the first 64 bits of 1 / (2 pi).
__device__ __forceinline__ unsigned long long turns(float f) {
    constexpr unsigned long long kInverse = 0xa2f9836e4e441529ull;  // 2^66 / (2 pi)
    const uint32_t bits = __float_as_uint(f), e = bits >> 23 & 0xffu;
    if (e == 0xffu) return 0;
    const uint32_t m = (bits & 0x7fffffu) | (e ? 0x800000u : 0u);
    const unsigned long long low = (unsigned long long)m * (uint32_t)kInverse,
                             high = (unsigned long long)m * (uint32_t)(kInverse >> 32) + (low >> 32);
    // the product, high 2^32 + (the lower half of low), times 2^-down
    const int down = 152 - (int)max(e, 1u);
    unsigned long long t;
    if (down >= 32) t = down < 96 ? high >> (down - 32) : 0;
    else if (down >= 0) t = (high << 32 | (uint32_t)low) >> down | (down ? high >> 32 << (64 - down) : 0);
    else t = down > -64 ? (high << 32 | (uint32_t)low) << -down : 0;
    return bits >> 31 ? 0 - t : t;
}

// PAIRS: neighbours are turned together, otherwise elements of two halves.
template <int D, bool PAIRS>
__global__ void __launch_bounds__(kWarps * 32, 8) rope_kernel(const RopeParams p) {
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // lanes to a head, heads at once
    constexpr int kBatch = 2;                           // steps whose loads are made together
    const RopeArgs &a = p.a;
    const int lane = threadIdx.x & 31, l = lane % kLanes, r = lane / kLanes;
    const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int part = (int)(item % p.parts);
    const long long token = item / p.parts;
    const int i = (int)(token % a.max_block);
    const long long b = token / a.max_block;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (b >= a.batch || (a.block_len && i >= a.block_len[b])) return;

    // the lane's two units of four elements
    const int rd8 = a.rotary_dim / 8;
    const bool turned = l < rd8;
    const int u0 = PAIRS ? 2 * l : turned ? l : 2 * l, u1 = PAIRS || !turned ? 2 * l + 1 : l + rd8;
    // (cs 2: of a pair that nothing turns, which passes as it is, as 0 times an infinity beside it would be NaN)
    float cs[4], sn[4];
    {
        const unsigned long long n = (a.prefix_len ? max(a.prefix_len[b], 0) : 0) + (long long)i;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            cs[j] = 2.f;
            sn[j] = 0.f;
            if (!turned) continue;
            const float f = a.inv_freq[4 * l + j];
            const float x = (float)(int)(n * turns(f) >> 32) * 4.656612873077393e-10f;  // half turns, 2^-31
            sincospif(x, &sn[j], &cs[j]);
            if (!(fabsf(f) < INFINITY)) cs[j] = 2.f;
        }
    }
    const bool some_still = __any_sync(kFull, cs[0] > 1.5f || cs[1] > 1.5f || cs[2] > 1.5f || cs[3] > 1.5f);
    // the heads of a kind that are this warp's
    int kind_begin = 0;
#pragma unroll 1
    for (int kind = 0; kind < 3; ++kind) {
        const int n = kind == 0 ? a.num_q_heads : a.kv_heads;
        const int begin = max(part * p.part - kind_begin, 0), end = min((part + 1) * p.part - kind_begin, n);
        kind_begin += n;
        const das_head_rows &src = a.in[kind];
        if (!src.data || begin >= end) continue;
        const uint16_t *const in = static_cast<const uint16_t *>(src.data) + b * src.batch_stride + i * src.token_stride;
        uint16_t *const out = static_cast<uint16_t *>(a.out[kind]) + (b * a.max_block + i) * n * D;
        float w[8];
        if (kind < 2) {
            weights(a.weight[kind], a.weights_bf16, u0, w);
            weights(a.weight[kind], a.weights_bf16, u1, w + 4);
        }
        for (int h0 = begin + r; h0 - r < end; h0 += kBatch * kRows) {
            uint2 x0[kBatch], x1[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int h = h0 + k * kRows;
                x0[k] = x1[k] = make_uint2(0, 0);
                if (h < end) {
                    const uint16_t *const row = in + h * src.head_stride;
                    x0[k] = *reinterpret_cast<const uint2 *>(row + 4 * u0);
                    x1[k] = *reinterpret_cast<const uint2 *>(row + 4 * u1);
                }
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int h = h0 + k * kRows;
                if (h - r >= end) break;
                if (kind < 2) {
                    float y[8];
                    unpack(x0[k], y);
                    unpack(x1[k], y + 4);
                    if (a.eps >= 0.f) {
                        float sum = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum += y[j] * y[j];
#pragma unroll
                        for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(kFull, sum, d);
                        const float f = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = y[j] * f * w[j];
                    }
                    float z[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // pair j: elements j of both units, or 2 j and 2 j + 1 of the eight
                        const float s = PAIRS ? y[2 * j] : y[j], t = PAIRS ? y[2 * j + 1] : y[j + 4];
                        const float zs = s * cs[j] - t * sn[j], zt = t * cs[j] + s * sn[j];
                        z[j] = zs;
                        z[j + 4] = zt;
                    }
                    if (some_still)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (cs[j] > 1.5f) {
                                z[j] = PAIRS ? y[2 * j] : y[j];
                                z[j + 4] = PAIRS ? y[2 * j + 1] : y[j + 4];
                            }
                    if (PAIRS) {
                        x0[k] = make_uint2(pack(z[0], z[4]), pack(z[1], z[5]));
                        x1[k] = make_uint2(pack(z[2], z[6]), pack(z[3], z[7]));
                    } else {
                        x0[k] = make_uint2(pack(z[0], z[1]), pack(z[2], z[3]));
                        x1[k] = make_uint2(pack(z[4], z[5]), pack(z[6], z[7]));
                    }
                }
                if (h < end) {
                    uint16_t *const row = out + h * D;
                    *reinterpret_cast<uint2 *>(row + 4 * u0) = x0[k];
                    *reinterpret_cast<uint2 *>(row + 4 * u1) = x1[k];
                }
            }
        }
    }
}

}  // namespace

cudaError_t rope_launch(const RopeArgs &a, int head_dim, cudaStream_t stream) {
    RopeParams p = {};
    p.a = a;
    p.heads = a.num_q_heads + a.kv_heads * (a.in[2].data ? 2 : 1);
    const long long tokens = (long long)a.batch * a.max_block;
    if (tokens == 0) return cudaSuccess;
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int sms = attn_grid_size(dev);
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int rows = 256 / head_dim;  // heads that a warp takes at once
    // warps to a token until there are 16 to an SM, each with whole steps (as measured when it was chosen, 16 x 16
    // tokens of 4 to 16 and 16 x 64: 4.2 and 6.8 us; until there are 8 4.5 and 7.5, 24 5.3 and 6.8; 256 tokens
    // 5.4, 4.7 and 6.7)
    p.part = p.heads;
    while (p.part > rows && tokens * ((p.heads + p.part - 1) / p.part) < (long long)sms * 16) p.part = (p.part / 2 + rows - 1) / rows * rows;
    p.parts = (p.heads + p.part - 1) / p.part;
    const long long ctas = (tokens * p.parts + kWarps - 1) / kWarps;
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
    void (*const kernel)(RopeParams) = head_dim == 128 ? (a.interleaved ? rope_kernel<128, true> : rope_kernel<128, false>)
                                                       : (a.interleaved ? rope_kernel<64, true> : rope_kernel<64, false>);
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace das
