// das_paged4_attention.cu -- depth-asynchronous attention (Eqs. 2-3) over the paged 4-bit
// cache.
//
// One CTA to a query row: its warps take every fourth key, a running maximum and sum
// each, and join at the end.
#include <algorithm>

#include "das_internal.h"
#include "das_tcgen05.h"

namespace das {
namespace {

using t5::kFull;
constexpr int kWarps = 4;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float scale_of(uint8_t byte) {
    float lo, hi;
    t5::unpack_f16((uint32_t)byte << 7, lo, hi);
    return lo;
}
__device__ __forceinline__ float unit_of(const float *unit, int h) {
    if (!unit) return 1.f;
    const uint32_t bits = __float_as_uint(unit[h]);
    const int e = bits >> 31 ? 0 : min(max((int)(bits >> 23) - 127, -40), 40);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}
__device__ __forceinline__ float bf(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

template <int D>
__global__ void __launch_bounds__(kWarps * 32) paged4_row_kernel(const Paged4AttnParams p) {
    constexpr int V = D / 32;
    __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row = blockIdx.x % p.rows_max, pair = blockIdx.x / p.rows_max;
    const int b = pair / p.Hkv, h = pair % p.Hkv, i = row / p.G, hq = h * p.G + row % p.G;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int P0 = p.prefix_len[b], T0 = p.block_len[b];
    const int P = min(max(P0, 0), p.max_pages * kTileKeys), T = min(max(T0, 0), p.max_block);
    if ((P != P0 || T != T0) && threadIdx.x == 0) atomicOr(p.status, kStatusClamped);
    uint16_t *out = p.out + (((size_t)b * p.max_block + i) * p.Hq + hq) * D;
    float *lse = p.lse + ((size_t)b * p.Hq + hq) * p.max_block + i;
    if (i >= T) {
        for (int d = threadIdx.x; d < D; d += kWarps * 32) out[d] = 0;
        if (threadIdx.x == 0) *lse = -INFINITY;
        return;
    }
    const float ku = unit_of(p.k_unit, h), vu = unit_of(p.v_unit, h);
    float q[V], o[V], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        q[j] = bf(p.q[(((size_t)b * p.max_block + i) * p.Hq + hq) * D + 32 * j + lane]);
        o[j] = 0.f;
    }
    for (int key = warp; key < P + i + 1; key += kWarps) {
        float k[V], v[V];
        if (key < P) {
            const int page = p.table[(size_t)b * p.max_pages + key / kTileKeys], t = key % kTileKeys;
            if (page < 0 || page >= p.pages) {
                atomicOr(p.status, kStatusBadPage);
                continue;
            }
            const size_t tile = (size_t)page * p.Hkv + h;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int d = 32 * j + lane;
                const int ck = p.k[(tile * kTileKeys + t) * (D / 2) + d / 2] >> (4 * (d & 1)) & 15;
                const int cv = p.v[((tile * 8 + t / 8) * D + d) * 4 + t % 8 / 2] >> (4 * (t & 1)) & 15;
                k[j] = (float)(ck - 8) * scale_of(p.k_scale[(tile * kTileKeys + t) * V + j]) * ku;
                v[j] = (float)(cv - 8) * scale_of(p.v_scale[(tile * V + j) * kTileKeys + t]) * vu;
            }
        } else {
            const size_t at = (((size_t)b * p.max_block + (key - P)) * p.Hkv + h) * D + lane;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                k[j] = bf(p.k_blk[at + 32 * j]);
                v[j] = bf(p.v_blk[at + 32 * j]);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) s += q[j] * k[j];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(kFull, s, d);
        s *= p.scale_log2;
        const float n = fmaxf(m, s), c = m == -INFINITY ? 0.f : exp2f(m - n), w = s == -INFINITY ? 0.f : exp2f(s - n);
        m = n;
        l = l * c + w;
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = o[j] * c + w * v[j];
    }
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) s_o[warp][32 * j + lane] = o[j];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w]);
    const float M0 = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < kWarps; ++w) L += s_l[w] * exp2f(s_m[w] - M0);
    for (int d = threadIdx.x; d < D; d += kWarps * 32) {
        float x = 0.f;
        for (int w = 0; w < kWarps; ++w) x += s_o[w][d] * exp2f(s_m[w] - M0);
        out[d] = (uint16_t)t5::pack_bf16(L == 0.f ? 0.f : x / L, 0.f);
    }
    if (threadIdx.x == 0) *lse = L == 0.f ? -INFINITY : (M0 + log2f(L)) * kLn2;
}

}  // namespace

size_t paged4_workspace_bytes(int device, int batch, int kv_heads, int rows_max, int head_dim) {
    return kWorkspaceHeader;
}

cudaError_t paged4_attn_launch(Paged4AttnParams &p, int head_dim, void *workspace, cudaStream_t stream) {
    p.status = static_cast<int32_t *>(workspace);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.B * p.Hkv * p.rows_max));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, head_dim == 128 ? paged4_row_kernel<128> : paged4_row_kernel<64>, p);
}

}  // namespace das
