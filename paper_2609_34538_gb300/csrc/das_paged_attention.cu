// das_paged_attention.cu -- depth-asynchronous attention (Eqs. 2-3) over the
// paged e4m3 cache with a scale per (page, kv head).
//
// Plain form: one CTA takes a range of the 64-key tiles of one (sequence, kv
// head) pair (a tile is a page; the block's own keys are the last tile),
// widens each tile to fp32 in shared memory and keeps the running maximum,
// sum and output of every row in registers; merge_kernel combines the ranges.
#include <cuda_bf16.h>

#include <algorithm>

#include "das_internal.h"

namespace das {
namespace {

constexpr int kThreads = 128;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float bf16(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float e4m3(uint8_t x) {
    uint32_t h;
    asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}\n"
        : "=r"(h)
        : "r"((uint32_t)x));
    float f;
    asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %1;\n cvt.f32.f16 %0, l;\n}\n" : "=f"(f) : "r"(h));
    return f;
}
__device__ __forceinline__ int clamped(int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); }

template <int D>
__global__ void __launch_bounds__(kThreads) paged_attn_kernel(const PagedAttnParams p, int splits) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ float sm[];
    float *qs = sm, *kv = qs + 64 * (D + 1), *ps = kv + 64 * (D + 1);
    const int s = blockIdx.x % splits, pair = blockIdx.x / splits;
    const int b = pair / p.Hkv, h = pair % p.Hkv;
    const int P = clamped(p.prefix_len[b], p.max_pages * 64), T = clamped(p.block_len[b], p.max_block);
    if (s == 0 && threadIdx.x == 0 && (P != p.prefix_len[b] || T != p.block_len[b]))
        atomicOr(p.status, kStatusClamped);
    const int nt = (P + 63) / 64 + 1;
    const int lo = (int)((long long)nt * s / splits), hi = (int)((long long)nt * (s + 1) / splits);
    const int rows = p.G * T, row = threadIdx.x >> 1, half = threadIdx.x & 1;
    const int irow = row / p.G;
    for (int i = threadIdx.x; i < rows * D; i += kThreads) {
        const int r = i / D, d = i % D;
        qs[r * (D + 1) + d] = bf16(
            p.q[(((size_t)b * p.max_block + r / p.G) * p.Hq + h * p.G + r % p.G) * D + d]);
    }
    float m = -INFINITY, l = 0.f, acc[D / 2];
    for (int d = 0; d < D / 2; ++d) acc[d] = 0.f;
    for (int t = lo; t < hi; ++t) {
        const bool blk = t == nt - 1;
        int n = blk ? T : min(64, P - t * 64);
        const int page = blk ? 0 : p.table[(size_t)b * p.max_pages + t];
        if (page < 0 || page >= p.pages) {
            if (threadIdx.x == 0) atomicOr(p.status, kStatusBadPage);
            n = 0;
        }
        const size_t tile = n ? (size_t)page * p.Hkv + h : 0;
        auto fill = [&](const uint8_t *codes, float scale, const uint16_t *own) {
            __syncthreads();
            for (int i = threadIdx.x; i < n * D; i += kThreads) {
                const int j = i / D, d = i % D;
                kv[j * (D + 1) + d] =
                    blk ? bf16(own[(((size_t)b * p.max_block + j) * p.Hkv + h) * D + d])
                        : e4m3(codes[tile * 64 * D + i]) * scale;
            }
            __syncthreads();
        };
        fill(p.k, p.k_scale[tile], p.k_blk);
        const int lim = row < rows ? (blk ? min(n, irow + 1) : n) : 0;
        float mt = m;
        for (int j = half; j < lim; j += 2) {
            float x = 0.f;
            for (int d = 0; d < D; ++d) x += qs[row * (D + 1) + d] * kv[j * (D + 1) + d];
            x *= p.scale_log2;
            ps[row * 65 + j] = x;
            mt = fmaxf(mt, x);
        }
        mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, 1));
        const float alpha = m == -INFINITY ? 0.f : exp2f(m - mt);
        m = mt;
        l *= alpha;
        for (int d = 0; d < D / 2; ++d) acc[d] *= alpha;
        for (int j = half; j < lim; j += 2) {
            const float w = exp2f(ps[row * 65 + j] - m);
            ps[row * 65 + j] = w;
            l += w;
        }
        fill(p.v, p.v_scale[tile], p.v_blk);
        for (int j = 0; j < lim; ++j) {
            const float w = ps[row * 65 + j];
#pragma unroll
            for (int d = 0; d < D / 2; ++d) acc[d] += w * kv[j * (D + 1) + half + 2 * d];
        }
    }
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    if (row < p.rows_max) {
        const size_t at = (size_t)blockIdx.x * p.rows_max + row;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        for (int d = 0; d < D / 2; ++d) p.part_o[at * D + half + 2 * d] = acc[d] * inv;
        if (half == 0) p.part_lse[at] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
}

template <int D>
__global__ void __launch_bounds__(D) paged_merge_kernel(const PagedAttnParams p, int splits) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int row = blockIdx.x % p.rows_max, pair = blockIdx.x / p.rows_max;
    const int b = pair / p.Hkv, h = pair % p.Hkv, d = threadIdx.x;
    float M = -INFINITY, L = 0.f, o = 0.f;
    const float *ls = p.part_lse + (size_t)pair * splits * p.rows_max + row;
    for (int s = 0; s < splits; ++s) M = fmaxf(M, ls[(size_t)s * p.rows_max]);
    for (int s = 0; s < splits; ++s) {
        const float w = M == -INFINITY ? 0.f : expf(ls[(size_t)s * p.rows_max] - M);
        L += w;
        o += w * p.part_o[(((size_t)pair * splits + s) * p.rows_max + row) * D + d];
    }
    const int i = row / p.G, g = h * p.G + row % p.G;
    const __nv_bfloat16 r = __float2bfloat16_rn(L > 0.f ? o / L : 0.f);
    p.out[(((size_t)b * p.max_block + i) * p.Hq + g) * D + d] = __bfloat16_as_ushort(r);
    if (d == 0)
        p.lse[((size_t)b * p.Hq + g) * p.max_block + i] = L > 0.f ? M + logf(L) : -INFINITY;
}

int splits_of(int device, int batch, int kv_heads) {
    const int C = attn_grid_size(device);
    return C <= 0 ? 0 : (int)std::max<long long>(1, 2ll * C / ((long long)batch * kv_heads));
}
size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

template <int D>
cudaError_t launch_d(const PagedAttnParams &p, int splits, cudaStream_t stream) {
    constexpr int smem = (2 * 64 * (D + 1) + 64 * 65) * 4;
    cudaError_t e = cudaFuncSetAttribute(paged_attn_kernel<D>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    paged_attn_kernel<D><<<p.B * p.Hkv * splits, kThreads, smem, stream>>>(p, splits);
    paged_merge_kernel<D><<<p.B * p.Hkv * p.rows_max, D, 0, stream>>>(p, splits);
    return cudaGetLastError();
}

}  // namespace

size_t paged_workspace_bytes(int device, int batch, int kv_heads, int rows_max, int head_dim) {
    const size_t slots = (size_t)batch * kv_heads * splits_of(device, batch, kv_heads);
    if (slots == 0) return 0;
    return kWorkspaceHeader + round256(slots * rows_max * head_dim * sizeof(float)) +
           round256(slots * rows_max * sizeof(float));
}

cudaError_t paged_attn_launch(PagedAttnParams &p, int head_dim, void *workspace,
                              cudaStream_t stream) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int splits = splits_of(dev, p.B, p.Hkv);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    p.status = reinterpret_cast<int32_t *>(ws);
    p.part_o = reinterpret_cast<float *>(ws + kWorkspaceHeader);
    p.part_lse = reinterpret_cast<float *>(
        ws + kWorkspaceHeader +
        round256((size_t)p.B * p.Hkv * splits * p.rows_max * head_dim * sizeof(float)));
    return head_dim == 128 ? launch_d<128>(p, splits, stream) : launch_d<64>(p, splits, stream);
}

}  // namespace das
