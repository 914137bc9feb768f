// das_paged.cu -- the paged cache's bookkeeping: block tables and slot maps
// from request lengths, and the commit that stores tokens as e4m3 codes with
// a scale per (page, kv head).
//
// Every kernel here is launched as a programmatic dependent of the previous
// kernel in the stream: it reads nothing before griddepcontrol.wait, and
// every CTA executes that wait.
#include <algorithm>

#include "das_internal.h"

namespace das {
namespace {

constexpr int kPage = DAS_PAGE_TOKENS;
constexpr uint32_t kFull = 0xffffffffu;

template <typename... Params, typename... Args>
cudaError_t launch_pdl(void (*kernel)(Params...), dim3 grid, dim3 block, cudaStream_t stream,
                       Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

// ---- page assignment ----------------------------------------------------------
constexpr int kAssignThreads = 1024;

// What one request asks for.
struct Ask {
    int have, want;      // pages before and after
    long long old_len, new_len;
    bool grows, fits, bad;
};

__device__ __forceinline__ Ask ask_of(const PageAssignArgs &a, int b) {
    Ask r = {};
    if (b >= a.batch) return r;
    const long long row = (long long)a.max_pages * kPage;
    const long long len = a.seq_len[b], g = a.grow[b];
    r.old_len = len < 0 ? 0 : (len > row ? row : len);
    r.bad = r.old_len != len;
    r.new_len = r.old_len + g < 0 ? 0 : r.old_len + g;
    r.grows = g > 0;
    r.fits = r.grows && r.new_len <= row;
    r.have = (int)((r.old_len + kPage - 1) / kPage);
    r.want = (int)((min(r.new_len, row) + kPage - 1) / kPage);
    return r;
}

// Exclusive sum over the CTA's threads; total is the sum of all.
__device__ __forceinline__ long long scan(long long v, long long &total, long long *sums) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    long long x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(kFull, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        long long s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(kFull, s, d);
            if (lane >= d) s += y;
        }
        sums[lane] = s;
    }
    __syncthreads();
    total = sums[31];
    const long long r = x - v + (warp > 0 ? sums[warp - 1] : 0);
    __syncthreads();  // sums may be written again
    return r;
}

__global__ void __launch_bounds__(kAssignThreads) page_assign_kernel(const PageAssignArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ long long sums[32];
    __shared__ int s_first[kAssignThreads], s_have[kAssignThreads], s_num[kAssignThreads],
        s_at[kAssignThreads];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int listed = *a.free_count;
    const int count = listed < 0 ? 0 : (listed > a.pages ? a.pages : listed);
    int flag = listed != count ? kFlagInvalid : 0;

    // pages given back, in request order
    long long gave = 0;
    for (int c0 = 0; c0 < a.batch; c0 += kAssignThreads) {
        const Ask r = ask_of(a, c0 + tid);
        if (r.bad) flag |= kFlagInvalid;
        const int give = r.grows ? 0 : r.have - r.want;
        long long total;
        const long long ex = scan(give, total, sums);
        s_first[tid] = r.want;
        s_num[tid] = give;
        s_at[tid] = (int)min(count + gave + ex, (long long)a.pages);
        __syncthreads();
        for (int i = warp; i < min(kAssignThreads, a.batch - c0); i += kAssignThreads / 32)
            for (int j = lane; j < s_num[i]; j += 32) {
                const long long at = (long long)s_at[i] + j;
                if (at < a.pages)
                    a.free_pages[at] = a.table[(size_t)(c0 + i) * a.max_pages + s_first[i] + j];
                else
                    flag |= kFlagInvalid;  // more pages than the pool has
            }
        gave += total;
        __syncthreads();
    }
    const long long avail = min(count + gave, (long long)a.pages);

    long long asked_pages = 0, asked_slots = 0, took = 0, placed = 0;
    for (int c0 = 0; c0 < a.batch; c0 += kAssignThreads) {
        const int b = c0 + tid;
        const Ask r = ask_of(a, b);
        const int need = r.fits ? r.want - r.have : 0;
        const long long more = r.fits ? r.new_len - r.old_len : 0;
        long long total;
        const long long p_in = asked_pages + scan(need, total, sums) + need;
        asked_pages += total;
        const long long s_in = asked_slots + scan(more, total, sums) + more;
        asked_slots += total;
        const bool served = r.fits && (need == 0 || p_in <= avail) && s_in <= a.max_slots;
        if (r.grows && !served) flag |= kFlagRefused;
        const int take = served ? need : 0;
        const long long num = served ? more : 0;
        const long long t_ex = took + scan(take, total, sums);
        took += total;
        const long long n_ex = placed + scan(num, total, sums);
        placed += total;
        if (b < a.batch) {
            a.new_len[b] = (int)(r.grows && !served ? r.old_len : r.new_len);
            a.slot_start[b] = (int)n_ex;
        }
        // pages from the stack's top into the rows' next entries
        s_have[tid] = r.have;
        s_num[tid] = take;
        s_at[tid] = (int)(avail - 1 - t_ex);
        __syncthreads();
        const int nreq = min(kAssignThreads, a.batch - c0);
        for (int i = warp; i < nreq; i += kAssignThreads / 32)
            for (int j = lane; j < s_num[i]; j += 32)
                a.table[(size_t)(c0 + i) * a.max_pages + s_have[i] + j] =
                    a.free_pages[s_at[i] - j];
        __syncthreads();
        s_first[tid] = (int)r.old_len;
        s_num[tid] = (int)num;
        s_at[tid] = (int)n_ex;
        __syncthreads();
        for (int i = warp; i < nreq; i += kAssignThreads / 32)
            for (int j = lane; j < s_num[i]; j += 32) {
                const int pos = s_first[i] + j;
                const int page = a.table[(size_t)(c0 + i) * a.max_pages + pos / kPage];
                const bool ok = page >= 0 && page < a.pages;
                if (!ok) flag |= kFlagInvalid;
                a.slots[s_at[i] + j] = ok ? page * kPage + pos % kPage : -1;
            }
        __syncthreads();
    }
    for (long long i = placed + tid; i < a.max_slots; i += kAssignThreads) a.slots[i] = -1;
    if (tid == 0) {
        a.slot_start[a.batch] = (int)placed;
        *a.new_free_count = (int)(avail - took);
    }
    if (flag) atomicOr(a.error_flag, flag);
}

// ---- commit -------------------------------------------------------------------
constexpr int kAppendThreads = 128;

__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    uint32_t r;
    asm("{\n .reg .b16 t;\n cvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\n cvt.u32.u16 %0, t;\n}"
        : "=r"(r)
        : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void unpack_e4m3(uint32_t a, float &lo, float &hi) {
    uint32_t h;
    asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}\n"
        : "=r"(h)
        : "r"(a));
    asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, u;\n}\n"
        : "=f"(lo), "=f"(hi)
        : "r"(h));
}

// The least 2^e, e in [-40, 120], with amax <= 448 * 2^e; amax: the bits of a
// non-negative finite bf16.  448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_of(uint32_t amax) {
    int e = (int)(amax >> 7) - 127 - 8 + ((amax & 0x7f) > 0x60 ? 1 : 0);
    e = e < -40 ? -40 : (e > 120 ? 120 : e);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

struct AppendArgs {
    uint8_t *codes[2];
    float *scales[2];
    const uint16_t *fresh[2];
    const int32_t *slots, *slot_start;
    int32_t *error_flag;
    int batch, W, pages, kv_heads, max_slots, pieces;
};

// One CTA: one page piece of one sequence, one kv head, one slab (depth,
// layer), keys or values.  A thread holds 8 elements of every 128 / (D / 8)-th
// of the page's tokens.
template <int D>
__global__ void __launch_bounds__(kAppendThreads) append_paged_kernel(const AppendArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int kLanes = D / 8, kStep = kAppendThreads / kLanes, kRowsEach = kPage / kStep;
    unsigned x = blockIdx.x;
    const int h = x % a.kv_heads;
    x /= a.kv_heads;
    const int which = x & 1;
    x >>= 1;
    const int piece = x % a.pieces;
    x /= a.pieces;
    const int b = x % a.batch;
    const size_t slab = x / a.batch;

    const int s0 = a.slot_start[b];
    const long long n = (long long)a.slot_start[b + 1] - s0;
    if (n < 0 || n > a.W || s0 < 0 || s0 + n > a.max_slots) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    if (n == 0) return;
    const int slot0 = a.slots[s0];
    if (slot0 < 0) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    const int o = slot0 % kPage;
    const int t0 = piece * kPage - o;  // the token at the page's first place (negative: an older one)
    if (t0 >= n) return;
    const int slot = piece ? a.slots[s0 + t0] : slot0;
    const int page = slot / kPage;
    if (slot < 0 || page >= a.pages || (piece && slot % kPage)) {
        if (threadIdx.x == 0) atomicOr(a.error_flag, kFlagInvalid);
        return;
    }
    const int first = piece ? 0 : o;                       // places [first, last) are new
    const int last = (int)min((long long)kPage, n - t0);
    const int lane = threadIdx.x % kLanes, row0 = threadIdx.x / kLanes;
    const uint16_t *src = a.fresh[which] + ((slab * a.batch + b) * a.W * a.kv_heads + h) * D + lane * 8;
    uint4 x4[kRowsEach];
    uint32_t amax = 0;
#pragma unroll
    for (int u = 0; u < kRowsEach; ++u) {
        const int i = row0 + u * kStep;
        x4[u] = make_uint4(0, 0, 0, 0);
        if (i >= first && i < last)
            x4[u] = __ldcs(reinterpret_cast<const uint4 *>(src + (size_t)(t0 + i) * a.kv_heads * D));
    }
#pragma unroll
    for (int u = 0; u < kRowsEach; ++u) {
        const uint32_t w[4] = {x4[u].x, x4[u].y, x4[u].z, x4[u].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
            if (lo < 0x7f80u) amax = max(amax, lo);
            if (hi < 0x7f80u) amax = max(amax, hi);
        }
    }
    __shared__ uint32_t s_max[kAppendThreads / 32];
    amax = __reduce_max_sync(kFull, amax);
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAppendThreads / 32; ++w) amax = max(amax, s_max[w]);

    const size_t tile = (slab * a.pages + page) * a.kv_heads + h;
    float scale = scale_of(amax), held = 0.f;
    if (first > 0) {
        held = a.scales[which][tile];
        scale = fmaxf(scale, held);
    }
    uint8_t *dst = a.codes[which] + tile * (kPage * D) + lane * 8;
    const bool again = first > 0 && scale != held;
    const float ratio = held / scale;
#pragma unroll
    for (int u = 0; u < kRowsEach; ++u) {
        const int i = row0 + u * kStep;
        uint2 *at = reinterpret_cast<uint2 *>(dst + i * D);
        if (i >= first && i < last) {
            const uint32_t w[4] = {x4[u].x, x4[u].y, x4[u].z, x4[u].w};
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[j] = pack_e4m3(__uint_as_float(w[j] << 16) / scale,
                                 __uint_as_float(w[j] & 0xffff0000u) / scale);
            *at = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        } else if (again && i < first) {
            const uint2 was = *at;
            const uint32_t w[4] = {was.x & 0xffffu, was.x >> 16, was.y & 0xffffu, was.y >> 16};
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float lo, hi;
                unpack_e4m3(w[j], lo, hi);
                c[j] = pack_e4m3(lo * ratio, hi * ratio);
            }
            *at = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
        }
    }
    // every thread has read the page's present scale before it changes
    __syncthreads();
    if (threadIdx.x == 0) a.scales[which][tile] = scale;
}

}  // namespace

cudaError_t page_assign_launch(const PageAssignArgs &a, cudaStream_t stream) {
    return launch_pdl(page_assign_kernel, dim3(1), dim3(kAssignThreads), stream, a);
}

cudaError_t append_paged_launch(const das_kv_cache_paged &c, const void *k_new, const void *v_new,
                                int batch, int W, const int32_t *slots, int max_slots,
                                const int32_t *slot_start, int32_t *error_flag,
                                cudaStream_t stream) {
    AppendArgs a = {};
    a.codes[0] = static_cast<uint8_t *>(c.k);
    a.codes[1] = static_cast<uint8_t *>(c.v);
    a.scales[0] = c.k_scale;
    a.scales[1] = c.v_scale;
    a.fresh[0] = static_cast<const uint16_t *>(k_new);
    a.fresh[1] = static_cast<const uint16_t *>(v_new);
    a.slots = slots;
    a.slot_start = slot_start;
    a.error_flag = error_flag;
    a.batch = batch;
    a.W = W;
    a.pages = c.pages;
    a.kv_heads = c.kv_heads;
    a.max_slots = max_slots;
    a.pieces = (W + 2 * kPage - 2) / kPage;
    const long long ctas =
        (long long)c.depths * c.layers * batch * a.pieces * 2 * c.kv_heads;
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
    if (ctas == 0) return cudaSuccess;
    return c.head_dim == 128 ? launch_pdl(append_paged_kernel<128>, dim3((unsigned)ctas),
                                          dim3(kAppendThreads), stream, a)
                             : launch_pdl(append_paged_kernel<64>, dim3((unsigned)ctas),
                                          dim3(kAppendThreads), stream, a);
}

}  // namespace das
