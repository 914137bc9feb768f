// das_sample.cu -- sampling with temperature, top-k, top-p and min-p from
// given random numbers, and the acceptance of proposals against the draws.
//
// A filter keeps a prefix of the tokens ordered by logit (largest first,
// equal ones by index), so each is one threshold: a key (the logit's bits made
// monotone) and how many of the tokens equal to it, lowest index first, stay.
// The threshold is where a sum over keys >= t first reaches a target: a sum of
// ones for top-k, of the whole-number weights for top-p.
//
// Every kernel here is launched as a programmatic dependent of the previous
// kernel in the stream: it reads nothing before griddepcontrol.wait, and
// every CTA executes that wait.
#include <algorithm>

#include "das_internal.h"

namespace das {
namespace {

using u64 = unsigned long long;
constexpr uint32_t kFull = 0xffffffffu;
constexpr int kThreads = 1024;
constexpr int kScanWarps = 4;

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

// One row by one CTA, reading it once for every step.
template <bool BF16>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
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
    for (int i = tid; i < V; i += kThreads) mine = max(mine, key(i));
    const uint32_t top =
        (uint32_t)block_reduce<u64>(mine, sums, [](u64 x, u64 y) { return x > y ? x : y; });
    if (top <= kKeyNone) {
        if (tid == 0) {
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
            for (int i = tid; i < V; i += kThreads) {
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
        for (int i = tid; i < V; i += kThreads) n += key(i) == t;
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
        for (int i = tid; i < V; i += kThreads) {
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
        for (int i0 = 0; i0 < V; i0 += kThreads) {
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
    for (int i = tid; i < V; i += kThreads) total += kept(i);
    total = block_reduce<u64>(total, sums, add);
    float u = a.uniforms[row];
    if (!(u >= 0.f)) u = 0.f;
    u64 r = (u64)((double)u * (double)total);
    if (r > total - 1) r = total - 1;
    // the token at which the running sum in index order passes r
    __shared__ int s_token;
    u64 seen = 0;
    for (int i0 = 0; i0 < V; i0 += kThreads) {
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

}  // namespace

cudaError_t sample_launch(const SampleArgs &a, cudaStream_t stream) {
    const long long rows = (long long)a.B * a.W;
    if (rows == 0) return cudaSuccess;
    return a.bf16 ? launch_pdl(sample_kernel<true>, dim3((unsigned)rows), dim3(kThreads), stream, a)
                  : launch_pdl(sample_kernel<false>, dim3((unsigned)rows), dim3(kThreads), stream, a);
}

cudaError_t sample_accept_launch(const SampleArgs &a, const int32_t *draft, int32_t *accepted,
                                 int32_t *next_token, int32_t *committed, cudaStream_t stream) {
    if (a.B == 0) return cudaSuccess;
    return launch_pdl(sample_accept_kernel, dim3((unsigned)((a.B + kScanWarps - 1) / kScanWarps)),
                      dim3(kScanWarps * 32), stream, static_cast<const int32_t *>(a.tokens), draft,
                      a.B, a.W, accepted, next_token, committed);
}

}  // namespace das
