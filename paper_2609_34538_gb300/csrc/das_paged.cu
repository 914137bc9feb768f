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
                       size_t smem, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

// ---- page assignment ----------------------------------------------------------
constexpr int kAssignThreads = 1024, kAssignFew = 256;
constexpr int kFillAlone = 4096;  // slots that one CTA writes along the way
constexpr int kFillFew = 1024;    // and that kAssignFew threads do

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

// Exclusive sums of two values over the CTA's NT threads, and their totals.
struct Pair {
    long long x, y;
};
template <int NT>
__device__ __forceinline__ Pair scan(Pair v, Pair &total, Pair (*sums)[NT / 32], int &turn) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Pair s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long x = __shfl_up_sync(kFull, s.x, d), y = __shfl_up_sync(kFull, s.y, d);
        if (lane >= d) {
            s.x += x;
            s.y += y;
        }
    }
    turn ^= 1;  // two sets in turn, so that one barrier does
    if (lane == 31) sums[turn][warp] = s;
    __syncthreads();
    // the warps' sums: by each thread for itself if they are few, else by a scan again
    Pair before = {0, 0};
    total = {0, 0};
    if constexpr (NT <= 256) {
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            const Pair p = sums[turn][w];
            if (w < warp) {
                before.x += p.x;
                before.y += p.y;
            }
            total.x += p.x;
            total.y += p.y;
        }
    } else {
        Pair all = lane < NT / 32 ? sums[turn][lane] : Pair{0, 0};
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long x = __shfl_up_sync(kFull, all.x, d), y = __shfl_up_sync(kFull, all.y, d);
            if (lane >= d) {
                all.x += x;
                all.y += y;
            }
        }
        total = {__shfl_sync(kFull, all.x, 31), __shfl_sync(kFull, all.y, 31)};
        before = {__shfl_sync(kFull, all.x, max(warp - 1, 0)), __shfl_sync(kFull, all.y, max(warp - 1, 0))};
        if (warp == 0) before = {0, 0};
    }
    return {before.x + s.x - v.x, before.y + s.y - v.y};
}

// One CTA, a thread to a request.  FILL: it writes the table entries and the slots
// too; otherwise slot_fill_kernel does, from new_len and slot_start.  Bound by
// latency: 16 requests that grow by up to 17 tokens take 2.5 us (3.0 a call in a
// loop), with the lengths, the stack's pages and the stores behind one another and
// a barrier for each sum.
template <int NT, bool FILL>
__global__ void __launch_bounds__(NT) page_assign_kernel(const PageAssignArgs a) {
    __shared__ Pair sums[2][NT / 32];
    __shared__ int s_first[NT], s_have[NT], s_num[NT], s_at[NT], s_top[NT];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int listed = *a.free_count;
    Ask r = ask_of(a, tid);
    const int count = listed < 0 ? 0 : (listed > a.pages ? a.pages : listed);
    int flag = listed != count ? kFlagInvalid : 0, turn = 0;
    Pair total;

    // pages given back, in request order
    long long gave = 0;
    for (int c0 = 0; c0 < a.batch; c0 += NT) {
        if (c0 > 0) r = ask_of(a, c0 + tid);
        if (r.bad) flag |= kFlagInvalid;
        const int give = r.grows ? 0 : r.have - r.want;
        const Pair ex = scan<NT>({give, 0}, total, sums, turn);
        if (total.x == 0) continue;  // the same in every thread
        s_first[tid] = r.want;
        s_num[tid] = give;
        s_at[tid] = (int)min(count + gave + ex.x, (long long)a.pages);
        __syncthreads();
        for (int i = warp; i < min(NT, a.batch - c0); i += NT / 32)
            for (int j = lane; j < s_num[i]; j += 32) {
                const long long at = (long long)s_at[i] + j;
                if (at < a.pages)
                    a.free_pages[at] = a.table[(size_t)(c0 + i) * a.max_pages + s_first[i] + j];
                else
                    flag |= kFlagInvalid;  // more pages than the pool has
            }
        gave += total.x;
        __syncthreads();
    }
    const long long avail = min(count + gave, (long long)a.pages);

    Pair asked = {0, 0}, took = {0, 0};  // pages, slots
    for (int c0 = 0; c0 < a.batch; c0 += NT) {
        const int b = c0 + tid;
        if (a.batch > NT) r = ask_of(a, b);
        const int need = r.fits ? r.want - r.have : 0;
        const long long more = r.fits ? r.new_len - r.old_len : 0;
        Pair ex = scan<NT>({need, more}, total, sums, turn);
        const bool served = r.fits && (need == 0 || asked.x + ex.x + need <= avail) &&
                            asked.y + ex.y + more <= a.max_slots;
        const bool refused = r.grows && !served;
        if (refused) flag |= kFlagRefused;
        asked.x += total.x;
        asked.y += total.y;
        const int take = served ? need : 0;
        const long long num = served ? more : 0;
        if (__syncthreads_or(refused)) ex = scan<NT>({take, num}, total, sums, turn);
        const long long t_ex = took.x + ex.x, n_ex = took.y + ex.y;
        took.x += total.x;
        took.y += total.y;
        if (b < a.batch) {
            a.new_len[b] = (int)(refused ? r.old_len : r.new_len);
            a.slot_start[b] = (int)n_ex;
        }
        if (!FILL) continue;
        // slots, and pages from the stack's top into the rows' next entries
        s_first[tid] = (int)r.old_len;
        s_have[tid] = r.have;
        s_num[tid] = (int)num;
        s_at[tid] = (int)n_ex;
        s_top[tid] = (int)(avail - 1 - t_ex);
        __syncthreads();
        for (int i = warp; i < min(NT, a.batch - c0); i += NT / 32)
            for (int j = lane; j < s_num[i]; j += 32) {
                const int pos = s_first[i] + j, at = pos / kPage, fresh = at - s_have[i];
                int32_t *const entry = a.table + (size_t)(c0 + i) * a.max_pages + at;
                const int page = fresh < 0 ? *entry : a.free_pages[s_top[i] - fresh];
                if (fresh >= 0 && pos % kPage == 0) *entry = page;
                const bool ok = page >= 0 && page < a.pages;
                if (!ok) flag |= kFlagInvalid;
                a.slots[s_at[i] + j] = ok ? page * kPage + pos % kPage : -1;
            }
        if (a.batch > NT) __syncthreads();
    }
    if (FILL)
        for (long long i = took.y + tid; i < a.max_slots; i += NT) a.slots[i] = -1;
    if (tid == 0) {
        a.slot_start[a.batch] = (int)took.y;
        *a.new_free_count = (int)(avail - took.x);
    }
    if (flag) atomicOr(a.error_flag, flag);
}

// Table entries and slots of the requests that page_assign_kernel served:
// CTA x writes slots [x per_cta, (x + 1) per_cta), and the table entry
// of every new page whose first token is among them.  Request b grew by n =
// slot_start[b + 1] - slot_start[b] to new_len[b] and took the pages past
// those of new_len[b] - n; the pages taken before its own, and by all, are
// summed up again by every CTA.  Four slots a thread share their search and mostly
// their page.  Bound by latency: 256 requests and 1.2 million slots take 9.1 us with
// the kernel before (9.2 to 9.5 a call in a loop), of which the slots' 4.9 MB would
// take 0.7.
constexpr int kFillThreads = 256, kFillBatch = 256;

__global__ void __launch_bounds__(kFillThreads) slot_fill_kernel(const PageAssignArgs a, int per_cta) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ long long sums[3 * kFillThreads / 32];
    __shared__ int s_start[kFillBatch + 1], s_old[kFillBatch], s_top[kFillBatch];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int i0 = blockIdx.x * per_cta, i1 = min(i0 + per_cta, a.max_slots);  // (below 2^30 + 2048)
    const int end = a.slot_start[a.batch], left = *a.new_free_count;
    const bool wide = (reinterpret_cast<uintptr_t>(a.slots) & 15) == 0;
    int flag = 0;
    auto pages = [](int n) { return (n + kPage - 1) / kPage; };
    auto taken = [&](int b, int &old) {
        const int n = a.slot_start[b + 1] - a.slot_start[b], len = a.new_len[b];
        old = len - n;
        return n > 0 ? pages(len) - pages(old) : 0;
    };
    if (i0 < end) {
        // b0: the first request with a slot past i0, the number of those that end before
        long long before = 0, all = 0;
        int b0 = 0, old;
        for (int b = tid; b < a.batch; b += kFillThreads) {
            const int n = taken(b, old);
            const bool done = a.slot_start[b + 1] <= i0;
            all += n;
            if (done) {
                before += n;
                ++b0;
            }
        }
        b0 = __reduce_add_sync(kFull, b0);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            before += __shfl_xor_sync(kFull, before, d);
            all += __shfl_xor_sync(kFull, all, d);
        }
        if (lane == 0) {
            sums[warp] = before;
            sums[warp + 8] = all;
            sums[warp + 16] = b0;
        }
        __syncthreads();
        before = all = 0;
        b0 = 0;
#pragma unroll
        for (int w = 0; w < kFillThreads / 32; ++w) {
            before += sums[w];
            all += sums[w + 8];
            b0 += (int)sums[w + 16];
        }
        __syncthreads();
        // the stack's place of the next page taken
        long long top = (long long)left + all - 1 - before;
        for (; b0 < a.batch; b0 += kFillBatch) {
            const int nb = min(kFillBatch, a.batch - b0);
            const int start = a.slot_start[b0], stop = a.slot_start[b0 + nb];
            if (start >= i1) break;
            // exclusive sum of the pages taken, a thread to a request
            const int n = tid < nb ? taken(b0 + tid, old) : 0;
            long long x = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long y = __shfl_up_sync(kFull, x, d);
                if (lane >= d) x += y;
            }
            if (lane == 31) sums[warp] = x;
            __syncthreads();
            long long sum = 0, batch_all = 0;
#pragma unroll
            for (int w = 0; w < kFillThreads / 32; ++w) {
                if (w < warp) sum += sums[w];
                batch_all += sums[w];
            }
            if (tid < nb) {
                s_start[tid] = a.slot_start[b0 + tid];
                s_old[tid] = old;
                s_top[tid] = (int)(top - (sum + x - n));
            }
            if (tid == 0) s_start[nb] = stop;
            __syncthreads();
            const int lo = max(i0, start), hi = min(i1, stop);
            // four slots a thread: one search, and mostly one page
            for (int i4 = (lo & ~3) + 4 * tid; i4 < hi; i4 += 4 * kFillThreads) {
                const int i_first = max(i4, lo), i_end = min(i4 + 4, hi);
                int r = 0;
                for (int h = nb - 1; r < h;) {  // the last request that starts by i_first
                    const int mid = (r + h + 1) / 2;
                    if (s_start[mid] <= i_first) r = mid;
                    else h = mid - 1;
                }
                int out[4] = {-1, -1, -1, -1}, page = -1, page_r = -1, page_at = -1;
                for (int i = i_first; i < i_end; ++i) {
                    while (s_start[r + 1] <= i) ++r;
                    const int pos = s_old[r] + i - s_start[r], at = pos / kPage;
                    if (r != page_r || at != page_at) {
                        const int have = pages(s_old[r]);
                        int32_t *entry = a.table + (size_t)(b0 + r) * a.max_pages + at;
                        page = at < have ? *entry : a.free_pages[s_top[r] - (at - have)];
                        if (at >= have && pos % kPage == 0) *entry = page;
                        if (page < 0 || page >= a.pages) {
                            flag |= kFlagInvalid;
                            page = -1;
                        }
                        page_r = r;
                        page_at = at;
                    }
                    out[i - i4] = page < 0 ? -1 : page * kPage + pos % kPage;
                }
                if (i_first == i4 && i_end == i4 + 4 && wide) {
                    *reinterpret_cast<int4 *>(a.slots + i4) = make_int4(out[0], out[1], out[2], out[3]);
                } else {
                    for (int i = i_first; i < i_end; ++i) a.slots[i] = out[i - i4];
                }
            }
            __syncthreads();  // the requests' numbers are written again
            top -= batch_all;
        }
    }
    for (int i = max(i0, end) + tid; i < i1; i += kFillThreads) a.slots[i] = -1;
    if (flag) atomicOr(a.error_flag, flag);
}

// ---- commit -------------------------------------------------------------------
constexpr int kAppendThreads = 128, kAppendWarps = kAppendThreads / 32;

__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    uint32_t r;
    asm("{\n .reg .b16 t;\n cvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\n cvt.u32.u16 %0, t;\n}"
        : "=r"(r)
        : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n .reg .b16 l, u;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n"
        " cvt.rn.satfinite.e4m3x2.f32 u, %4, %3;\n mov.b32 %0, {l, u};\n}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
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
    int batch, W, pages, kv_heads, max_slots, pieces, rows;
    unsigned jobs;  // CTAs to the same kAppendWarps heads
};

// The largest finite magnitude among eight elements, as bf16 bits.
__device__ __forceinline__ uint32_t finite_amax(uint4 x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t lo = w[j] & 0x7fffu, hi = (w[j] >> 16) & 0x7fffu;
        if (lo < 0x7f80u) amax = max(amax, lo);
        if (hi < 0x7f80u) amax = max(amax, hi);
    }
    return amax;
}

// Eight elements as codes under a scale.  A product with the reciprocal of a power
// of two (a normal number itself) is the exact quotient; other scales, which only
// pages that a caller has filled can have, take a division.
struct Divisor {
    __device__ __forceinline__ explicit Divisor(float scale) : scale(scale) {
        const uint32_t bits = __float_as_uint(scale);
        exact = (bits & 0x807fffffu) == 0 && bits >= 0x00800000u && bits < 0x7f000000u;
        inverse = __uint_as_float(0x7f000000u - bits);
    }
    template <typename F>
    __device__ __forceinline__ uint2 each(uint4 x, F f) const {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = f(__uint_as_float(w[j] << 16));
            v[2 * j + 1] = f(__uint_as_float(w[j] & 0xffff0000u));
        }
        return make_uint2(pack4_e4m3(v[0], v[1], v[2], v[3]), pack4_e4m3(v[4], v[5], v[6], v[7]));
    }
    __device__ __forceinline__ uint2 codes(uint4 x) const {
        return each(x, [&](float v) { return v * inverse; });
    }
    __device__ __forceinline__ uint2 divided(uint4 x) const {
        return each(x, [&](float v) { return v / scale; });
    }
    float scale, inverse;
    bool exact;
};

// The codes of rows i0, i0 + step, ... < end under a larger scale: times ratio.
__device__ __forceinline__ void rescale(uint8_t *dst, int D, int i0, int step, int end, float ratio) {
    for (int i = i0; i < end; i += step) {
        uint2 *at = reinterpret_cast<uint2 *>(dst + i * D);
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

// A warp to a (sequence, page piece, slab, keys or values, kv head); up to kPage tokens
// are one piece, on whichever two pages they lie.  The tokens go into shared memory
// while their places are looked up (of several pieces: the sequence's first place
// before), and are read there twice, for the scale and for the codes: no head
// waits for another, and short loops leave registers and instruction cache for
// many warps.  Bound by memory: 1001 tokens of 4 sequences at 8 depths and 4
// layers 92.3 us, 6.86 TB/s read and written; 83 tokens at 32 depths 17.9 us, 4.2 TB/s,
// where the chain of a warp's look-ups counts.  A CTA to a piece of all heads with
// the tokens in registers, which needs no shared memory, took 100 and 23 us: three
// times the instructions, and warps that wait for each other's maxima.
template <int D>
__global__ void __launch_bounds__(kAppendThreads) append_paged_kernel(const AppendArgs a) {
    extern __shared__ uint4 s_rows[];  // [warp][rows][D / 8]
    constexpr int kLanes = D / 8, kStep = 32 / kLanes;
    const int lane = threadIdx.x & 31, row = lane / kLanes, warp = threadIdx.x >> 5;
    unsigned x = blockIdx.x;
    const int job = (int)(x / a.jobs) * kAppendWarps + warp;
    const int which = job >= a.kv_heads, h = job - (which ? a.kv_heads : 0);
    x %= a.jobs;
    const int piece = x % a.pieces;
    x /= a.pieces;
    const int b = x % a.batch;
    const size_t slab = x / a.batch;
    uint4 *const mine = s_rows + warp * a.rows * kLanes + lane % kLanes;  // a lane reads what it copied
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
    if (a.pieces > 1) {
        if (slot < 0) {
            if (lane == 0) atomicOr(a.error_flag, kFlagInvalid);
            return;
        }
        const int t = piece * kPage - slot % kPage;  // the token at the page's first place
        if (t >= end) return;
        begin = max(t, 0);
        end = min(t + kPage, end);
        if (piece) slot = a.slots[s0 + begin];
    }
    {
        const size_t stride = (size_t)a.kv_heads * D;
        const uint16_t *src = a.fresh[which] + ((slab * a.batch + b) * a.W + begin + row) * stride +
                              h * D + lane % kLanes * 8;
        for (int t = begin + row; t < end; t += kStep, src += kStep * stride)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                             (uint32_t)__cvta_generic_to_shared(mine + (t - begin) * kLanes)),
                         "l"(src)
                         : "memory");
    }
    for (int t0 = begin; t0 < end;) {  // the tokens up to the page's end, then the others
        const int first = slot < 0 ? 0 : slot % kPage, page = slot / kPage;
        if (slot < 0 || page >= a.pages || ((t0 > 0 || piece) && first)) {
            if (lane == 0) atomicOr(a.error_flag, kFlagInvalid);
            break;
        }
        const int t1 = min(end, t0 + kPage - first);
        if (t1 < end) slot = a.slots[s0 + t1];
        const size_t tile = (slab * a.pages + page) * a.kv_heads + h;
        float *const at_scale = a.scales[which] + tile;
        const float held = first > 0 ? *at_scale : 0.f;
        asm volatile("cp.async.wait_all;" ::: "memory");
        // this lane's rows of the page: [i, i_end) in steps of kStep
        const int r0 = t0 - begin, i0 = r0 + (row + kStep - r0 % kStep) % kStep, i_end = t1 - begin;
        uint32_t amax = 0;
#pragma unroll 4
        for (int i = i0; i < i_end; i += kStep) {
            const uint4 x = mine[i * kLanes];
            amax = max_bf16x2(max_bf16x2(amax, max_bf16x2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu)),
                              max_bf16x2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
        }
        amax = max(amax & 0xffffu, amax >> 16);
        if (amax >= 0x7f80u) {  // an infinity (NaN loses): the largest finite one
            amax = 0;
#pragma unroll 1
            for (int i = i0; i < i_end; i += kStep) amax = max(amax, finite_amax(mine[i * kLanes]));
        }
        const float scale = fmaxf(scale_of(__reduce_max_sync(kFull, amax)), held);
        uint8_t *const codes = a.codes[which] + tile * (kPage * D) + lane % kLanes * 8;
        uint8_t *dst = codes + (first + i0 - r0) * D;
        const Divisor by(scale);
        if (by.exact) {
#pragma unroll 4
            for (int i = i0; i < i_end; i += kStep, dst += kStep * D)
                *reinterpret_cast<uint2 *>(dst) = by.codes(mine[i * kLanes]);
        } else {
#pragma unroll 1
            for (int i = i0; i < i_end; i += kStep, dst += kStep * D)
                *reinterpret_cast<uint2 *>(dst) = by.divided(mine[i * kLanes]);
        }
        if (first > 0 && scale != held) rescale(codes, D, row, kStep, first, held / scale);
        if (lane == 0) *at_scale = scale;
        t0 = t1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace

cudaError_t page_assign_launch(const PageAssignArgs &a, cudaStream_t stream) {
    // One CTA writes a few thousand slots along the way, but took 182 us for 256
    // requests and 1.2 million of them; a second kernel brings that to 9.1 us, with
    // little to write to 7 (one CTA: 6.3 us for 256 requests and 4352 slots, 8.1 for
    // 400 and 6800, 10.3 for 600 and 7800).
    // The fewer warps, the shorter the barriers and sums: 16 requests and 272 slots take
    // 2.5 us with 256 threads, 3.6 with 1024.  But the slots of a request are a
    // warp's: 200 requests and 3400 slots take 8.8 and 5.9 us, and 1000 requests
    // whose slots the second kernel writes 18.9 and 16.7.
    const bool fill = a.max_slots <= kFillAlone;
    const bool few = a.batch <= kAssignFew && (!fill || a.max_slots <= kFillFew);
    const auto kernel = few ? (fill ? page_assign_kernel<kAssignFew, true> : page_assign_kernel<kAssignFew, false>)
                            : (fill ? page_assign_kernel<kAssignThreads, true>
                                    : page_assign_kernel<kAssignThreads, false>);
    const cudaError_t e = launch_pdl(kernel, dim3(1), dim3(few ? kAssignFew : kAssignThreads), stream, 0, a);
    if (fill || e != cudaSuccess) return e;
    // More CTAs while they are few to an SM: 40,000 slots 7.9 us by 1024, 9.2 by 2048;
    // 1.2 million 10.2 and 9.1.
    const int per_cta = a.max_slots <= 500000 ? 1024 : 2048;
    return launch_pdl(slot_fill_kernel, dim3((unsigned)((a.max_slots + per_cta - 1) / per_cta)),
                      dim3(kFillThreads), stream, 0, a, per_cta);
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
    a.pieces = W <= kPage ? 1 : (W + 2 * kPage - 2) / kPage;
    a.rows = std::min(W, kPage);
    const long long jobs = (long long)c.depths * c.layers * batch * a.pieces;
    const long long ctas = jobs * ((2LL * c.kv_heads + kAppendWarps - 1) / kAppendWarps);
    if (ctas > 0x7fffffffLL) return cudaErrorInvalidValue;
    a.jobs = (unsigned)jobs;
    if (ctas == 0) return cudaSuccess;
    const auto kernel = c.head_dim == 128 ? append_paged_kernel<128> : append_paged_kernel<64>;
    const size_t smem = (size_t)kAppendWarps * a.rows * c.head_dim * 2;
    if (smem > 49152) {
        const cudaError_t e =
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3((unsigned)ctas), dim3(kAppendThreads), stream, smem, a);
}

}  // namespace das
