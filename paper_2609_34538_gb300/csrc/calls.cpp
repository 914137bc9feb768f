// calls.cpp -- the Python module _calls: the binding of the paged-cache and
// sampling calls.  It checks the tensors, allocates what the caller left out
// and calls the C ABI; the package's functions of the same names hold the
// signatures and turn a status into an exception.
//
// Most of these calls take 3 to 20 us on the GPU, no more than the same checks and
// allocations took in Python through ctypes (attention 21 us a call with two
// launches, sampled acceptance 25 us with its five results, of which the library
// itself 8 and 6), so a loop of them ran at the pace of the host.  With this module a
// call takes the host 2 to 8 us (commit 2.3, attention 5.4, page assignment 5.5,
// sampled acceptance 7.8, results allocated).
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <climits>
#include <initializer_list>

#include "das.h"

namespace {

using at::ScalarType;
using Shape = std::initializer_list<int64_t>;

// A Python exception is set: unwinds to the module function.
[[noreturn]] void fail() { throw python_error(); }

template <typename... Args>
[[noreturn]] void refuse(PyObject *type, const char *format, Args... args) {
    PyErr_Format(type, format, args...);
    fail();
}

const char *type_name(ScalarType t) {
    switch (t) {
        case at::kInt: return "torch.int32";
        case at::kFloat: return "torch.float32";
        case at::kBFloat16: return "torch.bfloat16";
        default: return "torch.uint8";
    }
}

PyObject *tuple_of(at::IntArrayRef sizes) {
    THPObjectPtr t(PyTuple_New((Py_ssize_t)sizes.size()));
    if (!t) fail();
    for (size_t i = 0; i < sizes.size(); ++i) {
        PyObject *v = PyLong_FromLongLong(sizes[i]);
        if (!v) fail();
        PyTuple_SET_ITEM(t.get(), i, v);
    }
    return t.release();
}

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a torch.Tensor", name);
    return THPVariable_Unpack(o);
}

void wrong_type(PyObject *o, const char *name, const char *wanted) {
    THPObjectPtr got(PyObject_GetAttrString(o, "dtype"));
    if (!got) fail();
    refuse(PyExc_TypeError, "%s must be %s, got %S", name, wanted, got.get());
}

// The GPU of a call, which all its tensors are on: the first one's that is looked at.
struct Gpu {
    void check(const at::Tensor &t, const char *name) {
        if (!t.is_cuda()) refuse(PyExc_ValueError, "%s must be on a CUDA device", name);
        const int i = t.device().index();
        if (index < 0) index = i;
        if (i != index) refuse(PyExc_ValueError, "%s is on cuda:%d, other arguments on cuda:%d", name, i, index);
    }
    int index = -1;
};

const at::Tensor &need(Gpu &gpu, PyObject *o, ScalarType type, const char *name, int dims) {
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != type) wrong_type(o, name, type_name(type));
    gpu.check(t, name);
    if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", name);
    if (t.dim() != dims) {
        THPObjectPtr got(tuple_of(t.sizes()));
        refuse(PyExc_ValueError, "%s must have %d dims, got %R", name, dims, got.get());
    }
    return t;
}

const at::Tensor &need(Gpu &gpu, PyObject *o, ScalarType type, const char *name, Shape shape) {
    const at::Tensor &t = need(gpu, o, type, name, (int)shape.size());
    if (t.sizes() != at::IntArrayRef(shape)) {
        THPObjectPtr want(tuple_of(shape)), got(tuple_of(t.sizes()));
        refuse(PyExc_ValueError, "%s must have shape %R, got %R", name, want.get(), got.get());
    }
    return t;
}

int to_int(int64_t v, const char *name) {
    if (v < INT_MIN || v > INT_MAX) refuse(PyExc_OverflowError, "%s does not fit 32 bits", name);
    return (int)v;
}

int int_of(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) fail();
    return to_int(v, name);
}

// The stream of a call: the current one of its GPU, or the given torch.cuda.Stream, on
// which results are then allocated too (memory in use on another stream is not handed
// out).  The call's GPU is the current one until it returns.
struct Stream {
    Stream(PyObject *o, const Gpu &gpu) {
        if (o == Py_None) {
            device.set_index((c10::DeviceIndex)gpu.index);
            handle = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)gpu.index).stream();
            return;
        }
        long long v[3];
        const char *names[3] = {"stream_id", "device_index", "device_type"};
        for (int i = 0; i < 3; ++i) {
            THPObjectPtr a(PyObject_GetAttrString(o, names[i]));
            if (!a) fail();
            v[i] = PyLong_AsLongLong(a.get());
            if (v[i] == -1 && PyErr_Occurred()) fail();
        }
        if (v[1] != gpu.index)
            refuse(PyExc_ValueError, "the stream is of cuda:%lld, the arguments on cuda:%d", v[1], gpu.index);
        const auto s = c10::cuda::CUDAStream::unpack3(v[0], (c10::DeviceIndex)v[1], (c10::DeviceType)v[2]);
        handle = s.stream();
        guard.reset_stream(s);
    }
    cudaStream_t handle;
    c10::cuda::OptionalCUDAGuard device;
    c10::cuda::OptionalCUDAStreamGuard guard;
};

// A result: the given tensor (checked), or a new one, allocated on the call's stream.
struct Result {
    Result(Gpu &gpu, PyObject *given, ScalarType type, const char *name, Shape shape) : type(type), sizes(shape) {
        if (given == Py_None) return;
        at = need(gpu, given, type, name, shape);
        object = Py_NewRef(given);
    }
    void ready(const Stream &, const at::Tensor &like) {
        if (object) return;
        at = at::empty(sizes, like.options().dtype(type));
        object = THPVariable_Wrap(at);
        if (!object) fail();
    }
    template <typename T = void>
    T *as() const { return static_cast<T *>(at.data_ptr()); }
    ScalarType type;
    c10::SmallVector<int64_t, 4> sizes;
    at::Tensor at;
    THPObjectPtr object;
};

template <typename... R>
PyObject *pack(R &...results) {
    THPObjectPtr t(PyTuple_New(sizeof...(R)));
    if (!t) fail();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(t.get(), i++, results.object.release()), ...);
    return t.release();
}

template <typename F>
das_status without_gil(F f) {
    struct Released {  // taken again on an exception too (a tensor without memory has no address)
        PyThreadState *const state = PyEval_SaveThread();
        ~Released() { PyEval_RestoreThread(state); }
    } released;
    return f();
}

template <typename T>
T *at_of(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }

template <typename Cache>
const Cache *cache_of(PyObject *o) {  // PagedKVCache.address, PagedKVCache4.address
    const void *p = PyLong_AsVoidPtr(o);
    if (!p) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no cache");
        fail();
    }
    return static_cast<const Cache *>(p);
}

void count_args(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) refuse(PyExc_TypeError, "%zd arguments, not %zd", want, n);
}

// Each function returns its results, or the status of a call that failed.
PyObject *page_assign(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 11);
    Gpu gpu;
    const at::Tensor &seq_len = need(gpu, a[0], at::kInt, "seq_len", 1);
    const int64_t B = seq_len.numel();
    const at::Tensor &grow = need(gpu, a[1], at::kInt, "grow", {B});
    const at::Tensor &table = need(gpu, a[2], at::kInt, "block_table", 2);
    if (table.size(0) != B) refuse(PyExc_ValueError, "block_table must be [batch][max_pages]");
    const at::Tensor &pages = need(gpu, a[3], at::kInt, "free_pages", 1);
    const at::Tensor &count = need(gpu, a[4], at::kInt, "free_count", {1});
    const at::Tensor &slots = need(gpu, a[5], at::kInt, "slots", 1);
    const at::Tensor &flag = need(gpu, a[6], at::kInt, "error_flag", {1});
    Result new_len(gpu, a[7], at::kInt, "new_len", {B});
    Result new_count(gpu, a[8], at::kInt, "new_free_count", {1});
    Result start(gpu, a[9], at::kInt, "slot_start", {B + 1});
    const Stream stream(a[10], gpu);
    for (Result *r : {&new_len, &new_count, &start}) r->ready(stream, seq_len);
    const int batch = to_int(B, "batch"), rows = to_int(table.size(1), "max_pages");
    const int n_pages = to_int(pages.numel(), "free_pages"), n_slots = to_int(slots.numel(), "slots");
    const das_status s = without_gil([&] {
        return das_page_assign(at_of<int32_t>(seq_len), at_of<int32_t>(grow), batch, at_of<int32_t>(table), rows,
                               at_of<int32_t>(pages), n_pages, at_of<int32_t>(count), at_of<int32_t>(slots), n_slots,
                               start.as<int32_t>(), new_len.as<int32_t>(), new_count.as<int32_t>(),
                               at_of<int32_t>(flag), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    return pack(new_len, new_count, start);
    END_HANDLE_TH_ERRORS
}

template <typename Cache, auto CALL>
PyObject *kv_append(PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 7);
    const Cache *cache = cache_of<Cache>(a[0]);
    Gpu gpu;
    const at::Tensor &k = need(gpu, a[1], at::kBFloat16, "k_new", 6);
    const at::Tensor &v = need(gpu, a[2], at::kBFloat16, "v_new", 6);
    const int64_t B = k.size(2), W = k.size(3);
    const int64_t want[] = {cache->depths, cache->layers, B, W, cache->kv_heads, cache->head_dim};
    if (k.sizes() != at::IntArrayRef(want) || k.sizes() != v.sizes())
        refuse(PyExc_ValueError, "k_new / v_new must be [depths][layers][batch][W][kv_heads][head_dim]");
    const at::Tensor &slots = need(gpu, a[3], at::kInt, "slots", 1);
    const at::Tensor &start = need(gpu, a[4], at::kInt, "slot_start", {B + 1});
    const at::Tensor &flag = need(gpu, a[5], at::kInt, "error_flag", {1});
    const Stream stream(a[6], gpu);
    const int batch = to_int(B, "batch"), width = to_int(W, "W"), n_slots = to_int(slots.numel(), "slots");
    const das_status s = without_gil([&] {
        return CALL(cache, k.data_ptr(), v.data_ptr(), batch, width, at_of<int32_t>(slots), n_slots,
                    at_of<int32_t>(start), at_of<int32_t>(flag), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyObject *kv_append_paged(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return kv_append<das_kv_cache_paged, das_kv_append_paged>(a, n);
}

PyObject *kv_append_paged4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return kv_append<das_kv_cache_paged4, das_kv_append_paged4>(a, n);
}

template <typename Cache, auto CALL>
PyObject *attention(PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 15);
    const Cache *cache = cache_of<Cache>(a[0]);
    const int layer = int_of(a[1], "layer"), key_depth = int_of(a[2], "key_depth");
    const int value_depth = int_of(a[3], "value_depth");
    Gpu gpu;
    const at::Tensor &table = need(gpu, a[4], at::kInt, "block_table", 2);
    const at::Tensor &q = need(gpu, a[7], at::kBFloat16, "q", 4);
    const int64_t B = q.size(0), T = q.size(1), Hq = q.size(2), D = cache->head_dim, H = cache->kv_heads;
    if (q.size(3) != D || table.size(0) != B)
        refuse(PyExc_ValueError, "q / table shapes do not match the cache");
    const at::Tensor &prefix = need(gpu, a[5], at::kInt, "prefix_len", {B});
    const at::Tensor &block = need(gpu, a[6], at::kInt, "block_len", {B});
    const at::Tensor &kb = need(gpu, a[8], at::kBFloat16, "k_blk", {B, T, H, D});
    const at::Tensor &vb = need(gpu, a[9], at::kBFloat16, "v_blk", {B, T, H, D});
    const at::Tensor &ws = need(gpu, a[10], at::kByte, "workspace", 1);
    const double scale = PyFloat_AsDouble(a[13]);
    if (scale == -1.0 && PyErr_Occurred()) fail();
    Result out(gpu, a[11], at::kBFloat16, "out", {B, T, Hq, D});
    Result lse(gpu, a[12], at::kFloat, "lse", {B, Hq, T});
    const Stream stream(a[14], gpu);
    for (Result *r : {&out, &lse}) r->ready(stream, q);
    const int batch = to_int(B, "batch"), width = to_int(T, "max_block"), heads = to_int(Hq, "num_q_heads");
    const int rows = to_int(table.size(1), "max_pages");
    const das_status s = without_gil([&] {
        return CALL(cache, layer, key_depth, value_depth, at_of<int32_t>(table), rows, at_of<int32_t>(prefix),
                    at_of<int32_t>(block), batch, width, q.data_ptr(), kb.data_ptr(), vb.data_ptr(), heads,
                    (float)scale, out.as<>(), lse.as<float>(), ws.data_ptr(), (size_t)ws.numel(), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    return pack(out, lse);
    END_HANDLE_TH_ERRORS
}

PyObject *mature_v_attention_paged(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return attention<das_kv_cache_paged, das_mature_v_attention_paged>(a, n);
}

PyObject *mature_v_attention_paged4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return attention<das_kv_cache_paged4, das_mature_v_attention_paged4>(a, n);
}

// Rows of heads [batch][max_block][heads][head_dim] at any strides that the call takes.
const at::Tensor &need_rows(Gpu &gpu, PyObject *o, const char *name, das_head_rows &rows) {
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != at::kBFloat16) wrong_type(o, name, type_name(at::kBFloat16));
    gpu.check(t, name);
    if (t.dim() != 4) {
        THPObjectPtr got(tuple_of(t.sizes()));
        refuse(PyExc_ValueError, "%s must have 4 dims, got %R", name, got.get());
    }
    if (t.stride(3) != 1) refuse(PyExc_ValueError, "%s must have contiguous rows of head_dim", name);
    int64_t stride[3];
    for (int i = 0; i < 3; ++i) {  // (the stride of a single one does not matter)
        stride[i] = t.size(i) > 1 ? t.stride(i) : 0;
        if (stride[i] % 4 != 0) refuse(PyExc_ValueError, "strides of %s must be multiples of 4", name);
    }
    rows = {nullptr, stride[0], stride[1], stride[2]};
    return t;
}

PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 14);
    Gpu gpu;
    das_head_rows rows[3] = {};
    const char *names[3] = {"q", "k", "v"}, *outs[3] = {"q_out", "k_out", "v_out"};
    const int parts = a[2] == Py_None ? 2 : 3;
    const at::Tensor *in[3] = {};
    for (int i = 0; i < parts; ++i) in[i] = &need_rows(gpu, a[i], names[i], rows[i]);
    const int64_t B = in[0]->size(0), T = in[0]->size(1), Hq = in[0]->size(2), D = in[0]->size(3), H = in[1]->size(2);
    for (int i = 1; i < parts; ++i)
        if (in[i]->sizes() != at::IntArrayRef({B, T, H, D}))
            refuse(PyExc_ValueError, "%s must be [batch][max_block][kv_heads][head_dim]", names[i]);
    const at::Tensor &freq = need(gpu, a[3], at::kFloat, "inv_freq", 1);
    const at::Tensor *lens[2] = {};
    const char *len_names[2] = {"prefix_len", "block_len"};
    for (int i = 0; i < 2; ++i)
        if (a[4 + i] != Py_None) lens[i] = &need(gpu, a[4 + i], at::kInt, len_names[i], {B});
    const at::Tensor *weight[2] = {};
    const char *weight_names[2] = {"q_weight", "k_weight"};
    ScalarType type = at::kFloat;
    for (int i = 0; i < 2; ++i) {
        if (a[6 + i] == Py_None) continue;
        const ScalarType got = tensor(a[6 + i], weight_names[i]).scalar_type();
        if (got != at::kFloat && got != at::kBFloat16) wrong_type(a[6 + i], weight_names[i], "float32 or bfloat16");
        if (i == 1 && weight[0] && got != type) wrong_type(a[7], "k_weight", "of q_weight's type");
        type = got;
        weight[i] = &need(gpu, a[6 + i], type, weight_names[i], {D});
    }
    double eps = -1.0;
    if (a[8] != Py_None) {
        eps = PyFloat_AsDouble(a[8]);
        if (eps == -1.0 && PyErr_Occurred()) fail();
        if (!(eps >= 0.0)) refuse(PyExc_ValueError, "eps must be at least 0 (None: no norm)");
    }
    const int interleaved = PyObject_IsTrue(a[9]);
    if (interleaved < 0) fail();
    if (parts == 2 && a[12] != Py_None) refuse(PyExc_ValueError, "v_out without v");
    Result q_out(gpu, a[10], at::kBFloat16, outs[0], {B, T, Hq, D});
    Result k_out(gpu, a[11], at::kBFloat16, outs[1], {B, T, H, D});
    Result v_out(gpu, a[12], at::kBFloat16, outs[2], {B, T, H, D});
    const Stream stream(a[13], gpu);
    q_out.ready(stream, *in[0]);
    k_out.ready(stream, *in[0]);
    if (parts == 3) v_out.ready(stream, *in[0]);
    const int batch = to_int(B, "batch"), width = to_int(T, "max_block"), heads = to_int(Hq, "num_q_heads");
    const int kv_heads = to_int(H, "kv_heads"), dim = to_int(D, "head_dim"), turned = to_int(2 * freq.numel(), "inv_freq");
    const das_status s = without_gil([&] {
        for (int i = 0; i < parts; ++i) rows[i].data = in[i]->data_ptr();
        return das_qk_norm_rope(&rows[0], &rows[1], parts == 3 ? &rows[2] : nullptr, batch, width, heads, kv_heads, dim,
                                weight[0] ? weight[0]->data_ptr() : nullptr, weight[1] ? weight[1]->data_ptr() : nullptr,
                                type == at::kFloat ? DAS_WEIGHTS_F32 : DAS_WEIGHTS_BF16, (float)eps,
                                turned ? at_of<float>(freq) : nullptr, turned, interleaved,
                                lens[0] ? at_of<int32_t>(*lens[0]) : nullptr, lens[1] ? at_of<int32_t>(*lens[1]) : nullptr,
                                q_out.as<>(), k_out.as<>(), parts == 3 ? v_out.as<>() : nullptr, stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    if (parts == 2) v_out.object = Py_NewRef(Py_None);
    return pack(q_out, k_out, v_out);
    END_HANDLE_TH_ERRORS
}

// Sampling parameters of one value per sequence: temperature, top_k, top_p, min_p.
struct Filters {
    Filters(Gpu &gpu, PyObject *const *params, int64_t B, bool draft = false) {
        const struct {
            const char *name, *draft_name;
            ScalarType type;
        } kinds[4] = {{"temperature", "draft_temperature", at::kFloat}, {"top_k", "draft_top_k", at::kInt},
                      {"top_p", "draft_top_p", at::kFloat}, {"min_p", "draft_min_p", at::kFloat}};
        for (int i = 0; i < 4; ++i)
            if (params[i] != Py_None)
                at[i] = &need(gpu, params[i], kinds[i].type, draft ? kinds[i].draft_name : kinds[i].name, {B});
    }
    template <typename T>
    const T *of(int i) const { return at[i] ? at_of<T>(*at[i]) : nullptr; }
    das_sampling sampling() const { return {of<float>(0), of<int32_t>(1), of<float>(2), of<float>(3)}; }
    const at::Tensor *at[4] = {};
};

// What the sampling calls share: logits, and uniforms of one value per row.
struct Rows {
    Rows(Gpu &gpu, PyObject *logits_o, PyObject *uniforms_o, const char *name = "logits")
        : logits(tensor(logits_o, name)) {
        const ScalarType type = logits.scalar_type();
        if (type != at::kFloat && type != at::kBFloat16) wrong_type(logits_o, name, "float32 or bfloat16");
        kind = type == at::kFloat ? DAS_LOGITS_F32 : DAS_LOGITS_BF16;
        gpu.check(logits, name);
        if (logits.dim() != 3) {
            THPObjectPtr got(tuple_of(logits.sizes()));
            refuse(PyExc_ValueError, "%s must have 3 dims, got %R", name, got.get());
        }
        B = logits.size(0);
        W = logits.size(1);
        const int64_t V = logits.size(2);
        stride = W > 1 ? logits.stride(1) : B > 1 ? logits.stride(0) : V;  // of a row: a vocabulary may be padded
        if ((V > 1 && logits.stride(2) != 1) || (B > 1 && logits.stride(0) != W * stride))
            refuse(PyExc_ValueError, "%s must have contiguous rows at one stride", name);
        u = &need(gpu, uniforms_o, at::kFloat, "uniforms", {B, W});
        batch = to_int(B, "batch");
        width = to_int(W, "W");
        vocab = to_int(V, "vocab");
    }
    const float *uniforms() const { return at_of<float>(*u); }
    const at::Tensor &logits, *u;
    das_logits_type kind;
    int64_t B, W, stride;
    int batch, width, vocab;
};

PyObject *sample(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 9);
    Gpu gpu;
    const Rows r(gpu, a[0], a[1]);
    const Filters filters(gpu, a + 2, r.B);
    Result tokens(gpu, a[6], at::kInt, "tokens", {r.B, r.W});
    Result logprobs(gpu, a[7], at::kFloat, "logprobs", {r.B, r.W});
    const Stream stream(a[8], gpu);
    for (Result *x : {&tokens, &logprobs}) x->ready(stream, r.logits);
    const das_sampling sampling = filters.sampling();
    const das_status s = without_gil([&] {
        return das_sample(r.logits.data_ptr(), r.kind, r.batch, r.width, r.vocab, r.stride, &sampling, r.uniforms(),
                          tokens.as<int32_t>(), logprobs.as<float>(), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    return pack(tokens, logprobs);
    END_HANDLE_TH_ERRORS
}

PyObject *sample_accept(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 13);
    Gpu gpu;
    const Rows r(gpu, a[0], a[2]);
    const Filters filters(gpu, a + 3, r.B);
    const at::Tensor &draft = need(gpu, a[1], at::kInt, "draft_ids", {r.B, r.W});
    Result accepted(gpu, a[7], at::kInt, "accepted", {r.B});
    Result target(gpu, a[8], at::kInt, "target_ids", {r.B, r.W});
    Result next(gpu, a[9], at::kInt, "next_token", {r.B});
    Result committed(gpu, a[10], at::kInt, "committed", {r.B});
    Result logprobs(gpu, a[11], at::kFloat, "logprobs", {r.B, r.W});
    const Stream stream(a[12], gpu);
    for (Result *x : {&accepted, &target, &next, &committed, &logprobs}) x->ready(stream, r.logits);
    const das_sampling sampling = filters.sampling();
    const das_status s = without_gil([&] {
        return das_sample_accept(r.logits.data_ptr(), r.kind, at_of<int32_t>(draft), r.batch, r.width, r.vocab,
                                 r.stride, &sampling, r.uniforms(), accepted.as<int32_t>(), target.as<int32_t>(),
                                 next.as<int32_t>(), committed.as<int32_t>(), logprobs.as<float>(), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    return pack(accepted, target, next, committed, logprobs);
    END_HANDLE_TH_ERRORS
}

PyObject *speculative_accept(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    count_args(n, 17);
    Gpu gpu;
    const Rows r(gpu, a[0], a[3], "target_logits"), d(gpu, a[1], a[3], "draft_logits");
    if (d.kind != r.kind) wrong_type(a[1], "draft_logits", "of target_logits' type");
    if (d.logits.sizes() != r.logits.sizes())
        refuse(PyExc_ValueError, "draft_logits must have target_logits' shape");
    const at::Tensor &draft = need(gpu, a[2], at::kInt, "draft_ids", {r.B, r.W});
    const at::Tensor &again = need(gpu, a[4], at::kFloat, "resample", {r.B});
    const Filters filters(gpu, a + 5, r.B), draft_filters(gpu, a + 9, r.B, true);
    Result accepted(gpu, a[13], at::kInt, "accepted", {r.B});
    Result next(gpu, a[14], at::kInt, "next_token", {r.B});
    Result committed(gpu, a[15], at::kInt, "committed", {r.B});
    Result records(gpu, Py_None, at::kByte, "records", {2 * DAS_RECORD_BYTES * r.B * r.W});
    const Stream stream(a[16], gpu);
    for (Result *x : {&accepted, &next, &committed, &records}) x->ready(stream, r.logits);
    const das_sampling sampling = filters.sampling();
    das_sampling draft_sampling = draft_filters.sampling();
    if (!draft_sampling.temperature) draft_sampling.temperature = sampling.temperature;
    if (!draft_sampling.top_k) draft_sampling.top_k = sampling.top_k;
    if (!draft_sampling.top_p) draft_sampling.top_p = sampling.top_p;
    if (!draft_sampling.min_p) draft_sampling.min_p = sampling.min_p;
    const das_status s = without_gil([&] {
        return das_speculative_accept(r.logits.data_ptr(), r.stride, d.logits.data_ptr(), d.stride, r.kind,
                                      at_of<int32_t>(draft), r.batch, r.width, r.vocab, &sampling, &draft_sampling,
                                      r.uniforms(), at_of<float>(again), accepted.as<int32_t>(), next.as<int32_t>(),
                                      committed.as<int32_t>(), records.as<>(), stream.handle);
    });
    if (s != DAS_OK) return PyLong_FromLong(s);
    return pack(accepted, next, committed);
    END_HANDLE_TH_ERRORS
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(page_assign), METHOD(kv_append_paged), METHOD(mature_v_attention_paged),
                         METHOD(kv_append_paged4), METHOD(mature_v_attention_paged4), METHOD(qk_norm_rope),
                         METHOD(sample), METHOD(sample_accept), METHOD(speculative_accept), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
