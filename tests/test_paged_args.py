"""What the paged-cache and sampling calls refuse on the host, without a GPU: status codes of the C
ABI (addresses are never used, since the checks fail first) and exceptions of the binding."""
import ctypes

import pytest
import torch

import paper_2609_34538_gb300 as das

L, A = das.LIB, ctypes.c_void_p(256)
NULL = ctypes.c_void_p(0)
BAD, UNSUPPORTED = das.DAS_ERR_INVALID_ARG, das.DAS_ERR_UNSUPPORTED


def cache(k=256, v=256, ks=256, vs=256, depths=2, layers=1, pages=4, heads=2, dim=64):
    return ctypes.byref(das.das_kv_cache_paged(k, v, ks, vs, depths, layers, pages, heads, dim))


@pytest.mark.parametrize("change", [dict(batch=-1), dict(max_pages=0), dict(max_pages=1 << 25), dict(pages=0),
                                    dict(pages=1 << 25), dict(max_slots=-1), dict(slots=NULL), dict(count=NULL),
                                    dict(seq=NULL), dict(table=NULL), dict(flag=NULL)])
def test_page_assign_refusals(change):
    a = dict(batch=2, max_pages=4, pages=8, max_slots=16, slots=A, count=A, seq=A, table=A, flag=A) | change
    assert L.das_page_assign(a["seq"], A, a["batch"], a["table"], a["max_pages"], A, a["pages"], a["count"], a["slots"],
                             a["max_slots"], A, A, A, a["flag"], NULL) == BAD


@pytest.mark.parametrize("change,code", [(dict(dim=96), UNSUPPORTED), (dict(k=0), BAD), (dict(v=8), BAD),
                                         (dict(ks=0), BAD), (dict(depths=0), BAD), (dict(depths=64), BAD),
                                         (dict(pages=0), BAD), (dict(pages=1 << 25), BAD), (dict(heads=0), BAD)])
def test_cache_refusals(change, code):
    c = cache(**change)
    assert L.das_kv_append_paged(c, A, A, 1, 4, A, 4, A, A, NULL) == code
    assert L.das_mature_v_attention_paged(c, 0, 1, 1, A, 4, A, A, 1, 1, A, A, A, 2, 0.0, A, A, A, 1 << 30, NULL) == code


def test_page_assign_limits():
    assert L.das_page_assign(A, A, (1 << 24) + 1, A, 4, A, 8, A, A, 16, A, A, A, A, NULL) == UNSUPPORTED
    assert L.das_page_assign(A, A, 2, A, 4, A, 8, A, A, (1 << 30) + 1, A, A, A, A, NULL) == UNSUPPORTED


def test_append_refusals():
    call = lambda c=cache(), k=A, batch=1, W=4, slots=A, n=4, start=A, flag=A: L.das_kv_append_paged(
        c, k, A, batch, W, slots, n, start, flag, NULL)
    assert call(c=None) == BAD and call(k=NULL) == BAD and call(k=ctypes.c_void_p(8)) == BAD
    assert call(batch=-1) == BAD and call(W=0) == BAD and call(slots=NULL) == BAD and call(n=-1) == BAD
    assert call(start=NULL) == BAD and call(flag=NULL) == BAD
    assert call(W=1 << 25) == UNSUPPORTED and call(c=cache(depths=63, layers=4096, heads=128), batch=1 << 10) == UNSUPPORTED


def test_attention_refusals():
    def call(layer=0, kd=1, vd=1, rows=4, batch=1, T=1, Hq=2, q=A, scale=0.0, table=A):
        return L.das_mature_v_attention_paged(cache(), layer, kd, vd, table, rows, A, A, batch, T, q, A, A, Hq, scale, A,
                                              A, A, 1 << 30, NULL)
    assert call(layer=1) == BAD and call(layer=-1) == BAD and call(kd=0) == BAD and call(vd=3) == BAD
    assert call(rows=0) == BAD and call(batch=0) == BAD and call(T=0) == BAD and call(Hq=3) == BAD and call(Hq=0) == BAD
    assert call(q=ctypes.c_void_p(264)) == BAD and call(scale=float("nan")) == BAD and call(table=NULL) == BAD
    assert call(T=65) == UNSUPPORTED and call(T=33, Hq=4) == UNSUPPORTED and call(batch=(1 << 20) + 1) == UNSUPPORTED
    size = L.das_workspace_size_paged
    assert size(None, 1, 2, 1) == 0 and size(cache(dim=32), 1, 2, 1) == 0 and size(cache(), 0, 2, 1) == 0
    assert size(cache(), 1, 3, 1) == 0 and size(cache(), 1, 2, 65) == 0


def test_sample_refusals():
    def call(logits=A, kind=0, B=1, W=1, V=10, stride=10, u=A, out=A):
        return L.das_sample(logits, kind, B, W, V, stride, None, u, out, NULL, NULL)
    assert call(logits=NULL) == BAD and call(kind=2) == BAD and call(B=-1) == BAD and call(W=0) == BAD
    assert call(W=1025) == BAD and call(V=0) == BAD and call(stride=9) == BAD and call(u=NULL) == BAD
    assert call(out=NULL) == BAD and call(logits=ctypes.c_void_p(258)) == BAD
    assert call(logits=ctypes.c_void_p(257), kind=1) == BAD
    accept = lambda draft=A, acc=A, nxt=A: L.das_sample_accept(A, 0, draft, 1, 1, 10, 10, None, A, acc, A, nxt, NULL, NULL,
                                                               NULL)
    assert accept(draft=NULL) == BAD and accept(acc=NULL) == BAD and accept(nxt=NULL) == BAD


def test_binding_refuses_host_tensors_and_wrong_types():
    i32, f32 = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2, 8))
    with pytest.raises(ValueError, match="CUDA"):
        das.das_page_assign(i32, i32, i32.view(2, 1), i32, i32[:1], i32, i32[:1])
    with pytest.raises(TypeError, match="int32"):
        das.das_page_assign(f32, i32, i32.view(2, 1), i32, i32[:1], i32, i32[:1])
    with pytest.raises(ValueError, match="CUDA"):
        das.das_sample(f32, f32[..., 0])
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        das.das_sample(f32.double(), f32[..., 0])
    with pytest.raises(TypeError, match="uint8"):
        das.PagedKVCache(f32, f32, f32, f32)


def test_binding_module_refuses_bad_numbers():
    desc = das.das_kv_cache_paged(256, 256, 256, 256, 2, 1, 4, 2, 64)
    t = torch.zeros((1, 4), dtype=torch.int32)
    call = lambda layer=0, address=ctypes.addressof(desc): das._calls.mature_v_attention_paged(
        address, layer, 1, 1, t, t[0, :1], t[0, :1], t, t, t, t, None, None, 0.0, None)
    with pytest.raises(OverflowError, match="layer"):
        call(layer=1 << 40)
    with pytest.raises(TypeError):
        call(layer=0.5)
    with pytest.raises(ValueError, match="cache"):
        call(address=0)
    with pytest.raises(ValueError, match="block_table must be on a CUDA device"):
        call()
    with pytest.raises(TypeError, match="9 arguments"):
        das._calls.sample(t, t)


@pytest.fixture
def fake():
    """Tensors that say which GPU they are on and have no memory: nothing can be launched on them."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        yield lambda dtype, *shape, gpu=0: torch.empty(shape, dtype=dtype, device=f"cuda:{gpu}")


OTHER_GPU = "on cuda:1, other arguments on cuda:0"


def test_page_assign_refuses_tensors_of_two_gpus(fake):
    shapes = dict(seq_len=(3,), grow=(3,), block_table=(3, 4), free_pages=(8,), free_count=(1,), slots=(16,),
                  error_flag=(1,), new_len=(3,), new_free_count=(1,), slot_start=(4,))
    for other in list(shapes)[1:]:
        args = {n: fake(torch.int32, *s, gpu=int(n == other)) for n, s in shapes.items()}
        with pytest.raises(ValueError, match=f"{other} is {OTHER_GPU}"):
            das.das_page_assign(**args)


def test_sampling_refuses_tensors_of_two_gpus(fake):
    i32, f32 = torch.int32, torch.float32
    shapes = dict(logits=(f32, 2, 3, 50), draft_ids=(i32, 2, 3), uniforms=(f32, 2, 3), temperature=(f32, 2), top_k=(i32, 2),
                  top_p=(f32, 2), min_p=(f32, 2), accepted=(i32, 2), target_ids=(i32, 2, 3), next_token=(i32, 2),
                  committed=(i32, 2), logprobs=(f32, 2, 3))
    for other in list(shapes)[1:]:
        args = {n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()}
        with pytest.raises(ValueError, match=f"{other} is {OTHER_GPU}"):
            das.das_sample_accept(**args)
    shapes = {n: s for n, s in shapes.items() if n in ("logits", "uniforms", "temperature", "top_k", "top_p", "min_p")}
    shapes |= dict(tokens=(i32, 2, 3), logprobs=(f32, 2, 3))
    for other in list(shapes)[1:]:
        args = {n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()}
        with pytest.raises(ValueError, match=f"{other} is {OTHER_GPU}"):
            das.das_sample(**args)


class CacheOnGpu0:
    """What the calls read of a PagedKVCache before they launch."""
    def __init__(self):
        self.desc = das.das_kv_cache_paged(256, 256, 256, 256, 2, 1, 4, 2, 64)
        self.address, self.gpu, self.shape = ctypes.addressof(self.desc), 0, (2, 1, 4, 2, 64)


def test_cache_calls_refuse_tensors_of_two_gpus(fake):
    i32, bf16 = torch.int32, torch.bfloat16
    c = CacheOnGpu0()
    shapes = dict(k_new=(bf16, 2, 1, 1, 4, 2, 64), v_new=(bf16, 2, 1, 1, 4, 2, 64), slots=(i32, 8), slot_start=(i32, 2),
                  error_flag=(i32, 1))
    for other in shapes:
        args = {n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()}
        with pytest.raises(ValueError, match="on cuda:1" if other == "k_new" else f"{other} is {OTHER_GPU}"):
            das.das_kv_append_paged(c, **args)
    shapes = dict(block_table=(i32, 1, 4), prefix_len=(i32, 1), block_len=(i32, 1), q=(bf16, 1, 2, 4, 64),
                  k_blk=(bf16, 1, 2, 2, 64), v_blk=(bf16, 1, 2, 2, 64), workspace=(torch.uint8, 1 << 20),
                  out=(bf16, 1, 2, 4, 64), lse=(torch.float32, 1, 4, 2))
    for other in shapes:
        args = {n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()}
        with pytest.raises(ValueError, match="on cuda:1"):
            das.das_mature_v_attention_paged(c, 0, 1, 1, **args)
    # all of them on one GPU, the cache on another
    for shapes, call in ((dict(k_new=(bf16, 2, 1, 1, 4, 2, 64), v_new=(bf16, 2, 1, 1, 4, 2, 64), slots=(i32, 8),
                               slot_start=(i32, 2), error_flag=(i32, 1)), lambda **a: das.das_kv_append_paged(c, **a)),
                         (shapes, lambda **a: das.das_mature_v_attention_paged(c, 0, 1, 1, **a))):
        with pytest.raises(ValueError, match="on cuda:1, the cache on cuda:0"):
            call(**{n: fake(*s, gpu=1) for n, s in shapes.items()})


def test_a_cache_is_on_one_gpu(fake):
    shapes = dict(k=(torch.uint8, 1, 1, 2, 1, 64, 64), v=(torch.uint8, 1, 1, 2, 1, 64, 64),
                  k_scale=(torch.float32, 1, 1, 2, 1), v_scale=(torch.float32, 1, 1, 2, 1))
    for other in list(shapes)[1:]:
        with pytest.raises(ValueError, match=f"{other} is on cuda:1, k on cuda:0"):
            das.PagedKVCache(**{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})


def test_a_stream_of_another_gpu_is_refused(fake):
    class Stream:                        # what the binding reads of a torch.cuda.Stream
        stream_id, device_index, device_type = 0, 1, 1
    logits, u = fake(torch.float32, 1, 2, 9), fake(torch.float32, 1, 2)
    with pytest.raises(ValueError, match="stream is of cuda:1, the arguments on cuda:0"):
        das.das_sample(logits, u, stream=Stream())


def test_empty_calls_do_nothing():
    """No sequences: whatever has no elements has no address either."""
    ok = das.DAS_OK
    assert L.das_kv_append_paged(cache(), NULL, NULL, 0, 4, NULL, 0, A, A, NULL) == ok
    assert L.das_kv_append_paged(cache(), NULL, NULL, 0, 4, A, 4, A, A, NULL) == ok
    for kind in (0, 1):
        assert L.das_sample(NULL, kind, 0, 3, 10, 10, None, NULL, NULL, NULL, NULL) == ok
        assert L.das_sample_accept(NULL, kind, NULL, 0, 3, 10, 10, None, NULL, NULL, NULL, NULL, NULL, NULL, NULL) == ok
    # what is out of range without any sequence is refused as with one
    assert L.das_kv_append_paged(cache(), NULL, NULL, 0, 0, NULL, 0, A, A, NULL) == BAD
    assert L.das_kv_append_paged(cache(), NULL, NULL, 0, 4, NULL, 4, A, A, NULL) == BAD
    assert L.das_kv_append_paged(cache(dim=96), NULL, NULL, 0, 4, NULL, 0, A, A, NULL) == UNSUPPORTED
    assert L.das_sample(NULL, 2, 0, 3, 10, 10, None, NULL, NULL, NULL, NULL) == BAD
    assert L.das_sample(NULL, 0, 0, 3, 10, 9, None, NULL, NULL, NULL, NULL) == BAD
