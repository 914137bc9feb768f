"""What the calls of the 4-bit cache, of norm and rotation, and of speculative acceptance refuse on the
host, without a GPU."""
import ctypes

import pytest
import torch

import paper_2609_34538_gb300 as das

L, A = das.LIB, ctypes.c_void_p(256)
NULL = ctypes.c_void_p(0)
OK, BAD, UNSUPPORTED = das.DAS_OK, das.DAS_ERR_INVALID_ARG, das.DAS_ERR_UNSUPPORTED


def cache(k=256, v=256, ks=256, vs=256, depths=2, layers=1, pages=4, heads=2, dim=64):
    return ctypes.byref(das.das_kv_cache_paged4(k, v, ks, vs, 0, 0, depths, layers, pages, heads, dim))


@pytest.mark.parametrize("change,code", [(dict(dim=96), UNSUPPORTED), (dict(k=0), BAD), (dict(v=8), BAD),
                                         (dict(ks=0), BAD), (dict(vs=24), BAD), (dict(depths=0), BAD),
                                         (dict(depths=64), BAD), (dict(pages=0), BAD), (dict(pages=1 << 25), BAD),
                                         (dict(heads=0), BAD)])
def test_cache_refusals(change, code):
    c = cache(**change)
    assert L.das_kv_append_paged4(c, A, A, 1, 4, A, 4, A, A, NULL) == code
    assert L.das_mature_v_attention_paged4(c, 0, 1, 1, A, 4, A, A, 1, 1, A, A, A, 2, 0.0, A, A, A, 1 << 30, NULL) == code


def test_append_refusals():
    call = lambda c=cache(), k=A, batch=1, W=4, slots=A, n=4, start=A, flag=A: L.das_kv_append_paged4(
        c, k, A, batch, W, slots, n, start, flag, NULL)
    assert call(c=None) == BAD and call(k=NULL) == BAD and call(k=ctypes.c_void_p(8)) == BAD
    assert call(batch=-1) == BAD and call(W=0) == BAD and call(slots=NULL) == BAD and call(n=-1) == BAD
    assert call(start=NULL) == BAD and call(flag=NULL) == BAD
    assert call(W=1 << 25) == UNSUPPORTED and call(c=cache(depths=63, layers=4096, heads=128), batch=1 << 10) == UNSUPPORTED


def test_attention_refusals():
    def call(layer=0, kd=1, vd=1, rows=4, batch=1, T=1, Hq=2, q=A, scale=0.0, table=A):
        return L.das_mature_v_attention_paged4(cache(), layer, kd, vd, table, rows, A, A, batch, T, q, A, A, Hq, scale, A,
                                               A, A, 1 << 30, NULL)
    assert call(layer=1) == BAD and call(layer=-1) == BAD and call(kd=0) == BAD and call(vd=3) == BAD
    assert call(rows=0) == BAD and call(batch=0) == BAD and call(T=0) == BAD and call(Hq=3) == BAD and call(Hq=0) == BAD
    assert call(q=ctypes.c_void_p(264)) == BAD and call(scale=float("nan")) == BAD and call(table=NULL) == BAD
    assert call(T=65) == UNSUPPORTED and call(T=33, Hq=4) == UNSUPPORTED and call(batch=(1 << 20) + 1) == UNSUPPORTED
    size = L.das_workspace_size_paged4
    assert size(None, 1, 2, 1) == 0 and size(cache(dim=32), 1, 2, 1) == 0 and size(cache(), 0, 2, 1) == 0
    assert size(cache(), 1, 3, 1) == 0 and size(cache(), 1, 2, 65) == 0


def rows(data=256, batch=1024, token=512, head=64):
    return ctypes.byref(das.das_head_rows(data, batch, token, head))


def test_norm_and_rotation_refusals():
    def call(q=rows(), k=rows(), v=rows(), B=1, T=2, Hq=4, H=2, D=64, qw=A, wt=0, eps=1e-6, freq=A, rd=64, qo=A, vo=A):
        return L.das_qk_norm_rope(q, k, v, B, T, Hq, H, D, qw, A, wt, eps, freq, rd, 0, A, A, qo, A, vo, NULL)
    assert call(q=None) == BAD and call(k=None) == BAD and call(v=None) == BAD and call(vo=NULL) == BAD
    assert call(q=rows(data=0)) == BAD and call(q=rows(data=260)) == BAD and call(k=rows(token=514)) == BAD
    assert call(v=rows(head=66)) == BAD and call(q=rows(batch=1)) == BAD
    assert call(B=-1) == BAD and call(T=0) == BAD and call(Hq=0) == BAD and call(H=0) == BAD
    assert call(eps=float("nan")) == BAD and call(freq=NULL) == BAD and call(rd=-8) == BAD and call(rd=12) == BAD
    assert call(rd=72) == BAD and call(wt=2) == BAD and call(qw=ctypes.c_void_p(264)) == BAD
    assert call(qw=ctypes.c_void_p(260), wt=1) == BAD and call(qo=NULL) == BAD and call(qo=ctypes.c_void_p(260)) == BAD
    assert call(D=96, rd=0) == UNSUPPORTED and call(B=1 << 20, T=1 << 12) == UNSUPPORTED
    assert call(Hq=1 << 21) == UNSUPPORTED


def test_speculative_acceptance_refusals():
    def call(t=A, d=A, ts=10, ds=10, kind=0, ids=A, B=1, W=1, V=10, u=A, again=A, acc=A, nxt=A, rec=A):
        return L.das_speculative_accept(t, ts, d, ds, kind, ids, B, W, V, None, None, u, again, acc, nxt, NULL, rec, NULL)
    for name in ("t", "d", "ids", "u", "again", "acc", "nxt", "rec"):
        assert call(**{name: NULL}) == BAD, name
    assert call(kind=2) == BAD and call(B=-1) == BAD and call(W=0) == BAD and call(W=1025) == BAD and call(V=0) == BAD
    assert call(ts=9) == BAD and call(ds=9) == BAD and call(t=ctypes.c_void_p(258)) == BAD
    assert call(d=ctypes.c_void_p(257), kind=1) == BAD and call(rec=ctypes.c_void_p(264)) == BAD
    assert call(B=1 << 30, W=1024) == BAD


def test_empty_calls_do_nothing():
    assert L.das_kv_append_paged4(cache(), NULL, NULL, 0, 4, NULL, 0, A, A, NULL) == OK
    for kind in (0, 1):
        assert L.das_speculative_accept(NULL, 10, NULL, 10, kind, NULL, 0, 3, 10, None, None, NULL, NULL, NULL, NULL, NULL,
                                        NULL, NULL) == OK
    r = ctypes.byref(das.das_head_rows(0, 0, 0, 0))
    assert L.das_qk_norm_rope(r, r, None, 0, 3, 4, 2, 64, NULL, NULL, 0, 1e-6, A, 64, 0, NULL, NULL, NULL, NULL, NULL,
                              NULL) == OK


def test_binding_refuses_host_tensors_and_wrong_types():
    x, i = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="q must be on a CUDA device"):
        das.das_qk_norm_rope(x, x, x, torch.ones(32), i)
    with pytest.raises(TypeError, match="q must be torch.bfloat16"):
        das.das_qk_norm_rope(x.float(), x, x, torch.ones(32), i)
    with pytest.raises(TypeError, match="uint8"):
        das.PagedKVCache4(x, x, x, x)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        das.das_speculative_accept(x[0].double(), x[0], i, i, i)


@pytest.fixture
def fake():
    """Tensors that say which GPU they are on and have no memory: nothing can be launched on them."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        yield lambda dtype, *shape, gpu=0: torch.empty(shape, dtype=dtype, device=f"cuda:{gpu}")


OTHER_GPU = "on cuda:1, other arguments on cuda:0"


def test_norm_and_rotation_take_matching_tensors_of_one_gpu(fake):
    b, f, i = torch.bfloat16, torch.float32, torch.int32
    shapes = dict(q=(b, 2, 3, 4, 64), k=(b, 2, 3, 2, 64), v=(b, 2, 3, 2, 64), inv_freq=(f, 32), prefix_len=(i, 2),
                  block_len=(i, 2), q_weight=(b, 64), k_weight=(b, 64), q_out=(b, 2, 3, 4, 64), k_out=(b, 2, 3, 2, 64),
                  v_out=(b, 2, 3, 2, 64))
    for other in list(shapes)[1:]:
        with pytest.raises(ValueError, match=f"{other} is {OTHER_GPU}"):
            das.das_qk_norm_rope(**{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})
    args = {n: fake(*s) for n, s in shapes.items()}

    def wrong(match, kind=ValueError, **change):
        with pytest.raises(kind, match=match):
            das.das_qk_norm_rope(**(args | change))
    wrong("k must be", k=fake(b, 2, 3, 2, 128))
    wrong("v must be", v=fake(b, 2, 3, 1, 64))
    wrong("4 dims", q=fake(b, 3, 4, 64))
    wrong("contiguous rows", q=fake(b, 2, 3, 64, 64).transpose(2, 3))
    wrong("multiples of 4", q=fake(b, 2, 3, 4, 66)[..., :64])
    wrong("prefix_len", prefix_len=fake(i, 3))
    wrong("q_weight", TypeError, q_weight=fake(torch.float16, 64))
    wrong("k_weight", TypeError, k_weight=fake(f, 64))
    wrong("q_weight must have shape", q_weight=fake(b, 32))
    wrong("eps", eps=-1.0)
    wrong("eps", eps=float("nan"))
    wrong("v_out without v", v=None)
    wrong("q_out must have shape", q_out=fake(b, 2, 3, 2, 64))


def test_speculative_acceptance_takes_matching_tensors_of_one_gpu(fake):
    i32, f32 = torch.int32, torch.float32
    shapes = dict(target_logits=(f32, 2, 3, 50), draft_logits=(f32, 2, 3, 50), draft_ids=(i32, 2, 3), uniforms=(f32, 2, 3),
                  resample=(f32, 2), temperature=(f32, 2), top_k=(i32, 2), top_p=(f32, 2), min_p=(f32, 2),
                  draft_temperature=(f32, 2), draft_top_k=(i32, 2), draft_top_p=(f32, 2), draft_min_p=(f32, 2),
                  accepted=(i32, 2), next_token=(i32, 2), committed=(i32, 2))
    for other in list(shapes)[1:]:
        with pytest.raises(ValueError, match=f"{other} is {OTHER_GPU}"):
            das.das_speculative_accept(**{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})
    args = {n: fake(*s) for n, s in shapes.items()}
    for change, kind, match in ((dict(draft_logits=fake(torch.bfloat16, 2, 3, 50)), TypeError, "of target_logits' type"),
                                (dict(draft_logits=fake(f32, 2, 3, 51)), ValueError, "target_logits' shape"),
                                (dict(draft_ids=fake(i32, 2, 4)), ValueError, "draft_ids"),
                                (dict(resample=fake(f32, 3)), ValueError, "resample"),
                                (dict(draft_top_k=fake(f32, 2)), TypeError, "draft_top_k"),
                                (dict(target_logits=fake(f32, 2, 50, 3).transpose(1, 2)), ValueError, "contiguous rows")):
        with pytest.raises(kind, match=match):
            das.das_speculative_accept(**(args | change))


class CacheOnGpu0:
    """What the calls read of a PagedKVCache4 before they launch."""
    def __init__(self):
        self.desc = das.das_kv_cache_paged4(256, 256, 256, 256, 0, 0, 2, 1, 4, 2, 64)
        self.address, self.gpu, self.shape = ctypes.addressof(self.desc), 0, (2, 1, 4, 2, 64)


def test_cache_calls_refuse_tensors_of_two_gpus(fake):
    i32, bf16 = torch.int32, torch.bfloat16
    c = CacheOnGpu0()
    shapes = dict(k_new=(bf16, 2, 1, 1, 4, 2, 64), v_new=(bf16, 2, 1, 1, 4, 2, 64), slots=(i32, 8), slot_start=(i32, 2),
                  error_flag=(i32, 1))
    for other in shapes:
        with pytest.raises(ValueError, match="on cuda:1"):
            das.das_kv_append_paged4(c, **{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})
    with pytest.raises(ValueError, match="k_new / v_new must be"):
        das.das_kv_append_paged4(c, **{n: fake(*s) for n, s in (shapes | dict(v_new=(bf16, 2, 1, 1, 5, 2, 64))).items()})
    shapes = dict(block_table=(i32, 1, 4), prefix_len=(i32, 1), block_len=(i32, 1), q=(bf16, 1, 2, 4, 64),
                  k_blk=(bf16, 1, 2, 2, 64), v_blk=(bf16, 1, 2, 2, 64), workspace=(torch.uint8, 1 << 20),
                  out=(bf16, 1, 2, 4, 64), lse=(torch.float32, 1, 4, 2))
    for other in shapes:
        with pytest.raises(ValueError, match="on cuda:1"):
            das.das_mature_v_attention_paged4(c, 0, 1, 1, **{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})
    with pytest.raises(ValueError, match="on cuda:1, the cache on cuda:0"):
        das.das_mature_v_attention_paged4(c, 0, 1, 1, **{n: fake(*s, gpu=1) for n, s in shapes.items()})


def test_a_cache_has_matching_tensors_on_one_gpu(fake):
    u8, f32 = torch.uint8, torch.float32
    shapes = dict(k=(u8, 1, 1, 2, 1, 64, 32), v=(u8, 1, 1, 2, 1, 8, 64, 4), k_scale=(u8, 1, 1, 2, 1, 64, 2),
                  v_scale=(u8, 1, 1, 2, 1, 2, 64), k_unit=(f32, 1, 1, 1), v_unit=(f32, 1, 1, 1))
    for other in list(shapes)[1:]:
        with pytest.raises(ValueError, match=f"{other} is on cuda:1, k on cuda:0"):
            das.PagedKVCache4(**{n: fake(*s, gpu=int(n == other)) for n, s in shapes.items()})
    for name, shape in (("k", (1, 1, 2, 1, 32, 32)), ("v", (1, 1, 2, 1, 8, 32, 4)), ("k_scale", (1, 1, 2, 1, 64, 4)),
                        ("v_scale", (1, 1, 2, 1, 64, 2)), ("k_unit", (1, 1, 2))):
        dt = f32 if name == "k_unit" else u8
        with pytest.raises(ValueError, match="pages must have 64" if name == "k" else name):
            das.PagedKVCache4(**{n: fake(dt, *shape) if n == name else fake(*s) for n, s in shapes.items()})


def test_weights_that_are_not_read_are_not_looked_at():
    """Without a norm the weights are not read, so their addresses do not matter either; with one they have to be aligned."""
    r = ctypes.byref(das.das_head_rows(0, 0, 0, 0))
    call = lambda qw, kw, wt, eps: L.das_qk_norm_rope(r, r, None, 0, 3, 4, 2, 64, ctypes.c_void_p(qw), ctypes.c_void_p(kw), wt,
                                                      eps, A, 64, 0, NULL, NULL, NULL, NULL, NULL, NULL)
    for qw, kw in ((1, 256), (256, 1), (1, 1)):
        for wt in (0, 1):
            assert call(qw, kw, wt, -1.0) == OK
            assert call(qw, kw, wt, 0.0) == BAD
