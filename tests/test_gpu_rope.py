"""Norm and rotation of queries and keys against the formula in 64 bits (tests/paged4_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged4_ref as ref
from tests.gpu_util import dev_i32, half_ulp_bf16

pytestmark = pytest.mark.gpu


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def make(seed, B, T, Hq, H, D, rd, base=10000.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = (torch.randn((B, T, Hq + 2 * H, D), generator=g, device="cuda") * 3).to(torch.bfloat16)
    w = [1 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    freq = (base ** (-torch.arange(0, rd, 2, device="cuda", dtype=torch.float64) / max(rd, 1))).float()
    return rows[:, :, :Hq], rows[:, :, Hq:Hq + H], rows[:, :, Hq + H:], w, freq


def check(got, x, weight, eps, place, freq, interleaved, live):
    """Half a bf16 step, and the binary32 arithmetic: a norm is off by 8e-7 of itself (a sum of 12 steps, its
    root, two products), an angle by 1e-6, the rotation by 2 roundings: 2.5e-6 of the pair's sizes."""
    w = None if weight is None else f64(weight)
    want, size = ref.norm_rope(f64(x), w, eps, ref.angles(place, freq.cpu().numpy()), interleaved)
    err = np.abs(f64(got) - want)
    bound = half_ulp_bf16(np.abs(want) + 2.5e-6 * size) + 2.5e-6 * size + 1e-38
    assert np.all((err <= bound)[live]), float((err / bound)[live].max())


@pytest.mark.parametrize("B,T,Hq,H,D,rd,interleaved,eps,wtype", [
    (1, 1, 1, 1, 64, 64, False, 1e-6, None), (1, 1, 32, 32, 128, 128, False, 1e-6, torch.bfloat16),
    (2, 3, 4, 1, 64, 32, True, 1e-5, torch.float32), (3, 17, 5, 5, 128, 64, True, 1e-6, torch.bfloat16),
    (2, 9, 8, 2, 128, 48, False, 0.0, torch.float32), (2, 5, 7, 3, 64, 8, False, None, None),
    (1, 70, 6, 2, 128, 0, False, 1e-6, torch.bfloat16), (5, 40, 3, 1, 128, 128, True, None, None),
    (2, 333, 16, 4, 64, 64, False, 1e-6, torch.float32), (33, 2, 1, 1, 128, 8, True, 1e-6, torch.bfloat16)])
def test_matches_the_formula(B, T, Hq, H, D, rd, interleaved, eps, wtype):
    q, k, v, w, freq = make(B + T + D + rd, B, T, Hq, H, D, rd)
    w = [None, None] if wtype is None else [x.to(wtype) for x in w]
    rng = np.random.default_rng(T)
    P, n = rng.integers(0, 40000, B), rng.integers(0, T + 1, B)
    n[0] = T
    outs = [torch.full((B, T, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H)]
    r = das.das_qk_norm_rope(q, k, v, freq, dev_i32(P), dev_i32(n), q_weight=w[0], k_weight=w[1], eps=eps,
                             interleaved=interleaved, q_out=outs[0], k_out=outs[1], v_out=outs[2])
    assert all(a is b for a, b in zip(r, outs))
    live = np.arange(T)[None] < n[:, None]
    place = P[:, None] + np.arange(T)[None]
    check(outs[0], q, w[0], eps, place, freq, interleaved, live)
    check(outs[1], k, w[1], eps, place, freq, interleaved, live)
    assert torch.equal(outs[2][torch.from_numpy(live)], v[torch.from_numpy(live)])
    for o in outs:                                        # rows past a block are left as they were
        assert (o[torch.from_numpy(~live)] == 7).all()


def test_far_positions():
    """Positions near 2^31: a binary32 product of position and frequency would be off by whole turns."""
    q, k, v, _, freq = make(1, 3, 4, 2, 2, 64, 64, base=500000.0)
    P = np.array([2 ** 31 - 8, 12345678, 2 ** 24 + 1])
    qo, ko, _ = das.das_qk_norm_rope(q, k, None, freq, dev_i32(P), eps=None)
    place = P[:, None] + np.arange(4)[None]
    live = np.ones((3, 4), bool)
    # (n f / 2 pi is held to 2^-52 of itself: 2^-23 turns at 2^31, 7e-7 more)
    check(qo, q, None, None, place, freq, False, live)
    check(ko, k, None, None, place, freq, False, live)


def test_defaults_and_lengths_left_out():
    q, k, v, _, freq = make(2, 2, 6, 4, 2, 128, 128)
    qo, ko, vo = das.das_qk_norm_rope(q, k, v, freq)
    place = np.broadcast_to(np.arange(6), (2, 6))
    check(qo, q, None, 1e-6, place, freq, False, np.ones((2, 6), bool))
    assert torch.equal(vo, v)
    neg, _, none = das.das_qk_norm_rope(q, k, None, freq, dev_i32([-5, 0]))
    assert none is None and torch.equal(neg, qo)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_strided(interleaved):
    q, k, v, w, freq = make(3, 2, 21, 8, 2, 128, 96)
    args = dict(q_weight=w[0], k_weight=w[1], interleaved=interleaved)
    want = das.das_qk_norm_rope(q, k, v, freq, dev_i32([5, 900]), **args)
    # heads before tokens, and a batch whose rows lie backwards in memory order
    t = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
    got = das.das_qk_norm_rope(t(q), t(k), t(v), freq, dev_i32([5, 900]), **args)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    own = [x.contiguous() for x in (q, k, v)]
    das.das_qk_norm_rope(*own, freq, dev_i32([5, 900]), q_out=own[0], k_out=own[1], v_out=own[2], **args)
    assert all(torch.equal(a, b) for a, b in zip(own, want))


def test_zero_rows_infinities_and_nan_stay_with_their_heads():
    q, k, v, _, freq = (x.clone() if torch.is_tensor(x) else x for x in make(4, 1, 4, 4, 1, 64, 64))
    clean, _, _ = das.das_qk_norm_rope(q, k, v, freq)
    q[0, 1, 2] = 0
    q[0, 2, 0, 5] = float("nan")
    q[0, 3, 1, 7] = float("inf")
    out, _, _ = das.das_qk_norm_rope(q, k, v, freq)
    assert (out[0, 1, 2] == 0).all() and out[0, 2, 0].isnan().all() and out[0, 3, 1].isnan().any()
    same = torch.ones((1, 4, 4), dtype=torch.bool)
    same[0, 1, 2] = same[0, 2, 0] = same[0, 3, 1] = False
    assert torch.equal(out[same], clean[same])


def test_empty_batch_other_stream_and_graph():
    q, k, v, _, freq = make(5, 0, 4, 4, 1, 64, 64)
    out = das.das_qk_norm_rope(q, k, v, freq, dev_i32([]))
    assert out[0].shape == (0, 4, 4, 64)
    q, k, v, _, freq = make(6, 3, 5, 4, 2, 64, 64)
    P = dev_i32([1, 2, 3])
    want = das.das_qk_norm_rope(q, k, v, freq, P)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = das.das_qk_norm_rope(q, k, v, freq, P, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    outs = [torch.zeros_like(x) for x in want]
    with torch.cuda.graph(graph):
        das.das_qk_norm_rope(q, k, v, freq, P, q_out=outs[0], k_out=outs[1], v_out=outs[2])
    P.fill_(77)                                           # the captured call reads lengths when it is replayed
    graph.replay()
    again = das.das_qk_norm_rope(q, k, v, freq, P)
    assert all(torch.equal(a, b) for a, b in zip(outs, again)) and not torch.equal(outs[0], want[0])


def test_frequencies_of_any_size():
    """Frequencies from 2^-149 to 2^40, of both signs; no others than finite ones turn anything.  A frequency up to 2^20 is
    held to 2^-46 turns (2^66 / (2 pi) is cut to a whole number), times 100 below 2^-39: nothing beside 2.5e-6."""
    q, k, _, _, _ = make(6, 2, 100, 2, 1, 128, 128)
    rng = np.random.default_rng(6)
    f = np.ldexp(rng.uniform(1, 2, 64), rng.integers(-40, 21, 64)) * rng.choice([-1, 1], 64)
    f[:6] = [0.0, -0.0, 2.0 ** -149, 1.0, 1048575.9375, -3.0 * 2.0 ** -140]
    freq = torch.from_numpy(f.astype(np.float32)).cuda()
    place = np.broadcast_to(np.arange(100), (2, 100))
    qo, ko, _ = das.das_qk_norm_rope(q, k, None, freq, eps=None)
    check(qo, q, None, None, place, freq, False, np.ones((2, 100), bool))
    freq[3], freq[9], freq[11] = torch.inf, -torch.inf, torch.nan
    got, _, _ = das.das_qk_norm_rope(q, k, None, freq, eps=None)
    still = [3, 9, 11, 67, 73, 75]
    assert torch.equal(got[..., still], q[..., still])
    rest = [i for i in range(128) if i not in still]
    assert torch.equal(got[..., rest], qo[..., rest])
    freq[5] = 2.0 ** 40                                      # held to 2^-26 turns at position 1
    got, _, _ = das.das_qk_norm_rope(q, k, None, freq, eps=None)
    turn = 2.0 ** 40 / (2 * np.pi) % 1.0                     # (binary64 has 2^-16 of it: 1e-4 of a turn)
    want = f64(q)[:, 1, :, 5] * np.cos(2 * np.pi * turn) - f64(q)[:, 1, :, 69] * np.sin(2 * np.pi * turn)
    size = np.abs(f64(q)[:, 1, :, 5]) + np.abs(f64(q)[:, 1, :, 69])
    assert (np.abs(f64(got)[:, 1, :, 5] - want) <= half_ulp_bf16(size) + 1e-3 * size).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rd", [(64, 0), (64, 32), (128, 8), (128, 64), (128, 120)])
def test_infinities_beside_what_is_not_rotated(D, rd, interleaved):
    """Elements from rotary_dim on are not rotated: without a norm they pass as they are, whatever stands beside them; with one
    an infinity makes its row's finite elements 0 and itself NaN."""
    q, k, _, w, freq = make(30 + rd, 2, 3, 2, 1, D, rd)
    q, k = q.clone(), k.clone()
    tail = list(range(rd, D))
    q[0, 1, 0, tail[1]], q[0, 2, 1, tail[2]], q[1, 0, 0, tail[4]] = torch.inf, torch.nan, -torch.inf
    k[1, 1, 0, tail[-1]], k[1, 2, 0, tail[0]] = -torch.inf, torch.inf
    P = dev_i32([3, 70])
    qo, ko, _ = das.das_qk_norm_rope(q, k, None, freq, P, eps=None, interleaved=interleaved)
    for got, x in ((qo, q), (ko, k)):
        a, b = f64(got)[..., rd:], f64(x)[..., rd:]
        assert np.array_equal(a, b, equal_nan=True) and np.isfinite(f64(got)[..., :rd]).all()
    place = np.array([3, 70])[:, None] + np.arange(3)
    qo, ko, _ = das.das_qk_norm_rope(q, k, None, freq, P, q_weight=w[0], k_weight=w[1], interleaved=interleaved)
    for got, x, weight in ((qo, q, w[0]), (ko, k, w[1])):
        with np.errstate(invalid="ignore"):
            want, _ = ref.norm_rope(f64(x), f64(weight), 1e-6, ref.angles(place, freq.cpu().numpy()), interleaved)
        got, bad = f64(got), np.isinf(f64(x)).any(-1)
        assert bad.sum() == np.isinf(f64(x)).sum() > 0        # one to a row
        assert np.array_equal(got[bad], want[bad], equal_nan=True) and not np.nan_to_num(got[bad]).any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_frequencies_that_are_not_finite_leave_infinities_alone(interleaved):
    q, k, _, _, freq = make(31, 1, 5, 2, 1, 64, 48)
    q = q.clone()
    freq[2], freq[7], freq[23] = torch.inf, torch.nan, -torch.inf
    pair = lambda j: (2 * j, 2 * j + 1) if interleaved else (j, j + 24)
    q[0, 1, 0, pair(2)[0]], q[0, 2, 1, pair(7)[1]], q[0, 3, 0, pair(23)[1]] = torch.inf, -torch.inf, torch.nan
    qo, _, _ = das.das_qk_norm_rope(q, k, None, freq, dev_i32([9]), eps=None, interleaved=interleaved)
    still = [e for j in (2, 7, 23) for e in pair(j)] + list(range(48, 64))
    assert np.array_equal(f64(qo)[..., still], f64(q)[..., still], equal_nan=True)
    rest = [e for e in range(48) if e not in still]
    assert qo[..., rest].isfinite().all()
