"""The commit into the 4-bit cache and attention over it, against plain references in 64 bits
(tests/paged4_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged4_ref as ref
from tests.gpu_util import LSE_ABS, dev_i32, half_ulp_bf16

pytestmark = pytest.mark.gpu
PAGE, GROUP = 64, 32


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.uint8).cuda()


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def host(cache):
    return [t.cpu().numpy() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]


# ---- commit -----------------------------------------------------------------------

def append_case(rng, R, L, H, D, first, n, W, N):
    z = lambda *s: rng.integers(0, 256, (R, L, N, H) + s).astype(np.uint8)
    old = [z(PAGE, D // 2), z(PAGE, D // GROUP), z(8, D, 4), z(D // GROUP, PAGE)]
    units = [2.0 ** rng.integers(-3, 4, (R, L, H)) for _ in range(2)]
    B = len(n)
    x = rng.normal(0, 1, (2, R, L, B, W, H, D)) * 2.0 ** rng.integers(-4, 5, (2, R, L, B, W, H, 1))
    ids, slots, start = list(rng.permutation(N)), [], [0]
    for b in range(B):
        pg = [ids.pop() for _ in range(-(-(first[b] + n[b]) // PAGE))]
        slots += [pg[(first[b] + j) // PAGE] * PAGE + (first[b] + j) % PAGE for j in range(n[b])]
        start.append(len(slots))
    return old, units, x, slots, start


def run_append(old, units, x, slots, start, repeat=1):
    cache = das.PagedKVCache4(u8(old[0]), u8(old[2]), u8(old[1]), u8(old[3]), *(u if u is None else f32(u) for u in units))
    flag = dev_i32([0])
    k, v = bf16(x[0]), bf16(x[1])
    for _ in range(repeat):
        das.das_kv_append_paged4(cache, k, v, dev_i32(slots if len(slots) else [0]), dev_i32(start), flag)
    return cache, f64(k), f64(v), flag.item()


def same(cache, want):
    k, ks, v, vs = want
    return all(np.array_equal(a, b) for a, b in zip(host(cache), (k, ks, v, vs)))


@pytest.mark.parametrize("repeat", [1, 2])
@pytest.mark.parametrize("R,L,H,D,first,n,W", [
    (1, 1, 1, 64, [0], [1], 1), (1, 1, 1, 128, [63], [1], 1), (2, 2, 3, 64, [5], [16], 16),
    (3, 1, 2, 128, [63, 0, 32], [1, 64, 33], 64), (1, 2, 8, 128, [10, 62], [200, 3], 201),
    (2, 1, 1, 128, [1, 0, 7], [0, 5, 0], 9), (1, 1, 5, 64, [33], [95], 95), (1, 1, 2, 64, [7, 8, 9], [2, 7, 8], 12)])
def test_append_codes_and_scales(R, L, H, D, first, n, W, repeat):
    rng = np.random.default_rng(D + W + H)
    old, units, x, slots, start = append_case(rng, R, L, H, D, first, n, W, 12)
    cache, k, v, flag = run_append(old, units, x, slots, start, repeat)
    assert same(cache, ref.append(*old, *units, k, v, slots, start)) and flag == 0


def test_append_extreme_values():
    rng = np.random.default_rng(3)
    old, units, x, slots, start = append_case(rng, 1, 1, 9, 64, [9], [20], 20, 2)
    for y in x:
        y[..., 0, :] *= 0.0
        y[..., 1, :] *= 2.0 ** 100
        y[..., 2, :] *= 2.0 ** -60
        y[..., 3, 5] = np.inf
        y[..., 4, 6] = np.nan
        y[..., 5, :] = 7.0
        y[..., 6, :] = np.sign(y[..., 6, :]) * np.inf
        y[..., 7, :32] = np.nan
        y[..., 8, :] = 2.0 ** -17 * 3.5 * rng.integers(-2, 3, y[..., 8, :].shape)   # at the least scales, and at ties
    for u in (units, [None, None], [np.full((1, 1, 9), 2.0 ** 40), np.full((1, 1, 9), 2.0 ** -40)]):
        cache, k, v, flag = run_append(old, u, x, slots, start)
        one = np.ones((1, 1, 9))
        want = ref.append(*old, *(one if t is None else t for t in u), k, v, slots, start)
        assert same(cache, want) and flag == 0


def test_append_ties_of_scales_and_codes():
    """Every bf16 significand as a group's largest, and multiples of half a step."""
    rng = np.random.default_rng(4)
    old, _, x, slots, start = append_case(rng, 1, 1, 4, 128, [0], [64], 64, 1)
    largest = (128 + np.arange(512) % 128) / 128.0 * 2.0 ** ((np.arange(512) // 128) - 2)
    x[0] = rng.uniform(-1, 1, x[0].shape)
    x[0].reshape(-1, 32)[:, 0] = 1.0
    x[0].reshape(-1, 32)[:] *= np.resize(largest, x[0].size // 32)[:, None]
    x[1] = rng.integers(-14, 15, x[1].shape) / 2.0        # ties, with the largest 7 or less
    cache, k, v, _ = run_append(old, [None, None], x, slots, start)
    one = np.ones((1, 1, 4))
    assert same(cache, ref.append(*old, one, one, k, v, slots, start))


@pytest.mark.parametrize("D", [64, 128])
def test_append_values_of_every_kind_side_by_side(D):
    """Groups that need care among many that do not, in every place of the four tokens that a lane has."""
    rng = np.random.default_rng(6)
    old, units, x, slots, start = append_case(rng, 2, 1, 4, D, [3, 40, 0], [130, 60, 25], 130, 8)
    groups = x.reshape(-1, 32)
    for y in (0.0, 2.0 ** -30, 2.0 ** 20, np.inf, np.nan, 2.0 ** -13):
        at = rng.choice(len(groups), len(groups) // 60, replace=False)
        few = rng.random((len(at), 32)) < 0.3
        groups[at] = np.where(few, y, groups[at] * (min(y, 1.0) if y == y else 1.0))
    x = groups.reshape(x.shape)
    cache, k, v, flag = run_append(old, units, x, slots, start, 2)
    assert same(cache, ref.append(*old, *units, k, v, slots, start)) and flag == 0


def test_append_two_streams_at_once():
    """Two sequences' tokens by two calls beside each other, on pages of their own."""
    rng = np.random.default_rng(7)
    old, units, x, slots, start = append_case(rng, 4, 2, 4, 128, [70, 5], [100, 100], 100, 8)
    want, k, v, _ = run_append(old, units, x, slots, start)
    cache = das.PagedKVCache4(u8(old[0]), u8(old[2]), u8(old[1]), u8(old[3]), *(f32(u) for u in units))
    flag, ks, vs = dev_i32([0]), bf16(x[0]), bf16(x[1])
    a = [(ks[:, :, b:b + 1].contiguous(), vs[:, :, b:b + 1].contiguous(), dev_i32(slots[start[b]:start[b + 1]]),
          dev_i32([0, 100])) for b in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for args, s in zip(a, streams):
            das.das_kv_append_paged4(cache, *args, flag, stream=s)
    torch.cuda.synchronize()
    assert same(cache, host(want)) and flag.item() == 0


def test_append_captured_with_page_assignment():
    """Steps of page assignment and commit, captured once and replayed: what they store is what eager steps store."""
    rng = np.random.default_rng(8)
    R, L, H, D, W = 2, 1, 3, 64, 10
    k, v = bf16(rng.normal(0, 1, (R, L, 2, W, H, D))), bf16(rng.normal(0, 1, (R, L, 2, W, H, D)))

    def books():
        cache = das.PagedKVCache4(*(u8(np.zeros(s, np.uint8)) for s in (
            (R, L, 8, H, PAGE, D // 2), (R, L, 8, H, 8, D, 4), (R, L, 8, H, PAGE, D // GROUP), (R, L, 8, H, D // GROUP, PAGE))))
        return cache, dev_i32([0, 0]), dev_i32(list(range(8))), dev_i32([8]), dev_i32([[0] * 4] * 2), dev_i32([0] * 2 * W), dev_i32([0])

    def step(b, grow):
        cache, length, free, count, table, slots, flag = b
        start = das.das_page_assign(length, grow, table, free, count, slots, flag, new_len=length, new_free_count=count)[2]
        das.das_kv_append_paged4(cache, k, v, slots, start, flag)

    a, b, grow = books(), books(), dev_i32([0, 0])
    step(a, grow)                                           # nothing grows
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, grow)
    for n in ([7, 3], [10, 0], [1, 9], [8, 8]) * 3:
        grow.copy_(dev_i32(n))
        graph.replay()
        step(b, grow)
    torch.cuda.synchronize()
    assert same(a[0], host(b[0])) and a[0].k.any() and all(torch.equal(x, y) for x, y in zip(a[1:], b[1:]))
    assert a[1].tolist() == [78, 60] and a[6].item() == 0


def test_append_leaves_what_it_refuses():
    rng = np.random.default_rng(5)
    old, units, x, slots, start = append_case(rng, 1, 1, 2, 64, [60, 0, 0, 0], [8, 4, 4, 4], 8, 8)
    slots = list(slots)
    slots[start[0] + 4] += 1                               # a second page that does not start at its first place
    slots[start[1]:start[2]] = [-1] * 4                    # no place
    slots[start[2]:start[3]] = [8 * PAGE + i for i in range(4)]  # a page past the pool
    cache, k, v, flag = run_append(old, units, x, slots, start)
    want = ref.append(*old, *units, k[:, :, :1], v[:, :, :1], slots[:4], [0, 4])
    want = ref.append(*want, *units, k[:, :, 3:], v[:, :, 3:], slots[start[3]:], [0, 4])
    assert flag == 2 and same(cache, want)
    for bad in ([0, 9, 9, 9, 9], [0, 0, 0, 0, 999], [4, 2, 2, 2, 2], [-3, -1, 0, 0, 0]):
        cache, k, v, flag = run_append(old, units, x, slots, bad)
        assert flag == 2 and same(cache, old)


# ---- attention --------------------------------------------------------------------

def attention_case(rng, D, Hq, Hkv, Tm, P, T, rows=None, poison=True):
    """Two depths: keys read at depth 1, values at depth 2; what no call may use reads as NaN."""
    B = len(P)
    need = [-(-p // PAGE) for p in P]
    rows = max(1, max(need)) if rows is None else rows
    N = sum(need) + 2
    ids = rng.permutation(N)
    table = np.full((B, rows), -1)
    at, used = 0, np.zeros((N, PAGE), bool)
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        for t in range(need[b]):
            used[table[b, t], :min(PAGE, P[b] - t * PAGE)] = True
        at += need[b]
    c = lambda *s: np.clip(np.rint(rng.normal(0, 2.6, (N, Hkv) + s)), -7, 7) + 8
    pack = lambda *s: (c(*s).astype(np.uint8) | c(*s).astype(np.uint8) << 4).astype(np.uint8)
    k, v = pack(PAGE, D // 2), pack(8, D, 4)
    ks, vs = (rng.integers(100, 117, (N, Hkv) + s).astype(np.uint8) for s in ((PAGE, D // GROUP), (D // GROUP, PAGE)))
    if poison:
        ks[np.broadcast_to(~used[:, None, :, None], ks.shape)] = 0xff
        vs[np.broadcast_to(~used[:, None, None, :], vs.shape)] = 0xff
    ku, vu = (2.0 ** rng.integers(-2, 2, Hkv) for _ in range(2))
    f = lambda *s: rng.normal(0, 1, s)
    q, kb, vb = f(B, Tm, Hq, D), f(B, Tm, Hkv, D), f(B, Tm, Hkv, D)
    if poison:
        for b in range(B):
            q[b, T[b]:], kb[b, T[b]:], vb[b, T[b]:] = np.nan, np.nan, np.nan
    return dict(k=k, ks=ks, v=v, vs=vs, ku=ku, vu=vu, table=table, P=np.array(P), T=np.array(T), q=q, kb=kb, vb=vb)


def cache_of(c):
    two = lambda a, first, other: u8(np.stack([a, np.full_like(a, other)] if first else [np.full_like(a, other), a])[:, None])
    unit = lambda a, first: f32(np.stack([a, a * 8] if first else [a * 8, a])[:, None])
    return das.PagedKVCache4(two(c["k"], True, 0), two(c["v"], False, 0), two(c["ks"], True, 0xff),
                             two(c["vs"], False, 0xff), unit(c["ku"], True), unit(c["vu"], False))


def assert_close(got, want, lse, l, dev, where=""):
    """An output is a mean of the values v_j with weights w_j (1 + d_j): off by sum w_j d_j (v_j - o) / sum w_j (1 + d_j),
    so by max |d| (1 + 2 max |d|) times the mean distance `dev` of the values from it, and by half a bf16 step.  d_j is the
    weight's rounding to bf16, 2^-8, and what binary32 leaves of its exponent: a score of up to 2^9 binary orders is off by
    2^-22 of itself in its sum, its product and its difference, 3 * 2^-13 in all, ln 2 of which is below 2^-11.  A weight
    below 2^-126 is lost, where one of the row's is 2^-61 or more: up to 2^14 keys' values, below 2^6 in size,
    lose 2^14 * 2^-65 * 2^6 = 2^-45 with them."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    d = 2.0 ** -8 + 2.0 ** -11
    off = d * (1 + 2 * d) * dev
    bound = off + half_ulp_bf16(np.abs(want) + off) + 2.0 ** -45
    err = np.abs(got - want)
    assert np.isfinite(got).all(), where
    assert np.all(err <= bound), f"{where}: {float((err / bound).max()):.3f} of the bound"
    lse, inf = np.asarray(lse, np.float64), np.isneginf(l)
    assert np.array_equal(np.isneginf(lse), inf) and np.abs(lse[~inf] - l[~inf]).max(initial=0.0) <= LSE_ABS, where


def reference(c, q, kb, vb, P, T, scale=None, masked=()):
    with np.errstate(invalid="ignore"):
        K, V = ref.keys(c["k"], c["ks"], c["ku"]), ref.values(c["v"], c["vs"], c["vu"])
    return ref.attention(K, V, c["table"], P, T, q, kb, vb, scale=scale, masked=masked)


def run_attention(c, scale=0.0, stream=None, status=0, masked=(), where="", repeat=1):
    cache = cache_of(c)
    B, Tm, Hq, D = c["q"].shape
    ws = das.new_workspace_paged4(cache, B, Hq, Tm)
    qd, kbd, vbd = (bf16(c[n]) for n in ("q", "kb", "vb"))
    torch.cuda.synchronize()
    for _ in range(repeat):
        out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 2, dev_i32(c["table"]), dev_i32(c["P"]),
                                                     dev_i32(c["T"]), qd, kbd, vbd, ws, softmax_scale=scale,
                                                     stream=stream)
    torch.cuda.synchronize()
    assert das.workspace_status(ws) == status
    Pc, Tc = np.clip(c["P"], 0, c["table"].shape[1] * PAGE), np.clip(c["T"], 0, Tm)
    o, l, dev = reference(c, f64(qd), f64(kbd), f64(vbd), Pc, Tc, scale=scale or None, masked=masked)
    assert_close(f64(out), o, lse.cpu().numpy(), l, dev, where=where)
    for b in range(B):
        assert not out[b, Tc[b]:].any() and torch.isneginf(lse[b, :, Tc[b]:]).all()
    return out, lse


SHAPES = [  # D, Hq, Hkv, max_block, prefix lengths, block lengths
    (64, 4, 4, 4, [256], [4]), (64, 1, 1, 1, [0], [1]), (64, 1, 1, 1, [1], [1]), (128, 1, 1, 1, [63], [1]),
    (128, 2, 2, 1, [64, 65], [1, 1]), (128, 8, 2, 16, [127, 0, 128], [16, 3, 0]), (128, 5, 1, 12, [1000], [11]),
    (64, 10, 2, 12, [129, 700], [12, 1]), (128, 32, 8, 8, [300, 64, 1, 449], [8, 7, 1, 0]),
    (128, 1, 1, 64, [190], [64]), (64, 8, 1, 8, [4097], [8]), (128, 32, 32, 1, [513], [1]),
    (128, 4, 4, 16, [2000, 5], [16, 16]), (128, 6, 2, 9, [320] * 5, [9, 8, 7, 6, 5]),
    (128, 4, 2, 16, [0] * 40, list(range(16)) * 2 + [16] * 8), (64, 2, 1, 32, list(range(0, 99, 3)), [32] * 33),
    (128, 16, 4, 4, [640, 64, 1], [4, 4, 4]), (128, 3, 1, 21, [777], [20]), (64, 64, 1, 1, [130, 3], [1, 0]),
    (128, 4, 1, 4, [12000], [4]), (64, 8, 1, 5, [9000, 130], [5, 2]), (128, 32, 8, 2, [190] * 60, [2] * 60)]


@pytest.mark.parametrize("shape", SHAPES, ids=[str(s)[:60] for s in SHAPES])
def test_attention_matches_64_bits(shape):
    D, Hq, Hkv, Tm, P, T = shape
    rng = np.random.default_rng(D + Hq + Tm + len(P))
    run_attention(attention_case(rng, D, Hq, Hkv, Tm, P, T), where=str(shape)[:60], repeat=2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tm", [1, 7, 16])
def test_attention_sharp_and_rising_scores(D, Tm):
    """Maxima that keep moving along the prefix, weights of one key near 1."""
    rng = np.random.default_rng(D + Tm)
    c = attention_case(rng, D, 4, 2, Tm, [1500, 700], [Tm, max(1, Tm - 1)])
    keep = c["ks"].copy()
    for b in range(2):                                      # scores grow page by page
        for t in range(-(-int(c["P"][b]) // PAGE)):
            pg = c["table"][b, t]
            c["ks"][pg] = np.where(keep[pg] == 0xff, 0xff, 8 * (9 + min(t, 6)))
    run_attention(c, scale=0.5, where="rising")
    c["ks"] = np.where(keep == 0xff, 0xff, 8 * 14).astype(np.uint8)
    run_attention(c, scale=1.0, where="sharp")


def test_attention_one_dominant_key_among_thousands():
    """What thousands of keys add beside one of 40 nats more is kept: the dominant key has no values, so that
    the output is the others' alone."""
    rng = np.random.default_rng(18)
    for gap in (12.0, 16.0, 40.0):
        D = 64
        c = attention_case(rng, D, 2, 1, 2, [4000], [2], poison=False)
        q = np.zeros((1, 2, 2, D))
        q[..., 0] = 1.0
        c["q"], c["kb"], c["vb"] = q, np.zeros_like(c["kb"]), np.zeros_like(c["vb"])
        c["kb"][..., 0] = -1000.0                             # the block's own keys have no weight
        c["ku"], c["vu"] = np.ones(1), np.ones(1)
        c["k"][:], c["ks"][:] = 0x88, 8 * 15                   # scores 0 but for one key, scale 1
        pg = c["table"][0, 7]
        c["k"][pg, 0, 5, 0] = 8 + 4 | 8 << 4                   # 4 in element 0
        c["v"][pg, 0, 0, :, 2] = c["v"][pg, 0, 0, :, 2] & 0x0f | 8 << 4   # token 5's values are 0
        cache = cache_of(c)
        ws = das.new_workspace_paged4(cache, 1, 2, 2)
        out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 2, dev_i32(c["table"]), dev_i32([4000]), dev_i32([2]),
                                                     bf16(c["q"]), bf16(c["kb"]), bf16(c["vb"]), ws,
                                                     softmax_scale=gap / 4)
        o, l, dev = reference(c, c["q"], c["kb"], c["vb"], [4000], [2], scale=gap / 4)
        assert np.abs(o).max() > 0
        assert_close(f64(out), o, lse.cpu().numpy(), l, dev, where=f"gap {gap}")


@pytest.mark.parametrize("Hq,Tm", [(1, 2), (4, 7), (8, 8)])
@pytest.mark.parametrize("gap", [8.0, 61.0, 63.0, 70.0, 140.0, 300.0])
def test_attention_steps_of_the_largest_score(Hq, Tm, gap):
    """Keys' scores are steps of `gap` binary orders: the first key's is 7 below 0, then come keys of 0, of 1 and of 2 steps
    within a tile and tiles later, so that the reference moves early, late, by a little or by more than a float's range, and
    what was summed before it still counts where the step is small.  Rows have scores of their own; values are as they come."""
    rng = np.random.default_rng(int(gap) + Tm)
    D = 64
    c = attention_case(rng, D, Hq, 1, Tm, [900, 300], [Tm, Tm - 1], poison=False)
    c["q"] = np.zeros_like(c["q"])
    c["q"][..., 0] = 1.0
    c["q"][:, :, -1, 0] = 0.25                                # (a row whose steps are a quarter)
    c["kb"] = np.zeros_like(c["kb"])
    c["kb"][..., 0] = -6.0
    c["ku"], c["k"][:], c["ks"][:] = np.ones(1), 0x88, 8 * 15   # scores 0, scale 1
    code = lambda x: 8 + x | 8 << 4
    for b, at in ((0, {0: -7, 100: 1, 500: 1, 501: 2, 700: 1}), (1, {0: -7, 1: -6, 290: 1})):
        for t, x in at.items():
            c["k"][c["table"][b, t // PAGE], 0, t % PAGE, 0] = code(x)
    if gap < 10:                                              # all keys within a few steps of one another
        for b in range(2):
            for t in range(int(c["P"][b])):
                c["k"][c["table"][b, t // PAGE], 0, t % PAGE, 0] = code(int(rng.integers(-7, 8)))
    run_attention(c, scale=gap * float(np.log(2)) / 7, where=f"gap {gap} first")
    run_attention(c, scale=gap * float(np.log(2)), where=f"gap {gap}")


def test_attention_scales_far_apart():
    """Scales from 2^-14 to 60 in one sequence, groups of zeros, queries whose rows differ by 2^40 in size."""
    rng = np.random.default_rng(8)
    c = attention_case(rng, 128, 4, 1, 8, [64 * 12 + 5], [8])
    pages = c["table"][0]
    for a, lo in (("ks", 30), ("vs", 0)):
        for i, pg in enumerate(pages[:12]):
            c[a][pg] = lo + 7 * (i % 12)
    c["vs"][pages[3]] = 0
    c["ks"][pages[5]] = 0
    run_attention(c, where="scales")
    c["q"][0, 3] *= 2.0 ** -40
    c["q"][0, 5] *= 2.0 ** 3
    run_attention(c, where="queries")


def test_attention_units():
    rng = np.random.default_rng(9)
    c = attention_case(rng, 64, 2, 2, 2, [100, 64], [0, 2])
    c["vu"] = np.array([2.0 ** -40, 2.0 ** -38])
    c["vb"] = c["vb"] * 2.0 ** -40
    run_attention(c, where="small values")
    c = attention_case(rng, 64, 2, 2, 2, [100, 164], [1, 2])
    c["ku"] = np.array([2.0 ** 3, 2.0 ** -30])
    c["vb"][:] = 0
    c["vu"] = np.array([2.0 ** -1, 2.0 ** -2])
    run_attention(c, scale=0.05, where="key units")


def test_attention_entries_that_are_no_pages_are_masked_and_flagged():
    rng = np.random.default_rng(10)
    for P in ([300, 200], [3000, 64]):
        c = attention_case(rng, 128, 4, 2, 4, P, [4, 4])
        c["table"][0, 2], c["table"][1, 0] = -1, 10 ** 9
        run_attention(c, status=4, masked={(0, 2), (1, 0)}, where="bad pages")
    c = attention_case(rng, 64, 2, 2, 1, [64, 100], [1, 1])
    c["table"][:] = -7                                      # the block alone is left
    run_attention(c, status=4, masked={(0, 0), (1, 0), (1, 1)}, where="no pages")


def test_attention_rows_without_keys():
    """No prefix and no block: nothing is seen."""
    rng = np.random.default_rng(11)
    c = attention_case(rng, 64, 4, 2, 3, [0, 70, 0], [0, 0, 2])
    run_attention(c, where="no keys")


def test_attention_nan_stays_with_its_rows():
    """A group that reads as NaN makes the rows that see it NaN, keys lse too, and no others."""
    rng = np.random.default_rng(15)
    for prefix in (70, 1500, 20000):
        for which in ("ks", "vs"):
            c = attention_case(rng, 64, 4, 2, 3, [prefix, 90], [3, 2], poison=False)
            at = (c["table"][0, 1], 1, 2, 1) if which == "ks" else (c["table"][0, 1], 1, 1, 2)
            c[which][at] = 0xff                               # sequence 0, kv head 1
            cache = cache_of(c)
            ws = das.new_workspace_paged4(cache, 2, 4, 3)
            out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 2, dev_i32(c["table"]), dev_i32(c["P"]),
                                                         dev_i32(c["T"]), bf16(c["q"]), bf16(c["kb"]), bf16(c["vb"]), ws)
            out, lse = f64(out), lse.cpu().numpy()
            bad = np.zeros(out.shape, bool)
            bad[0, :3, 2:, slice(None) if which == "ks" else slice(32, 64)] = True
            assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all()
            assert np.isfinite(lse[1, :, :2]).all() and np.isfinite(lse[0, :2]).all()
            assert np.isnan(lse[0, 2:]).all() if which == "ks" else np.isfinite(lse[0, 2:]).all()
            assert das.workspace_status(ws) == 0


def test_attention_lengths_that_change_between_calls():
    """Calls in a row on one workspace, each with lengths that the one before it did not have."""
    rng = np.random.default_rng(16)
    c = attention_case(rng, 128, 4, 2, 4, [2000, 900, 64], [4, 4, 4], poison=False)
    cache = cache_of(c)
    ws = das.new_workspace_paged4(cache, 3, 4, 4)
    q, kb, vb = (bf16(c[n]) for n in ("q", "kb", "vb"))
    table, P, T = dev_i32(c["table"]), dev_i32([0, 0, 0]), dev_i32([0, 0, 0])
    steps = [([2000, 900, 64], [4, 4, 4]), ([0, 0, 0], [1, 0, 4]), ([1, 899, 0], [2, 2, 2]), ([1999, 65, 63], [0, 0, 0]),
             ([640, 640, 64], [4, 1, 3])]
    new = [(dev_i32(p), dev_i32(t)) for p, t in steps]
    got = []
    torch.cuda.synchronize()
    for p, t in new:                                        # no host wait in between
        P.copy_(p)
        T.copy_(t)
        got.append(das.das_mature_v_attention_paged4(cache, 0, 1, 2, table, P, T, q, kb, vb, ws))
    for (p, t), (out, lse) in zip(steps, got):
        o, l, dev = reference(c, f64(q), f64(kb), f64(vb), p, t)
        assert_close(f64(out), o, lse.cpu().numpy(), l, dev, where=f"lengths {p}")
    assert das.workspace_status(ws) == 0


def test_attention_clamps_and_flags_lengths():
    rng = np.random.default_rng(11)
    c = attention_case(rng, 64, 2, 1, 4, [128, 64], [4, 4], rows=2, poison=False)
    c["P"], c["T"] = np.array([10 ** 9, -3]), np.array([9, -1])
    c["table"][1, 1] = 0
    run_attention(c, status=2, where="lengths")


def test_attention_on_another_stream_twice_and_in_wide_tables():
    rng = np.random.default_rng(12)
    c = attention_case(rng, 128, 8, 2, 8, [500, 70], [8, 5])
    a = run_attention(c, stream=torch.cuda.Stream())
    b = run_attention(c)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c["table"] = np.pad(c["table"], ((0, 0), (0, 1000)), constant_values=-9)
    b = run_attention(c)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_two_graphs_that_share_a_workspace():
    rng = np.random.default_rng(19)
    cases = [attention_case(rng, 128, 8, 2, 4, P, [4, 3]) for P in ([3000, 700], [64, 5000])]
    caches = [cache_of(c) for c in cases]
    ws = das.new_workspace_paged4(caches[0], 2, 8, 4)
    graphs, outs, args = [], [], []
    for c, cache in zip(cases, caches):
        a = [dev_i32(c[n]) for n in ("table", "P", "T")] + [bf16(c[n]) for n in ("q", "kb", "vb")]
        das.das_mature_v_attention_paged4(cache, 0, 1, 2, *a, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(das.das_mature_v_attention_paged4(cache, 0, 1, 2, *a, ws))
        graphs.append(g)
        args.append(a)
    for i in (0, 1, 1, 0, 1, 0):
        for o in outs[i]:
            o.fill_(float("nan"))
        graphs[i].replay()
        torch.cuda.synchronize()
        c, a = cases[i], args[i]
        o, l, dev = reference(c, *(f64(x) for x in a[3:]), c["P"], c["T"])
        assert_close(f64(outs[i][0]), o, outs[i][1].cpu().numpy(), l, dev, where=f"graph {i}")
    assert das.workspace_status(ws) == 0


@pytest.mark.parametrize("D,Hq,Hkv,Tm", [(64, 4, 2, 3), (128, 32, 4, 4)])
def test_attention_segments_of_every_number_of_tiles(D, Hq, Hkv, Tm):
    """Pairs of one tile to many, which the softmax groups begin in either order and of which one group may have none: both
    read both groups' sums in the end.  Runs repeat each other bit for bit."""
    rng = np.random.default_rng(D + Hq)
    P = [128 * n + int(rng.integers(0, 128)) for n in (0, 1, 2, 3, 4, 5, 0, 1, 0, 9, 2, 30, 0)] + [0, 0, 0]
    c = attention_case(rng, D, Hq, Hkv, Tm, P, [max(1, Tm - b % 2) for b in range(len(P))])
    first = run_attention(c)
    for _ in range(5):
        again = run_attention(c, repeat=20)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_attention_shapes_that_share_a_workspace():
    """One workspace of the largest size serves batches, heads, blocks and head sizes in turn: each call joins its segments,
    whatever the ones before it have left there."""
    rng = np.random.default_rng(20)
    shapes = [(128, 32, 8, 16, [rng.integers(1, 3000) for _ in range(16)]), (128, 8, 8, 1, [9000]), (64, 4, 2, 7, [4000, 0, 777]),
              (128, 64, 1, 1, [20000]), (64, 1, 1, 64, [64 * 150, 1])]
    cases, calls, size = [], [], 0
    for D, Hq, Hkv, Tm, P in shapes:
        c = attention_case(rng, D, Hq, Hkv, Tm, P, [max(1, Tm - b % 3) for b in range(len(P))], poison=False)
        cache = cache_of(c)
        size = max(size, das.new_workspace_paged4(cache, len(P), Hq, Tm).numel())
        cases.append((c, cache, [dev_i32(c[n]) for n in ("table", "P", "T")] + [bf16(c[n]) for n in ("q", "kb", "vb")]))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for i in (0, 1, 0, 2, 0, 3, 1, 4, 2, 0, 4, 3, 0):
        c, cache, args = cases[i]
        B, Tm, Hq, D = c["q"].shape
        out = torch.full((B, Tm, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((B, Hq, Tm), float("nan"), device="cuda")
        das.das_mature_v_attention_paged4(cache, 0, 1, 2, *args, ws, out=out, lse=lse)
        calls.append((i, out, lse))
    wants = [reference(c, *(f64(x) for x in args[3:]), c["P"], c["T"]) for c, _, args in cases]
    for at, (i, out, lse) in enumerate(calls):
        o, l, dev = wants[i]
        assert_close(f64(out), o, lse.cpu().numpy(), l, dev, where=f"call {at}, shape {i}")
    assert das.workspace_status(ws) == 0


def test_attention_graphs_of_two_batches_that_share_a_workspace():
    """A server's captured steps, one for each batch size, over one workspace."""
    rng = np.random.default_rng(21)
    c = attention_case(rng, 128, 8, 2, 4, [3000, 700, 1500, 64, 5000, 900], [4, 3, 4, 4, 1, 2], poison=False)
    cache = cache_of(c)
    ws = das.new_workspace_paged4(cache, 6, 8, 4)
    host_args = [c[n] for n in ("table", "P", "T", "q", "kb", "vb")]
    graphs, outs = {}, {}
    for B in (6, 1, 4):
        a = [dev_i32(x[:B]) for x in host_args[:3]] + [bf16(x[:B]) for x in host_args[3:]]
        das.das_mature_v_attention_paged4(cache, 0, 1, 2, *a, ws)
        torch.cuda.synchronize()
        graphs[B] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[B]):
            outs[B] = das.das_mature_v_attention_paged4(cache, 0, 1, 2, *a, ws) + (a,)
    o, l, dev = reference(c, *(f64(x) for x in outs[6][2][3:]), c["P"], c["T"])
    for B in (6, 1, 6, 4, 6, 6, 1, 4, 6):
        out, lse, _ = outs[B]
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graphs[B].replay()
        torch.cuda.synchronize()
        assert_close(f64(out), o[:B], lse.cpu().numpy(), l[:B], dev[:B], where=f"batch of {B}")
    assert das.workspace_status(ws) == 0


def test_attention_offsets_past_32_bits():
    """Pages whose codes lie more than 4 GiB into the cache, and commits to them."""
    rng = np.random.default_rng(13)
    D, H, P = 128, 8, 200
    pages = (5 << 30) // (H * PAGE * D // 2)
    cache = das.PagedKVCache4.empty(1, 1, pages, H, D)
    ids = [pages - 1, 3, pages - 7, pages // 2 + 1]
    new = bf16(rng.normal(0, 1, (2, 1, 1, 1, P, H, D)))
    flag = dev_i32([0])
    slots = [ids[t // PAGE] * PAGE + t % PAGE for t in range(P)]
    das.das_kv_append_paged4(cache, new[0], new[1], dev_i32(slots), dev_i32([0, P]), flag)
    part = [t[0, 0, ids].cpu().numpy() for t in (cache.k, cache.k_scale, cache.v, cache.v_scale)]
    zero = [np.zeros((1, 1) + a.shape, np.uint8) for a in part]
    one = np.ones((1, 1, H))
    want = ref.append(*zero, one, one, f64(new[0]), f64(new[1]), np.arange(P), [0, P])
    K, V = ref.keys(want[0][0, 0], want[1][0, 0], one[0, 0]), ref.values(want[2][0, 0], want[3][0, 0], one[0, 0])
    got_k, got_v = ref.keys(part[0], part[1], one[0, 0]), ref.values(part[2], part[3], one[0, 0])
    flat = lambda a: np.swapaxes(a, 1, 2).reshape(-1, H, D)[:P]
    assert flag.item() == 0 and np.array_equal(flat(got_k), flat(K)) and np.array_equal(flat(got_v), flat(V))
    ws = das.new_workspace_paged4(cache, 1, H, 4)
    q, kb, vb = (bf16(rng.normal(0, 1, (1, 4, H, D))) for _ in range(3))
    out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 1, dev_i32([ids]), dev_i32([P]), dev_i32([4]), q, kb, vb, ws)
    o, l, dev = ref.attention(K, V, np.array([[0, 1, 2, 3]]), [P], [4], f64(q), f64(kb), f64(vb))
    assert_close(f64(out), o, lse.cpu().numpy(), l, dev, where="far pages")


def test_attention_over_the_longest_table():
    """Prefixes of up to 2^31 - 64 tokens, all on one page: keys are 0 and values 1, so that weights are equal powers of two whose
    sums are exact (a segment has fewer than 2^24 keys), outputs 1 and the lse the logarithm of the number of keys seen."""
    D, rows = 64, (1 << 25) - 1
    z = lambda *s: np.zeros((1, 1, 1, 1) + s, np.uint8)
    one = 8 * 15                                            # the scale byte of 1
    cache = das.PagedKVCache4(u8(z(PAGE, D // 2) + 0x88), u8(z(8, D, 4) + 0x99), u8(z(PAGE, D // GROUP) + one),
                              u8(z(D // GROUP, PAGE) + one))
    ws = das.new_workspace_paged4(cache, 1, 2, 2)
    table = torch.zeros((1, rows), dtype=torch.int32, device="cuda")
    q = bf16(np.random.default_rng(22).normal(0, 1, (1, 2, 2, D)))
    kb, vb = bf16(np.zeros((1, 2, 1, D))), bf16(np.ones((1, 2, 1, D)))
    for P in (rows * PAGE, rows * PAGE - 64, 2 ** 31 - 127, 2 ** 31 - 300, 1 << 30):
        out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 1, table, dev_i32([P]), dev_i32([2]), q, kb, vb, ws)
        want = np.log(P + np.array([1.0, 2.0]))
        assert (out == 1).all() and np.abs(lse[0].cpu().numpy() - want).max() <= LSE_ABS, P
    assert das.workspace_status(ws) == 0


def test_attention_first_key_without_weight():
    """A key with a score of -inf at the head of a block, or of what a group of warps has of a prefix, while all others lie far
    below 0: the others are the row's weights.  Scores are of up to 2^9 binary orders, whose sum, product and difference are off
    by 3 * 2^-13 orders together (as in assert_close), and the lse is their size: 2^-11 more than for small ones."""
    rng = np.random.default_rng(23)

    def check(c, rows, where):
        B, Tm, Hq, _ = c["q"].shape
        cache = cache_of(c)
        ws = das.new_workspace_paged4(cache, B, Hq, Tm)
        out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 2, dev_i32(c["table"]), dev_i32(c["P"]), dev_i32(c["T"]),
                                                     bf16(c["q"]), bf16(c["kb"]), bf16(c["vb"]), ws, softmax_scale=1.0)
        with np.errstate(invalid="ignore"):
            o, l, dev = reference(c, *(f64(bf16(c[n])) for n in ("q", "kb", "vb")), c["P"], c["T"], scale=1.0)
        o, l, dev, out, lse = o[:, rows], l[..., rows], dev[:, rows], f64(out)[:, rows], lse.cpu().numpy()[..., rows]
        assert_close(out, o, l, l, dev, where=where)
        inf = np.isneginf(l)
        assert np.array_equal(np.isneginf(lse), inf) and np.abs(lse[~inf] - l[~inf]).max() <= LSE_ABS + 2.0 ** -11, where
        assert das.workspace_status(ws) == 0

    for D, Hq, Tm, T in ((64, 2, 5, 5), (128, 8, 8, 7)):
        c = attention_case(rng, D, Hq, 1, Tm, [0, 0], [T, T - 1], poison=False)
        c["q"][..., 0], c["q"][..., 1] = 1.0, 20.0
        c["kb"][..., 0], c["kb"][..., 1] = 0.0, -16.0          # scores about -320
        c["kb"][:, 0, 0, 0] = -np.inf
        check(c, slice(1, None), "block")                       # (the first row sees that key alone)
    for Hq, Tm in ((1, 1), (8, 8)):
        c = attention_case(rng, 64, Hq, 1, Tm, [900, 129], [Tm, Tm], poison=False)
        c["q"][..., 0], c["q"][..., 1] = -2.0 ** 126, 1.0
        c["kb"][..., 0], c["kb"][..., 1] = 0.0, -300.0
        c["ku"], c["ks"][..., 0], c["k"][..., :16] = np.ones(1), 0xa7, 0x88   # elements 0 to 31: scale 60, but for two 0
        c["k"][..., 0] = 3 << 4 | 8                             # elements 0 and 1: 0 and -5 steps, -300
        for b in range(2):
            for t in range(0, int(c["P"][b]), 128):             # the first key of every tile: 7 steps times -2^126
                c["k"][c["table"][b, t // PAGE], 0, t % PAGE, 0] = 3 << 4 | 15
        check(c, slice(None), "prefix")


def test_attention_block_values_past_the_units():
    """A value of the block's own whose quotient by a small unit is past bf16 counts as the most units that there are, or as
    infinite, to the rows that see it, one that is not finite as NaN, and either as nothing to the rows that do not."""
    rng = np.random.default_rng(24)
    for D, Hq, Tm, T, big in ((64, 2, 6, 6, 2.0 ** 100), (128, 8, 8, 7, -2.0 ** 89), (64, 1, 4, 4, np.inf)):
        c = attention_case(rng, D, Hq, 1, Tm, [140, 0], [T, T], poison=False)
        c["vu"] = np.array([2.0 ** -40])
        c["vb"] = c["vb"] * 2.0 ** -40
        clean = c["vb"].copy()
        c["vb"][:, 2, 0, 5] = big
        cache = cache_of(c)
        ws = das.new_workspace_paged4(cache, 2, Hq, Tm)
        out, lse = das.das_mature_v_attention_paged4(cache, 0, 1, 2, dev_i32(c["table"]), dev_i32(c["P"]), dev_i32(c["T"]),
                                                     bf16(c["q"]), bf16(c["kb"]), bf16(c["vb"]), ws)
        o, l, dev = reference(c, *(f64(bf16(x)) for x in (c["q"], c["kb"], clean)), c["P"], c["T"])
        out, bad = f64(out), np.zeros(o.shape, bool)
        bad[:, 2:T, :, 5] = True
        if np.isinf(big):
            assert np.isnan(out[bad]).all()
        else:                                               # (weights of the 150 keys are some thousandths or more)
            assert (out[bad] * np.sign(big) > 2.0 ** 70).all()
        # (values are of the size of 2^-40: what is lost of them is as much less)
        err = np.abs(np.where(bad, 0.0, out - o))
        off = (2.0 ** -8 + 2.0 ** -11) * (1 + 2.0 ** -6) * dev
        assert (err <= off + half_ulp_bf16(np.abs(o) + off) + 2.0 ** -85).all()
        assert np.abs(lse.cpu().numpy()[:, :, :T] - l[:, :, :T]).max() <= LSE_ABS
