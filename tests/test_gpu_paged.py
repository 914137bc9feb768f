"""Page assignment, the commit into the paged block-scaled cache and attention
over it, against plain references in 64 bits (tests/paged_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged_ref as ref
from tests.gpu_util import assert_close, dev_i32

pytestmark = pytest.mark.gpu
PAGE = 64


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


# ---- page assignment --------------------------------------------------------------

def random_pool(rng, B, rows, spare, max_len):
    """Lengths, a table and a free stack over disjoint pages; unused entries are garbage."""
    seq = rng.integers(0, min(max_len, rows * PAGE) + 1, B)
    have = -(-seq // PAGE)
    pages = int(have.sum()) + spare
    ids = rng.permutation(max(pages, 1))
    table = rng.integers(-5, 1 << 30, (B, rows))
    at = 0
    for b in range(B):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    free = np.full(max(pages, 1), -7)
    free[:spare] = ids[at:at + spare]
    return seq, table, free, spare


def check_assign(seq, grow, table, free, count, max_slots, in_place=False):
    want = ref.page_assign(seq, grow, table, free, count, max_slots)
    d = [dev_i32(x) for x in (seq, grow, table, free, [count])]
    slots = torch.full((max_slots,), 12345, dtype=torch.int32, device="cuda")
    flag = dev_i32([0])
    out = dict(new_len=d[0], new_free_count=d[4]) if in_place else {}
    for _ in range(1 if in_place else 2):   # with outputs apart the call can be repeated
        n, c, start = das.das_page_assign(d[0], d[1], d[2], d[3], d[4], slots, flag, **out)
    new_len, t, stack, cnt, sl, st, fl = want
    assert n.tolist() == new_len and c.tolist() == [cnt] and start.tolist() == st
    assert slots.tolist() == [int(x) for x in sl] + [-1] * (max_slots - len(sl))
    assert d[2].cpu().numpy().tolist() == t.tolist()
    assert d[3][:cnt].tolist() == [int(x) for x in stack]
    assert flag.item() == fl


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,rows,spare,max_len,max_grow,max_slots", [
    (1, 1, 1, 0, 64, 64), (1, 3, 0, 130, 2, 2), (3, 4, 2, 200, 80, 400), (16, 40, 20, 2000, 17, 300),
    (40, 9, 30, 500, 300, 3000), (300, 3, 5, 192, 40, 2000), (1500, 4, 700, 256, 90, 40000),
    (2050, 2, 2000, 128, 128, 65), (7, 100, 650, 0, 6400, 20000)])
def test_assign_matches_one_request_after_the_other(B, rows, spare, max_len, max_grow, max_slots, in_place):
    rng = np.random.default_rng(B * 7 + rows)
    seq, table, free, count = random_pool(rng, B, rows, spare, max_len)
    grow = rng.integers(-max_grow, max_grow + 1, B)
    grow[rng.random(B) < 0.15] = -(1 << 30)
    check_assign(seq, grow, table, free, count, max_slots, in_place)


def test_assign_no_request_and_no_growth():
    check_assign(np.zeros(0, int), np.zeros(0, int), np.zeros((0, 1), int), np.array([4, 3]), 2, 5)
    check_assign(np.array([64, 0, 1]), np.zeros(3, int), np.array([[0], [9], [1]]), np.array([2, 0]), 1, 0)


def test_assign_flags_values_out_of_range():
    table, free, flag = dev_i32([[0, 1], [2, 3]]), dev_i32([4, 5]), dev_i32([0])
    slots = dev_i32([0] * 8)
    n, c, start = das.das_page_assign(dev_i32([-5, 10 ** 9]), dev_i32([3, 1]), table, free, dev_i32([99]), slots, flag)
    # -5 counts as 0 tokens, 1e9 as the row's 128 (no room for another), 99 free pages as the pool's 2;
    # page 5 is none of those 2, so its tokens get no place
    assert n.tolist() == [3, 128] and c.tolist() == [1] and start.tolist() == [0, 3, 3]
    assert slots.tolist() == [-1] * 8
    assert flag.item() == 3
    flag.zero_()
    n, c, start = das.das_page_assign(dev_i32([-5, 10 ** 9]), dev_i32([3, 0]), table, dev_i32([1, 0]), dev_i32([99]),
                                      slots, flag)
    assert n.tolist() == [3, 128] and c.tolist() == [1] and start.tolist() == [0, 3, 3]
    assert slots.tolist() == [0, 1, 2] + [-1] * 5 and flag.item() == 2


# ---- commit -----------------------------------------------------------------------

def append_case(rng, R, L, H, D, first, n, W, N, amp=lambda b, t: 1.0):
    codes = rng.integers(0, 127, (R, L, N, H, PAGE, D)).astype(np.uint8)
    scales = 2.0 ** rng.integers(-12, 3, (R, L, N, H))
    B = len(n)
    x = rng.normal(0, 1, (R, L, B, W, H, D))
    for b in range(B):
        for t in range(W):
            x[:, :, b, t] *= amp(b, t)
    ids, slots, start = list(rng.permutation(N)), [], [0]
    for b in range(B):
        pg = [ids.pop() for _ in range(-(-(first[b] + n[b]) // PAGE))]
        slots += [pg[(first[b] + j) // PAGE] * PAGE + (first[b] + j) % PAGE for j in range(n[b])]
        start.append(len(slots))
    return codes, scales, x, slots, start


def run_append(codes, scales, x, slots, start, flag=None, repeat=1):
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()
    cache = das.PagedKVCache(dev(codes, torch.uint8), dev(codes[..., ::-1], torch.uint8),
                             dev(scales, torch.float32), dev(2 * scales, torch.float32))
    flag = dev_i32([0]) if flag is None else flag
    k, v = bf16(x), bf16(-3 * x)
    for _ in range(repeat):
        das.das_kv_append_paged(cache, k, v, dev_i32(slots if len(slots) else [0]), dev_i32(start), flag)
    return cache, f64(k), f64(v), flag


def same_codes(got, want):
    """Equal codes; a NaN may carry either sign."""
    got = got.cpu().numpy()
    nan = (want & 127) == 127
    return np.array_equal(got[~nan], want[~nan]) and np.all((got[nan] & 127) == 127)


@pytest.mark.parametrize("repeat", [1, 2])
@pytest.mark.parametrize("R,L,H,D,first,n,W", [
    (1, 1, 1, 64, [0], [1], 1), (2, 2, 3, 64, [5], [16], 16), (3, 1, 2, 128, [63, 0, 32], [1, 64, 33], 64),
    (1, 2, 8, 128, [10, 62], [200, 3], 201), (2, 1, 1, 128, [1, 0, 7], [0, 5, 0], 9), (1, 1, 5, 64, [33], [95], 95)])
def test_append_codes_and_scales(R, L, H, D, first, n, W, repeat):
    rng = np.random.default_rng(D + W + H)
    # later tokens of a sequence are larger, so that scales of started pages have to grow for some
    case = append_case(rng, R, L, H, D, first, n, W, 12, amp=lambda b, t: 2.0 ** (-6 + 9 * ((b + t) % 3)))
    codes, scales, x, slots, start = case
    cache, k, v, flag = run_append(*case, repeat=repeat)
    wk, wks = ref.append(codes, scales, k, slots, start)
    wv, wvs = ref.append(codes[..., ::-1], 2 * scales, v, slots, start)
    assert same_codes(cache.k, wk) and same_codes(cache.v, wv)
    assert np.array_equal(cache.k_scale.cpu().numpy(), wks) and np.array_equal(cache.v_scale.cpu().numpy(), wvs)
    assert flag.item() == 0


def test_append_extreme_values():
    rng = np.random.default_rng(3)
    codes, scales, x, slots, start = append_case(rng, 1, 1, 7, 64, [9], [20], 20, 2)
    x[..., 0, :] *= 0.0                                   # all zero: the least scale
    x[..., 1, :] *= 2.0 ** 100
    x[..., 2, :] *= 2.0 ** -60
    x[..., 3, 5] = np.inf
    x[..., 4, 6] = np.nan
    x[..., 5, :] = 448.0                                   # a scale of exactly 1
    x[..., 6, :] = np.sign(x[..., 6, :]) * np.inf
    scales[:, :, :, 2] = 2.0 ** -41                        # held scales below the least
    cache, k, v, flag = run_append(codes, scales, x, slots, start)
    wk, wks = ref.append(codes, scales, k, slots, start)
    assert same_codes(cache.k, wk) and np.array_equal(cache.k_scale.cpu().numpy(), wks)
    assert flag.item() == 0


def test_append_held_scales_that_are_no_powers_of_two():
    rng = np.random.default_rng(4)
    codes, scales, x, slots, start = append_case(rng, 1, 1, 4, 128, [30], [10], 10, 2)
    scales = np.float32(scales * rng.uniform(1, 2, scales.shape)).astype(np.float64)
    cache, k, _, _ = run_append(codes, scales, x, slots, start)
    wk, wks = ref.append(codes, scales, k, slots, start)
    assert np.array_equal(cache.k_scale.cpu().numpy().astype(np.float64), wks)
    # binary32 quotients differ from exact ones by 2^-24: only an exact half-way case could round apart
    assert (cache.k.cpu().numpy() != wk).mean() < 1e-3


def test_append_leaves_what_it_refuses():
    rng = np.random.default_rng(5)
    codes, scales, x, slots, start = append_case(rng, 1, 1, 2, 64, [60, 0, 0, 0], [8, 4, 4, 4], 8, 8)
    slots = list(slots)
    slots[start[0] + 4] += 1                               # a second page that does not start at its first place
    slots[start[1]:start[2]] = [-1] * 4                    # no place
    slots[start[2]:start[3]] = [8 * PAGE + i for i in range(4)]  # a page past the pool
    cache, k, _, flag = run_append(codes, scales, x, slots, start)
    wk, wks = ref.append(codes, scales, k[:, :, :1], slots[:4], [0, 4])
    last = start[3]
    wk, wks = ref.append(wk, wks, k[:, :, 3:], slots[last:], [0, 4])
    assert flag.item() == 2
    assert same_codes(cache.k, wk) and np.array_equal(cache.k_scale.cpu().numpy(), wks)
    # counts past W, and starts past the slots, write nothing
    for bad in ([0, 9, 9, 9, 9], [0, 0, 0, 0, 999], [4, 2, 2, 2, 2], [-3, -1, 0, 0, 0]):
        cache, k, _, flag = run_append(codes, scales, x, slots, bad)
        assert flag.item() == 2 and same_codes(cache.k, codes)


# ---- attention --------------------------------------------------------------------

def attention_case(rng, D, Hq, Hkv, Tm, P, T, rows=None, amp=1.0, poison=True):
    """A two-depth cache: keys read at depth 1, values at depth 2; what no call may use is NaN."""
    B = len(P)
    need = [-(-p // PAGE) for p in P]
    rows = max(1, max(need)) if rows is None else rows
    N = sum(need) + 2
    ids = rng.permutation(N)
    table = np.full((B, rows), -1)
    shape = (N, Hkv, PAGE, D)
    kc, vc = ref.to_e4m3(rng.normal(0, 60, shape)), ref.to_e4m3(rng.normal(0, 60, shape))
    ks, vs = (2.0 ** rng.integers(-8, -4, (N, Hkv)) for _ in range(2))
    ks = ks * amp
    at = 0
    used = np.zeros((N, PAGE), bool)
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        for t in range(need[b]):
            used[table[b, t], :min(PAGE, P[b] - t * PAGE)] = True
        at += need[b]
    if poison:
        for c in (kc, vc):
            c[np.broadcast_to(~used[:, None, :, None], shape)] = 0x7F
        ks[~used.any(1)] = np.nan
        vs[~used.any(1)] = np.nan
    f = lambda *s: rng.normal(0, 1, s)
    q, kb, vb = f(B, Tm, Hq, D), f(B, Tm, Hkv, D), f(B, Tm, Hkv, D)
    if poison:
        for b in range(B):
            q[b, T[b]:], kb[b, T[b]:], vb[b, T[b]:] = np.nan, np.nan, np.nan
    return kc, ks, vc, vs, table, np.array(P), np.array(T), q, kb, vb


def run_attention(kc, ks, vc, vs, table, P, T, q, kb, vb, scale=0.0, stream=None, status=0, masked=(), where=""):
    other = np.full_like(kc, 0x7F)                          # the depths that are not read: NaN
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()
    cache = das.PagedKVCache(dev(np.stack([kc, other])[:, None], torch.uint8),
                             dev(np.stack([other, vc])[:, None], torch.uint8),
                             dev(np.stack([ks, ks * np.nan])[:, None], torch.float32),
                             dev(np.stack([vs * np.nan, vs])[:, None], torch.float32))
    B, Tm, Hq, D = q.shape
    ws = das.new_workspace_paged(cache, B, Hq, Tm)
    qd, kbd, vbd = bf16(q), bf16(kb), bf16(vb)
    torch.cuda.synchronize()
    out, lse = das.das_mature_v_attention_paged(cache, 0, 1, 2, dev_i32(table), dev_i32(P), dev_i32(T), qd, kbd, vbd,
                                                ws, softmax_scale=scale, stream=stream)
    torch.cuda.synchronize()
    assert das.workspace_status(ws) == status
    Pc, Tc = np.clip(P, 0, table.shape[1] * PAGE), np.clip(T, 0, Tm)
    o, l = ref.attention(kc, np.float32(ks), vc, np.float32(vs), table, Pc, Tc, f64(qd), f64(kbd), f64(vbd),
                         scale=scale or None, masked=masked)
    assert_close(f64(out), o, lse.cpu().numpy(), l, where=where)
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
    (128, 16, 4, 4, [640, 64, 1], [4, 4, 4]), (128, 3, 1, 21, [777], [20]), (64, 64, 1, 1, [130, 3], [1, 0])]


@pytest.mark.parametrize("shape", SHAPES, ids=[str(s)[:60] for s in SHAPES])
def test_attention_matches_64_bits(shape):
    D, Hq, Hkv, Tm, P, T = shape
    rng = np.random.default_rng(D + Hq + Tm + len(P))
    run_attention(*attention_case(rng, D, Hq, Hkv, Tm, P, T), where=str(shape)[:60])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tm", [1, 7, 16])
def test_attention_sharp_and_rising_scores(D, Tm):
    """Maxima that keep moving along the prefix, weights of one key near 1."""
    rng = np.random.default_rng(D + Tm)
    c = list(attention_case(rng, D, 4, 2, Tm, [1500, 700], [Tm, max(1, Tm - 1)]))
    for b in range(2):                                      # scores grow page by page
        for t in range(-(-int(c[5][b]) // PAGE)):
            c[1][c[4][b, t]] = 2.0 ** (-9 + min(t, 6))
    run_attention(*c, scale=0.5, where="rising")
    c[1] = np.where(np.isnan(c[1]), c[1], 2.0 ** -6)
    run_attention(*c, scale=1.0, where="sharp")


def test_attention_scales_far_apart():
    """Value scales from 2^-40 to 2^30 in one sequence, scales that are no powers of two, zero pages."""
    rng = np.random.default_rng(8)
    c = list(attention_case(rng, 128, 4, 1, 8, [64 * 12 + 5], [8]))
    pages = c[4][0]
    c[3][pages, 0] = np.float32([1.0, 2.0 ** -40, 3.7e-3, 2.0 ** -20, 0.9, 1.1, 1e-6, 0.37, 0.01, 0.5, 2.0 ** -40, 0.3,
                                 0.77])
    c[1][pages, 0] = np.float32([2.0 ** -40, 0.011, 2.0 ** -8, 0.013, 1e-4, 2.0 ** -6, 0.02] + [0.015] * 6)
    c[2][pages[10], 0] = 0
    run_attention(*c, where="scales")
    big = list(c)
    big[3] = c[3] * 2.0 ** -3
    run_attention(*big, where="scales / 8")


def test_attention_only_small_values():
    """A sequence whose every page has the least scale."""
    rng = np.random.default_rng(9)
    c = list(attention_case(rng, 64, 2, 2, 2, [100, 64], [0, 2]))
    c[3] = np.where(np.isnan(c[3]), c[3], 2.0 ** -40)
    c[9] = c[9] * 2.0 ** -36
    run_attention(*c, where="small values")


def test_attention_entries_that_are_no_pages_are_masked_and_flagged():
    rng = np.random.default_rng(10)
    c = list(attention_case(rng, 128, 4, 2, 4, [300, 200], [4, 4]))
    c[4] = c[4].copy()
    c[4][0, 2], c[4][1, 0] = -1, 10 ** 9
    run_attention(*c, status=4, masked={(0, 2), (1, 0)}, where="bad pages")


def test_attention_nan_stays_with_its_rows():
    """A stored NaN makes the rows that see it NaN, lse too, and no others."""
    rng = np.random.default_rng(15)
    for prefix in (70, 1500):                               # one segment, and several joined
        c = list(attention_case(rng, 64, 4, 2, 3, [prefix, 90], [3, 2]))
        c[0] = c[0].copy()
        c[0][c[4][0, 1], 1, 2, 7] = 0x7F                    # sequence 0, kv head 1
        out, lse = run_attention_raw(*c)
        bad = np.zeros(out.shape[:3], bool)
        bad[0, :3, 2:] = True
        assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all()
        assert np.isnan(lse.transpose(0, 2, 1)[bad]).all()
        assert np.isfinite(lse[1, :, :2]).all() and np.isfinite(lse[0, :2]).all()


def run_attention_raw(kc, ks, vc, vs, table, P, T, q, kb, vb):
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()[None, None]
    cache = das.PagedKVCache(dev(kc, torch.uint8), dev(vc, torch.uint8), dev(ks, torch.float32), dev(vs, torch.float32))
    ws = das.new_workspace_paged(cache, q.shape[0], q.shape[2], q.shape[1])
    out, lse = das.das_mature_v_attention_paged(cache, 0, 1, 1, dev_i32(table), dev_i32(P), dev_i32(T), bf16(q), bf16(kb),
                                                bf16(vb), ws)
    return out.float().cpu().numpy(), lse.cpu().numpy()


def test_attention_lengths_that_change_between_calls():
    """Calls in a row on one workspace, each with lengths that the one before it did not have."""
    rng = np.random.default_rng(16)
    c = list(attention_case(rng, 128, 4, 2, 4, [2000, 900, 64], [4, 4, 4], poison=False))
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()[None, None]
    cache = das.PagedKVCache(dev(c[0], torch.uint8), dev(c[2], torch.uint8), dev(c[1], torch.float32),
                             dev(c[3], torch.float32))
    ws = das.new_workspace_paged(cache, 3, 4, 4)
    q, kb, vb = (bf16(x) for x in c[7:])
    table, P, T = dev_i32(c[4]), dev_i32([0, 0, 0]), dev_i32([0, 0, 0])
    steps = [([2000, 900, 64], [4, 4, 4]), ([0, 0, 0], [1, 0, 4]), ([1, 899, 0], [2, 2, 2]), ([1999, 65, 63], [0, 0, 0]),
             ([640, 640, 64], [4, 1, 3])]
    new = [(dev_i32(p), dev_i32(t)) for p, t in steps]
    got = []
    torch.cuda.synchronize()
    for p, t in new:                                        # no host wait in between
        P.copy_(p)
        T.copy_(t)
        got.append(das.das_mature_v_attention_paged(cache, 0, 1, 1, table, P, T, q, kb, vb, ws))
    for (p, t), (out, lse) in zip(steps, got):
        o, l = ref.attention(c[0], np.float32(c[1]), c[2], np.float32(c[3]), c[4], p, t, f64(q), f64(kb), f64(vb))
        assert_close(f64(out), o, lse.cpu().numpy(), l, where=f"lengths {p}")
    assert das.workspace_status(ws) == 0


def test_attention_clamps_and_flags_lengths():
    rng = np.random.default_rng(11)
    c = list(attention_case(rng, 64, 2, 1, 4, [128, 64], [4, 4], rows=2, poison=False))
    c[5], c[6] = np.array([10 ** 9, -3]), np.array([9, -1])
    run_attention(*c, status=2, where="lengths")


def test_attention_on_another_stream_and_twice():
    rng = np.random.default_rng(12)
    c = attention_case(rng, 128, 8, 2, 8, [500, 70], [8, 5])
    a = run_attention(*c, stream=torch.cuda.Stream())
    b = run_attention(*c)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_offsets_past_32_bits():
    """Pages whose codes lie more than 4 GiB into the cache."""
    rng = np.random.default_rng(13)
    D, H, P = 128, 8, 200
    pages = (5 << 30) // (H * PAGE * D)
    codes = torch.zeros((1, 1, pages, H, PAGE, D), dtype=torch.uint8, device="cuda")
    scales = torch.ones((1, 1, pages, H), device="cuda")
    ids = [pages - 1, 3, pages - 7, pages // 2 + 1]
    part = ref.to_e4m3(rng.normal(0, 60, (4, H, PAGE, D)))
    codes[0, 0, ids] = torch.from_numpy(part).cuda()
    scales[0, 0, ids] = 2.0 ** -6
    cache = das.PagedKVCache(codes, codes, scales, scales)
    ws = das.new_workspace_paged(cache, 1, H, 4)
    q, kb, vb = (bf16(rng.normal(0, 1, (1, 4, H, D))) for _ in range(3))
    out, lse = das.das_mature_v_attention_paged(cache, 0, 1, 1, dev_i32([ids]), dev_i32([P]), dev_i32([4]), q, kb, vb, ws)
    s = np.full((4, H), 2.0 ** -6)
    o, l = ref.attention(part, s, part, s, np.array([[0, 1, 2, 3]]), [P], [4], f64(q), f64(kb), f64(vb))
    assert_close(f64(out), o, lse.cpu().numpy(), l, where="far pages")
    # the commit reaches them too (keys and values are one tensor here, so both get the same tokens)
    flag = dev_i32([0])
    das.das_kv_append_paged(cache, vb[None, None], vb[None, None], dev_i32([ids[0] * PAGE + i for i in range(4)]),
                            dev_i32([0, 4]), flag)
    got = ref.TABLE[codes[0, 0, ids[0], :, :4].cpu().numpy()] * scales[0, 0, ids[0]].cpu().numpy()[:, None, None]
    assert flag.item() == 0 and np.abs(got - f64(vb)[0].transpose(1, 0, 2)).max() <= 4 * 2.0 ** -4


# ---- together ---------------------------------------------------------------------

def test_assign_append_attend():
    """Prompts and steps of ragged requests; one ends and its pages serve another."""
    rng = np.random.default_rng(14)
    D, H, Hq, B, N, rows, R = 64, 2, 4, 3, 16, 6, 2
    cache = das.PagedKVCache.empty(R, 1, N, H, D)
    cache.k.fill_(0x7F)
    cache.v.fill_(0x7F)
    table, free, count = dev_i32(np.full((B, rows), -1)), dev_i32(rng.permutation(N)), dev_i32([N])
    length, flag = dev_i32([0] * B), dev_i32([0])
    ws = das.new_workspace_paged(cache, B, Hq, 4)
    kept = [np.zeros((R, 2, 0, H, D)) for _ in range(B)]
    for grow in ([130, 64, 1], [1, 3, 16], [-500, 2, 60], [200, 1, -20], [5, 1, 1]):
        W = max(1, max(grow))
        slots = torch.empty(max(1, sum(max(g, 0) for g in grow)), dtype=torch.int32, device="cuda")
        _, _, start = das.das_page_assign(length, dev_i32(grow), table, free, count, slots, flag, new_len=length,
                                          new_free_count=count)
        kn, vn = (bf16(rng.normal(0, 1 + abs(grow[1]), (R, 1, B, W, H, D))) for _ in range(2))
        das.das_kv_append_paged(cache, kn, vn, slots, start, flag)
        for b, g in enumerate(grow):
            new = np.stack([f64(kn)[:, 0, b], f64(vn)[:, 0, b]], 1)[:, :, :max(g, 0)]
            kept[b] = np.concatenate([kept[b][:, :, :max(0, kept[b].shape[2] + min(g, 0))], new], 2)
        assert length.tolist() == [x.shape[2] for x in kept] and flag.item() == 0
        tb, P = table.cpu().numpy(), length.tolist()
        k, v, ks, vs = (t.cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))
        for b in range(B):      # stored values: within an e4m3 rounding of the page's largest scale
            for t in range(P[b]):
                pg = tb[b, t // PAGE]
                for which, (c, s) in enumerate(((k, ks), (v, vs))):
                    x = kept[b][:, which, t]
                    got = ref.TABLE[c[:, 0, pg, :, t % PAGE]] * s[:, 0, pg][..., None]
                    # one rounding to 4 bits, and one more for a code that a grown scale made subnormal
                    assert np.all(np.abs(got - x) <= np.abs(x) / 16 + s[:, 0, pg][..., None] * 2.0 ** -9)
        q, kb, vb = bf16(rng.normal(0, 1, (B, 4, Hq, D))), *(bf16(rng.normal(0, 1, (B, 4, H, D))) for _ in range(2))
        T = [4, 1, 2]
        out, lse = das.das_mature_v_attention_paged(cache, 0, 1, 2, table, length, dev_i32(T), q, kb, vb, ws)
        o, l = ref.attention(k[0, 0], ks[0, 0], v[1, 0], vs[1, 0], tb, P, T, f64(q), f64(kb), f64(vb))
        # values grow with the step: compare relative to the largest
        assert np.abs(f64(out) - o).max() <= 2.0 ** -7 * max(1.0, np.abs(o).max())
        fin = np.isfinite(l)
        assert np.abs(lse.cpu().numpy()[fin] - l[fin]).max() <= 1e-5 * max(10.0, np.abs(l[fin]).max())
    assert das.workspace_status(ws) == 0


@pytest.mark.parametrize("H,D,first,n,W", [(3, 128, [10, 62], [3, 60], 64), (5, 64, [33, 1], [80, 63], 100),
                                           (1, 64, [63, 9], [1, 15], 15), (2, 128, [40, 7], [64, 64], 64)])
@pytest.mark.parametrize("held", [1.5 * 2.0 ** 5, 1.5 * 2.0 ** -20])
def test_append_into_pages_with_other_scales(H, D, first, n, W, held):
    """Scales that are no powers of two, kept (large) and replaced (small); infinities among the
    new tokens, whose scale comes from the finite ones.  x / (1.5 2^j) is exact or lies a third
    of a bfloat16's last place off every tie, so the rounding through binary32 changes no code."""
    rng = np.random.default_rng(W + D)
    codes, scales, x, slots, start = append_case(rng, 1, 1, H, D, first, n, W, 6)
    scales[:] = held
    x[..., 0, 3] = np.inf
    cache, k, v, flag = run_append(codes, scales, x, slots, start)
    wk, wks = ref.append(codes, scales, k, slots, start)
    wv, wvs = ref.append(codes[..., ::-1], 2 * scales, v, slots, start)
    assert same_codes(cache.k, wk) and same_codes(cache.v, wv)
    assert np.array_equal(cache.k_scale.cpu().numpy(), wks) and np.array_equal(cache.v_scale.cpu().numpy(), wvs)
    assert flag.item() == 0


@pytest.mark.parametrize("shape", SHAPES, ids=[str(s)[:60] for s in SHAPES])
def test_attention_with_a_wide_table(shape):
    """Tables far wider than the prefixes, whose unused entries name no page: the pairs' tiles are
    then split as one list, where a narrow table has a pair's tiles shared by a cluster."""
    D, Hq, Hkv, Tm, P, T = shape
    rng = np.random.default_rng(D + Hq + Tm + len(P))
    case = list(attention_case(rng, D, Hq, Hkv, Tm, P, T))
    wide = np.full((len(P), 600), 10 ** 6, dtype=case[4].dtype)
    for b, n in enumerate(P):
        wide[b, :-(-n // PAGE)] = case[4][b, :-(-n // PAGE)]
    case[4] = wide
    run_attention(*case, where=str(shape)[:60])


@pytest.mark.parametrize("D,Hq,Hkv,Tm,P,T", [
    (128, 32, 32, 8, [1500], [8]), (128, 64, 16, 3, [1100], [2]), (64, 8, 8, 16, [2900], [16]),
    (128, 8, 4, 32, [2047], [31]), (64, 76, 76, 1, [640], [1]), (128, 2, 2, 64, [450, 3], [64, 1]),
    (128, 9, 3, 5, [0, 511, 64], [5, 0, 4])])
def test_attention_of_pairs_shared_by_clusters(D, Hq, Hkv, Tm, P, T):
    """One to several tiles a CTA, CTAs without any, rows of every number, and a row count that no
    cluster divides; the same result every time."""
    rng = np.random.default_rng(D + Hq + Tm)
    case = attention_case(rng, D, Hq, Hkv, Tm, P, T)
    out, lse = run_attention(*case, where="cluster")
    again, lse2 = run_attention(*case, where="cluster")
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def widen(case, columns=600):
    case = list(case)
    wide = np.full((case[4].shape[0], columns), 10 ** 6, dtype=case[4].dtype)
    wide[:, :case[4].shape[1]] = case[4]
    case[4] = wide
    return case


@pytest.mark.parametrize("Hkv", [2, 40])                    # joined by two warps a row, by one
def test_attention_nan_in_joined_segments(Hkv):
    rng = np.random.default_rng(17)
    c = list(attention_case(rng, 64, 2 * Hkv, Hkv, 3, [1500, 90], [3, 2]))
    c[0] = c[0].copy()
    c[0][c[4][0, 1], 1, 2, 7] = 0x7F                        # sequence 0, kv head 1
    out, lse = run_attention_raw(*widen(c))
    bad = np.zeros(out.shape[:3], bool)
    bad[0, :3, 2:4] = True
    assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all()
    bad_lse = bad.transpose(0, 2, 1)
    assert np.isnan(lse[bad_lse]).all() and np.isfinite(lse[0][~bad_lse[0]]).all()
    assert np.isfinite(lse[1, :, :2]).all() and np.isneginf(lse[1, :, 2]).all()


def test_attention_bad_pages_in_a_wide_table():
    rng = np.random.default_rng(10)
    c = widen(attention_case(rng, 128, 4, 2, 4, [300, 200], [4, 4]))
    c[4][0, 2], c[4][1, 0] = -1, 10 ** 9
    run_attention(*c, status=4, masked={(0, 2), (1, 0)}, where="bad pages")


@pytest.mark.parametrize("columns", [32, 600])
def test_attention_lengths_of_equal_sums_between_calls(columns):
    """Lengths that change while their sum stays, from call to call on one workspace."""
    rng = np.random.default_rng(18)
    c = widen(attention_case(rng, 128, 8, 4, 4, [1000, 1000], [4, 4], poison=False), columns)
    c[4][c[4] == 10 ** 6] = -1
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()[None, None]
    cache = das.PagedKVCache(dev(c[0], torch.uint8), dev(c[2], torch.uint8), dev(c[1], torch.float32),
                             dev(c[3], torch.float32))
    ws = das.new_workspace_paged(cache, 2, 8, 4)
    q, kb, vb = (bf16(x) for x in c[7:])
    table, P, T = dev_i32(c[4]), dev_i32([500, 500]), dev_i32([4, 4])
    steps = [[900, 100], [100, 900], [1000, 0], [0, 1000], [500, 500]]
    new = [dev_i32(p) for p in steps]
    torch.cuda.synchronize()
    got = []
    for p in new:                                           # no host wait in between
        P.copy_(p)
        got.append(das.das_mature_v_attention_paged(cache, 0, 1, 1, table, P, T, q, kb, vb, ws))
    for p, (out, lse) in zip(steps, got):
        o, l = ref.attention(c[0], np.float32(c[1]), c[2], np.float32(c[3]), c[4], p, [4, 4], f64(q), f64(kb), f64(vb))
        assert_close(f64(out), o, lse.cpu().numpy(), l, where=f"lengths {p}")
    assert das.workspace_status(ws) == 0


@pytest.mark.parametrize("D,Hq,Hkv,Tm,P,T", [
    (128, 16, 8, 3, [(37 * b) % 449 for b in range(20)], [b % 4 for b in range(20)]),
    (64, 8, 8, 2, [(29 * b) % 193 for b in range(40)], [1 + b % 2 for b in range(40)]),
    (128, 40, 40, 1, [0, 64, 65, 1, 0, 200], [1, 0, 1, 1, 1, 1])])
def test_attention_of_many_short_pairs(D, Hq, Hkv, Tm, P, T):
    """More pairs than SMs, few tiles to each: ranges of whole pairs, the same result every time and,
    to the rounding of a joined row, as with the equal ranges of a wide table."""
    rng = np.random.default_rng(D + Hq)
    case = attention_case(rng, D, Hq, Hkv, Tm, P, T)
    out, lse = run_attention(*case, where="short pairs")
    again, lse2 = run_attention(*case, where="short pairs")
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    run_attention(*widen(case), where="short pairs, wide table")


def test_attention_of_many_short_pairs_with_changing_lengths():
    rng = np.random.default_rng(19)
    B = 24
    c = list(attention_case(rng, 64, 8, 8, 2, [256] * B, [2] * B, poison=False))
    dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()[None, None]
    cache = das.PagedKVCache(dev(c[0], torch.uint8), dev(c[2], torch.uint8), dev(c[1], torch.float32),
                             dev(c[3], torch.float32))
    ws = das.new_workspace_paged(cache, B, 8, 2)
    q, kb, vb = (bf16(x) for x in c[7:])
    table, P, T = dev_i32(c[4]), dev_i32([256] * B), dev_i32([2] * B)
    steps = [[256] * B, [0] * B, [(b * 31) % 257 for b in range(B)], [256 - (b * 31) % 257 for b in range(B)]]
    new = [dev_i32(p) for p in steps]
    torch.cuda.synchronize()
    got = []
    for p in new:                                           # no host wait in between
        P.copy_(p)
        got.append(das.das_mature_v_attention_paged(cache, 0, 1, 1, table, P, T, q, kb, vb, ws))
    for p, (out, lse) in zip(steps, got):
        o, l = ref.attention(c[0], np.float32(c[1]), c[2], np.float32(c[3]), c[4], p, [2] * B, f64(q), f64(kb), f64(vb))
        assert_close(f64(out), o, lse.cpu().numpy(), l, where="lengths")
    assert das.workspace_status(ws) == 0


def sink_case(rng, D, Hq, Hkv, Tm, P, T, gap, sinks):
    """One key, or one of each page, whose score lies about `gap` above those of all others (deviation
    0.3), with values of 0; the others' values have mean 0.5.  The output is then the others' share."""
    kc, ks, vc, vs, table, P, T, q, kb, vb = attention_case(rng, D, Hq, Hkv, Tm, P, T)
    used, pages = kc != 0x7F, np.unique(table[table >= 0])
    sigma = 0.3 * 2.0 ** 4
    k, v = rng.normal(0, sigma, kc.shape), rng.normal(0.5, 0.2, vc.shape) * 2.0 ** 6
    k[..., 0] = 0                                           # a dimension of the sinks alone
    ks[pages], vs[pages] = 2.0 ** -4, 2.0 ** -6
    first = table[:, 0] if sinks == "first" else pages
    k[first, :, 0, :], v[first, :, 0, :] = 0, 0
    k[first, :, 0, 0] = 256.0
    q[..., 0] = np.where(np.isnan(q[..., 0]), np.nan, gap * np.sqrt(D) / 16.0)
    kb[..., 0], vb = np.where(np.isnan(kb[..., 0]), np.nan, -4.0), vb * 0.0
    return (np.where(used, ref.to_e4m3(k), kc), ks, np.where(vc != 0x7F, ref.to_e4m3(v), vc), vs, table, P, T, q, kb, vb)


@pytest.mark.parametrize("gap", [12.0, 16.0])
@pytest.mark.parametrize("D,Hq,Hkv,Tm,P,sinks,columns", [
    (128, 4, 2, 4, [32768], "first", 513), (128, 4, 2, 16, [8000, 3000], "pages", 600),
    (64, 16, 1, 4, [5000], "pages", 600),                   # equal ranges and a merge
    (128, 8, 8, 8, [4096], "pages", 64), (128, 8, 2, 8, [2500], "pages", 40),
    (64, 4, 4, 1, [3000], "pages", 47), (128, 2, 2, 64, [1500], "pages", 24),  # clusters
    (128, 8, 8, 2, [190] * 25, "pages", 3), (64, 32, 8, 16, [250, 128, 100, 64] * 6, "pages", 4)])  # whole pairs
def test_attention_keeps_small_weights(D, Hq, Hkv, Tm, P, sinks, columns, gap):
    """Thousands of keys of weight e^-gap beside one of weight 1: their share is kept."""
    rng = np.random.default_rng(D + Hq + int(gap))
    case = list(sink_case(rng, D, Hq, Hkv, Tm, P, [Tm] * len(P), gap, sinks))
    if columns > case[4].shape[1]:
        case = widen(case, columns)
    out, lse = run_attention(*case, where=f"sinks, gap {gap}")
    assert float(out[0, 0].float().abs().max()) > 0


def test_a_step_without_requests():
    """Empty tensors through every call of a step that takes them, and requests without new tokens."""
    H, D, N = 2, 64, 3
    cache = das.PagedKVCache.empty(2, 1, N, H, D)
    cache.k.fill_(7)
    free, count, flag = dev_i32(range(N)), dev_i32([N]), dev_i32([0])
    f32, none = torch.float32, lambda dtype, *s: torch.empty(s, dtype=dtype, device="cuda")
    out = das.das_sample_accept(none(f32, 0, 3, 50), none(torch.int32, 0, 3), none(f32, 0, 3), temperature=none(f32, 0))
    assert [x.shape[0] for x in out] == [0] * 5
    ids, logp = das.das_sample(none(torch.bfloat16, 0, 3, 50), none(f32, 0, 3))
    assert ids.shape == logp.shape == (0, 3)
    empty = none(torch.int32, 0)
    n, c, start = das.das_page_assign(empty, out[3], none(torch.int32, 0, 4), free, count, empty, flag)
    assert n.shape == (0,) and c.item() == N and start.tolist() == [0]
    das.das_kv_append_paged(cache, none(torch.bfloat16, 2, 1, 0, 3, H, D), none(torch.bfloat16, 2, 1, 0, 3, H, D), empty,
                            start, flag)
    # two requests, none of which has committed a token: there are no slots
    new = bf16(np.ones((2, 1, 2, 3, H, D)))
    das.das_kv_append_paged(cache, new, new, empty, dev_i32([0, 0, 0]), flag)
    assert flag.item() == 0 and bool((cache.k == 7).all())
    das.das_kv_append_paged(cache, new, new, empty, dev_i32([0, 1, 1]), flag)   # a token without a slot is flagged
    assert flag.item() == 2 and bool((cache.k == 7).all())


@pytest.mark.parametrize("gap", [10.3, 12.9, 14.1, 15.2, 15.556, 15.645])
def test_attention_rounds_equal_small_weights(gap):
    """As above with equal scores beside the sinks', whose weights are rounded alike: off by up to 0.6 %
    (2^-30 of a page's sum, beside e^-15.7 of it), and the output by up to 0.4 % more."""
    rng = np.random.default_rng(int(10 * gap))
    case = list(sink_case(rng, 128, 8, 2, 8, [1500, 700], [8, 3], gap, "pages"))
    used = (case[0] != 0x7F) & (ref.TABLE[case[0]][..., :1] == 0)       # all keys but the sinks
    case[0] = np.where(used, 0, case[0])
    run_attention(*case, where=f"equal, gap {gap}")
    run_attention(*widen(case), where=f"equal, gap {gap}, wide table")
