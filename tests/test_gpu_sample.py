"""Sampling and sampled acceptance against a draw in whole numbers (tests/paged_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged_ref as ref
from tests.gpu_util import dev_i32

pytestmark = pytest.mark.gpu


def f32(x):
    return torch.tensor(np.asarray(x, dtype=np.float32)).cuda()


def e32(row, T):
    """The binary32 e_v of a row (torch on the GPU): 1 at the maximum, exp((l - m) / T) elsewhere."""
    x = torch.where(torch.isnan(row), -torch.inf, row)
    m = x.max()
    # a quotient by a tensor: one by a number may be taken as a product with its reciprocal
    e = torch.exp((x - m) / f32(min(float(T), 3.4028234e38))) if T > 0 else torch.zeros_like(x)
    e = torch.where(torch.isneginf(x), 0.0, e)
    return torch.where(x == m, 1.0, e).double().cpu().numpy()


def check(logits, u, T, k, p, min_p, draft=None):
    """logits [B][W][V] on the device; the parameters are lists of B."""
    B, W, V = logits.shape
    par = dict(temperature=f32(T), top_k=dev_i32(k), top_p=f32(p), min_p=f32(min_p))
    ids, logp = das.das_sample(logits, f32(u), **par)
    got, lp = ids.cpu().numpy(), logp.double().cpu().numpy()
    for b in range(B):
        Tb, pb, mb = float(np.float32(T[b])), float(np.float32(p[b])), float(np.float32(min_p[b]))
        for i in range(W):
            row = logits[b, i].float()
            e = e32(row, Tb)
            x = row.double().cpu().numpy()
            t, R, kept = ref.sample_row(x, e, Tb, k[b], pb, mb, np.float32(u[b][i]))
            assert got[b, i] == t, (b, i, got[b, i], t, kept.sum())
            if t < 0:
                assert lp[b, i] == -np.inf
            else:
                # binary32: a difference, a quotient, a logarithm and their sum, each within 2^-23 of its size
                z = (x[t] - np.nanmax(x)) / Tb if Tb > 0 and x[t] < np.nanmax(x) else 0.0
                want = z - np.log(R * 2.0 ** -32)
                assert abs(lp[b, i] - want) <= 2.0 ** -22 * (abs(z) + abs(np.log(R * 2.0 ** -32)) + 1)
    return ids, logp


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 1000, 4096, 5003, 40001])
def test_draws_match(V, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    B, W = 6, 2
    logits = (3 * torch.randn((B, W, V), generator=g, device="cuda")).to(dtype)
    u = torch.rand((B, W), generator=g, device="cuda").cpu().numpy()
    u[0, 0], u[1, 0] = 0.0, np.float32(1.0) - np.float32(2.0 ** -24)
    check(logits, u, [1.0, 0.7, 1.3, 0.0, 0.5, 2.0], [0, 50, 3, 0, V, 1], [1.0, 0.9, 0.5, 0.3, 0.95, 0.2],
          [0.0, 0.01, 0.0, 0.0, 0.2, 1.0])


@pytest.mark.parametrize("filters", [(0, 1.0, 0.0), (7, 1.0, 0.0), (0, 0.37, 0.0), (0, 0.9999, 0.0), (11, 0.37, 0.0),
                                     (0, 1.0, 0.6), (0, 1e-9, 0.0), (5, 0.999, 0.9)])
def test_many_equal_logits(filters):
    """Equal logits: the lowest indices stay, and the draw is exact."""
    rng = np.random.default_rng(1)
    V, B, W = 3001, 3, 4
    values = np.array([[0.0, 0.0, 0.0], [0.0, -0.0, -1.0], [2.0, 1.5, 1.0]])
    logits = f32(np.stack([rng.choice(values[b], (W, V)) for b in range(B)]))
    k, p, m = filters
    check(logits, rng.random((B, W)), [1.0, 0.5, 1.0], [k] * B, [p] * B, [m] * B)


def test_uniform_row_draws_the_index():
    V = 1000
    u = (np.arange(V) + 0.5) / V
    ids, logp = das.das_sample(torch.zeros((1, V, V), device="cuda"), f32(u[None]))
    assert ids[0].tolist() == list(range(V))
    assert (logp + np.log(V)).abs().max() < 1e-6 * np.log(V) + 1e-6


def test_infinities_and_nan():
    V, inf, nan = 200, np.inf, np.nan
    rows = np.full((7, V), -inf)
    rows[1, 17] = -3e38                       # one token alone
    rows[2, :] = nan                          # nothing
    rows[3, [3, 150]] = inf                   # two infinite ones
    rows[3, 7] = 5.0
    rows[4, ::2], rows[4, 1::2] = nan, 1.0    # NaN is masked
    rows[5, 10], rows[5, 20] = 3.4e38, -3.4e38
    rows[6, 5:9] = -1e-40                     # below the normal range
    for u in (0.0, 0.4, 0.999):
        for T, k, p, m in ((1.0, 0, 1.0, 0.0), (1e-30, 3, 0.9, 0.0), (1e30, 0, 0.5, 0.5), (0.0, 0, 1.0, 0.0)):
            check(f32(rows)[:, None], np.full((7, 1), u), [T] * 7, [k] * 7, [p] * 7, [m] * 7)


def test_parameters_out_of_range_mean_none():
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn((1, 5, 700), generator=g, device="cuda")
    u = torch.rand((1, 5), generator=g, device="cuda")
    want = das.das_sample(logits, u)
    for kw in (dict(top_k=dev_i32([-3])), dict(top_k=dev_i32([10 ** 9])), dict(top_p=f32([np.nan])),
               dict(top_p=f32([7.0])), dict(min_p=f32([-1.0])), dict(min_p=f32([np.nan])), dict(temperature=f32([1.0]))):
        got = das.das_sample(logits, u, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), kw
    first = logits.argmax(-1).int()
    for kw in (dict(temperature=f32([-1.0])), dict(temperature=f32([np.nan])), dict(top_p=f32([0.0])),
               dict(top_p=f32([-2.0])), dict(min_p=f32([5.0])), dict(top_k=dev_i32([1]))):
        assert torch.equal(das.das_sample(logits, u, **kw)[0], first), kw
    for bad in (-0.5, np.nan, 1.0, 7.0, -np.inf, np.inf):   # a random number out of range is clamped
        t = das.das_sample(logits, torch.full_like(u, bad), top_k=dev_i32([2]))[0]
        two = logits.topk(2, -1).indices
        assert torch.equal(t, (two.amax(-1) if bad >= 1 else two.amin(-1)).int())


def test_padded_rows_and_odd_addresses():
    g = torch.Generator(device="cuda").manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        whole = torch.randn((3, 2, 1031), generator=g, device="cuda").to(dtype)
        u = torch.rand((3, 2), generator=g, device="cuda")
        part = whole[..., 3:1030]
        want = das.das_sample(part.contiguous(), u, top_p=f32([0.8] * 3))
        got = das.das_sample(part, u, top_p=f32([0.8] * 3))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        one = das.das_sample(whole[1:2, 1:2, 1:], u[1:2, 1:2].contiguous())
        same = das.das_sample(whole[1:2, 1:2, 1:].contiguous(), u[1:2, 1:2].contiguous())
        assert torch.equal(one[0], same[0]) and torch.equal(one[1], same[1])


@pytest.mark.parametrize("B,W,V", [(1, 1, 50), (1, 8, 32000), (5, 3, 777), (9, 40, 65), (70, 2, 300)])
def test_acceptance(B, W, V):
    g = torch.Generator(device="cuda").manual_seed(B + W)
    logits = 2 * torch.randn((B, W, V), generator=g, device="cuda")
    u = torch.rand((B, W), generator=g, device="cuda")
    par = dict(temperature=f32([0.9] * B), top_k=dev_i32([40] * B))
    ids, logp = das.das_sample(logits, u, **par)
    draft = ids.clone()
    rng = np.random.default_rng(W)
    for b in range(B):
        if rng.random() < 0.7:
            draft[b, rng.integers(0, W)] ^= 1
    acc, tid, nxt, com, lp = das.das_sample_accept(logits, draft, u, **par)
    assert torch.equal(tid, ids) and torch.equal(lp, logp)
    same = (draft == ids).int().cumprod(1).sum(1).int()
    assert torch.equal(acc, same) and torch.equal(com, (same + 1).clamp(max=W))
    want = torch.where(same < W, ids.gather(1, same.clamp(max=W - 1).long()[:, None])[:, 0], draft[:, -1])
    assert torch.equal(nxt, want)


def test_acceptance_at_temperature_zero_is_greedy_acceptance():
    g = torch.Generator(device="cuda").manual_seed(4)
    logits = torch.randn((4, 6, 3000), generator=g, device="cuda").round(decimals=1)
    draft = logits.argmax(-1).int()
    draft[1, 3] += 1
    a, t, n = das.das_greedy_accept(logits, draft)
    acc, tid, nxt, _, lp = das.das_sample_accept(logits, draft, torch.rand((4, 6), device="cuda"), temperature=f32([0.0] * 4))
    assert torch.equal(a, acc) and torch.equal(t, tid) and torch.equal(n, nxt) and not lp.any()


def test_a_row_without_tokens_is_never_accepted():
    logits = torch.full((1, 2, 9), -torch.inf, device="cuda")
    acc, tid, nxt, com, lp = das.das_sample_accept(logits, dev_i32([[-1, -1]]), f32([[0.5, 0.5]]))
    assert acc.tolist() == [0] and tid.tolist() == [[-1, -1]] and nxt.tolist() == [-1] and com.tolist() == [1]


def test_draws_follow_the_distribution():
    """4096 draws over 8 tokens: counts within 5 standard deviations."""
    n = 4096
    row = f32([0.0, 1.0, -1.0, 2.0, 0.5, -2.0, 1.5, 0.2])
    g = torch.Generator(device="cuda").manual_seed(5)
    ids, _ = das.das_sample(row.expand(n // 1024, 1024, 8).contiguous(), torch.rand((n // 1024, 1024), generator=g, device="cuda"))
    prob = torch.softmax(row.double(), -1).cpu().numpy()
    got = np.bincount(ids.flatten().cpu().numpy(), minlength=8)
    assert np.all(np.abs(got - n * prob) <= 5 * np.sqrt(n * prob * (1 - prob)))


def test_another_stream():
    g = torch.Generator(device="cuda").manual_seed(6)
    logits, u = torch.randn((2, 2, 5000), generator=g, device="cuda"), torch.rand((2, 2), generator=g, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a = das.das_sample(logits, u, stream=s)
    s.synchronize()
    b = das.das_sample(logits, u)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("B,W,V,dtype", [(1, 1, 300001, torch.float32), (1, 2, 600007, torch.bfloat16),
                                         (1, 1, 262144, torch.float32), (40, 4, 70001, torch.bfloat16),
                                         (160, 1, 33000, torch.float32)])
def test_long_rows_and_many_rows(B, W, V, dtype):
    """Rows past what a cluster holds, rows of several CTAs, and more rows than SMs."""
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = (3 * torch.randn((B, W, V), generator=g, device="cuda")).to(dtype)
    u = torch.rand((B, W), generator=g, device="cuda")
    some = [0, B // 2, B - 1] if B > 2 else list(range(B))
    par = ([0.8] * B, [0, 900, 40][:1] * B, [0.9] * B, [0.0] * B)
    for k, p, m in ((0, 0.9, 0.0), (900, 0.95, 0.001), (40, 1.0, 0.0), (0, 1.0, 0.0)):
        kw = dict(temperature=f32([0.8] * B), top_k=dev_i32([k] * B), top_p=f32([p] * B), min_p=f32([m] * B))
        ids, logp = das.das_sample(logits, u, **kw)
        part, part_u = logits[some].contiguous(), u[some].contiguous().cpu().numpy()
        want = [[ref.sample_row(part[b, i].double().cpu().numpy(), e32(part[b, i].float(), float(np.float32(0.8))),
                                float(np.float32(0.8)), k, float(np.float32(p)), float(np.float32(m)),
                                part_u[b, i])[0] for i in range(W)] for b in range(len(some))]
        assert ids[some].tolist() == want, (k, p, m)


@pytest.mark.parametrize("kind", ["outlier", "lowest", "steps", "cluster", "half"])
@pytest.mark.parametrize("filters", [(0, 0.7, 0.0), (37, 1.0, 0.0), (2500, 0.9, 0.0), (600, 0.5, 0.1)])
def test_rows_that_crowd_one_bin(kind, filters):
    """Distributions that leave many distinct logits in one bin of the first histogram."""
    g = torch.Generator(device="cuda").manual_seed(7)
    V = 20011
    x = torch.randn((2, 3, V), generator=g, device="cuda")
    if kind == "outlier":
        x[..., 5] = 1e6
        x[1] *= 1e-3
    elif kind == "lowest":               # masked by the type's lowest value
        x[..., ::3] = torch.finfo(torch.float32).min
        x[1, :, 100:] = torch.finfo(torch.float32).min
    elif kind == "steps":                # a few values only, next to each other
        x = 1 + torch.randint(0, 300, x.shape, generator=g, device="cuda") * 2.0 ** -23
    elif kind == "cluster":
        x = 5 + x * 1e-5
    else:                                # one half of the vocabulary is masked
        x[..., : V // 2 + 7] = -torch.inf
    k, p, m = filters
    rng = np.random.default_rng(8)
    check(x.contiguous(), rng.random((2, 3)), [1.0, 0.3], [k, k], [p, p], [m, m])


@pytest.mark.parametrize("T", [float(np.nextafter(np.float32(2), np.float32(0))), 1e-19, 3e19, 1.0 / 3, 0.7 + 2 ** -24])
def test_temperatures_whose_quotients_round_awkwardly(T):
    g = torch.Generator(device="cuda").manual_seed(9)
    scale = min(max(T, 1e-19), 1e19)
    x = torch.randn((1, 8, 3001), generator=g, device="cuda") * 4 * scale
    u = np.random.default_rng(10).random((1, 8))
    check(x, u, [T], [0], [0.95], [0.0])
    check(x, u, [T], [300], [1.0], [0.0])


@pytest.mark.parametrize("V", [9001, 140003])
@pytest.mark.parametrize("kind", ["normal", "huge", "large", "small", "sliver", "around zero", "negative", "infinite"])
@pytest.mark.parametrize("filters", [(0, 0.6, 0.0), (2500, 1.0, 0.0), (1500, 0.9, 0.0), (0, 1e-9, 0.0), (7001, 0.9999, 0.1)])
def test_rows_of_16_bit_logits(V, kind, filters):
    """Few distinct values, below, in and above the range of 2^-8 to 2^8 in size."""
    g = torch.Generator(device="cuda").manual_seed(12)
    x = torch.randn((2, 1, V), generator=g, device="cuda")
    T = [1.0, 0.4]
    if kind == "huge":                   # past the range, of both signs
        x, T = x * 1e4, [3e3, 50.0]
    elif kind == "large":                # the largest is below 2^8, many are below -2^8
        x, T = (x * 100).clamp(max=255.0), [30.0, 5.0]
    elif kind == "small":                # all below 2^-8
        x, T = x * 1e-4, [1.0, 1e-5]
    elif kind == "sliver":               # a few values in the range, the others below it
        x = x * 2.0 ** -10
        x[..., 11::1000] += 0.5
    elif kind == "around zero":          # the threshold lies among logits below 2^-8
        x = torch.where(torch.rand(x.shape, generator=g, device="cuda") < 0.7, x * 1e-3, x)
    elif kind == "negative":
        x, T = x - 40, [2.0, 0.1]
    elif kind == "infinite":
        x[..., 5::200] = torch.inf
        x[1, :, ::3] = -torch.inf
    k, p, m = filters
    check(x.to(torch.bfloat16), np.random.default_rng(13).random((2, 1)), T, [k, k], [p, p], [m, m])


@pytest.mark.parametrize("V,dtype", [(360416, torch.float32), (360417, torch.float32), (524256, torch.bfloat16),
                                     (524257, torch.bfloat16), (400009, torch.float32)])
def test_rows_at_the_end_of_what_a_cluster_holds(V, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = (3 * torch.randn((1, 1, V), generator=g, device="cuda")).to(dtype)
    for k, p, m in ((0, 0.9, 0.0), (60, 0.95, 0.001), (0, 1.0, 0.0)):
        check(logits, np.array([[0.37]]), [0.8], [k], [p], [m])


def test_more_equal_logits_than_a_half_word_counts():
    """Every weight 2^32, and weights whose low halves are all ones, in one bin of a CTA."""
    V = 524256
    for x in (torch.zeros((1, 1, V), device="cuda"), torch.full((1, 1, V), -2.0, device="cuda")):
        x[0, 0, 7] = 0.0
        for dtype in (torch.bfloat16, torch.float32):
            y = x.to(dtype)[..., : V if dtype == torch.bfloat16 else 360416].contiguous()
            for T, k, p in ((1.0, 0, 0.6), (1.0, 400000 if dtype == torch.bfloat16 else 300000, 0.99), (3e8, 0, 0.5)):
                check(y, np.array([[0.77]]), [T], [k], [p], [0.0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C", [(1, 8), (19, 8), (25, 4), (40, 2)])
@pytest.mark.parametrize("k,p,values", [(512, 0.9, "distinct"), (450, 1.0, "ties"), (500, 0.7, "ties"), (512, 1.0, "distinct")])
def test_many_candidates_of_a_small_top_k(B, C, dtype, k, p, values):
    """Rows of C CTAs whose candidates are too many to be sorted: all tokens but 1025 to 2048 C are
    masked, most of the rest stand at the start of the slices, unevenly.  The same result every time."""
    g = torch.Generator(device="cuda").manual_seed(k + C)
    V = 40003 if dtype == torch.bfloat16 else 33001
    slice_ = (-(-V // C) + 3) // 4 * 4
    logits = torch.full((B, 1, V), -torch.inf, device="cuda")
    for r in range(C):
        n = min(1500 if r % 4 == 0 else 90 + 400 * (r % 3), slice_ // 2, V - r * slice_)
        x = 2 * torch.randn((B, n), generator=g, device="cuda")
        if values == "ties":             # the k-th largest is one of many equal ones
            x = x.round().clamp(max=1.0)
            x[:, ::17] += 3
        logits[:, 0, r * slice_: r * slice_ + n] = x
    logits[:, 0, V - 3:] = 0.5
    logits = logits.to(dtype)
    u = np.random.default_rng(k).random((B, 1))
    par = dict(temperature=f32([0.8] * B), top_k=dev_i32([k] * B), top_p=f32([p] * B))
    runs = [das.das_sample(logits, f32(u), **par) for _ in range(40)]
    for ids, logp in runs[1:]:
        assert torch.equal(ids, runs[0][0]) and torch.equal(logp, runs[0][1])
    some = sorted({0, B // 2, B - 1})
    n = len(some)
    ids, logp = check(logits[some].contiguous(), u[some], [0.8] * n, [k] * n, [p] * n, [0.0] * n)
    assert torch.equal(ids, runs[0][0][some]) and torch.equal(logp, runs[0][1][some])


def test_tensors_without_memory_are_refused():
    """Inside vmap a tensor has no address: an exception, with the interpreter as it was."""
    u = torch.rand((1, 2), device="cuda")
    with pytest.raises(RuntimeError, match="storage"):
        torch.vmap(lambda x: das.das_sample(x, u)[0])(torch.randn((3, 1, 2, 9), device="cuda"))
    ids, _ = das.das_sample(torch.randn((1, 2, 9), device="cuda"), u)
    assert ids.shape == (1, 2)


@pytest.mark.parametrize("B,W,V,dtype", [(9, 1, 33001, torch.float32), (19, 1, 70001, torch.bfloat16),
                                         (12, 2, 33001, torch.float32), (25, 3, 20003, torch.bfloat16),
                                         (100, 2, 9001, torch.float32), (2, 1, 363001, torch.float32),
                                         (3, 1, 530003, torch.bfloat16)])
def test_parameters_of_each_sequence(B, W, V, dtype):
    """Greedy, filtered and plain rows in one call, from eight CTAs a row to one, and past a cluster:
    tokens and log-probabilities of every eighth row, and of the first and last ones."""
    g = torch.Generator(device="cuda").manual_seed(V + B)
    logits = (3 * torch.randn((B, W, V), generator=g, device="cuda")).to(dtype)
    u = torch.rand((B, W), generator=g, device="cuda")
    kinds = [(1.0, 40, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.3, 700, 1.0, 0.02), (0.7, 5, 0.5, 0.1),
             (1.0, 0, 1.0, 0.0), (-1.0, 9, 0.3, 0.5), (2.0, 0, 1.0, 0.3), (0.9, V, 0.999, 0.0)]
    T, k, p, m = zip(*(kinds[b % len(kinds)] for b in range(B)))
    ids, logp = das.das_sample(logits, u, temperature=f32(T), top_k=dev_i32(k), top_p=f32(p), min_p=f32(m))
    some = sorted({0, B - 1, *range(0, B, 8), *range(min(B, 3))})
    pick = lambda x: [x[b] for b in some]
    part, part_u = logits[some].contiguous(), u[some].cpu().numpy()
    want = check(part, part_u, pick(T), pick(k), pick(p), pick(m))      # (a call of its own, of other CTAs a row)
    assert torch.equal(ids[some], want[0]) and torch.equal(logp[some], want[1])
