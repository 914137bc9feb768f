"""Speculative acceptance against a plain reference in whole numbers (tests/paged4_ref.py)."""
import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged4_ref as ref
from tests.gpu_util import dev_i32

pytestmark = pytest.mark.gpu


def weights(logits, T):
    """The binary32 e_v of rows [..., V] at a temperature, as float64."""
    z = torch.where(logits.isnan(), -torch.inf, logits.float()) + 0.0
    m = z.max(-1, keepdim=True).values
    T = torch.tensor(T if T > 0 else 1.0, dtype=torch.float32, device=z.device)
    e = torch.where(z == m, 1.0, torch.exp((z - m) / T))
    return torch.where(z.isneginf(), 0.0, e).cpu().numpy().astype(np.float64)


def check(target, drafter, ids, u, again, params, draft_params=None, **more):
    """params, draft_params: lists of (T, k, p, min_p) per sequence."""
    B, W, V = target.shape
    col = lambda ps, i, dt: None if ps is None else torch.tensor([x[i] for x in ps], dtype=dt, device="cuda")
    kinds = (torch.float32, torch.int32, torch.float32, torch.float32)
    accepted, nxt, committed = das.das_speculative_accept(
        target, drafter, ids, u, again, *(col(params, i, k) for i, k in enumerate(kinds)),
        *(col(draft_params, i, k) for i, k in enumerate(kinds)), **more)
    torch.cuda.synchronize()
    t, d = (x.float().cpu().numpy().astype(np.float64) for x in (target, drafter))
    iu, ia, ii = u.cpu().numpy(), again.cpu().numpy(), ids.cpu().numpy()
    got = list(zip(accepted.tolist(), nxt.tolist(), committed.tolist()))
    for b in range(B):
        tp, dp = params[b], (draft_params or params)[b]
        f = lambda x, lg, ps: [ref.probabilities(x[b, i], lg[i], *(ps[0], ps[1], np.float32(ps[2]), np.float32(ps[3])))
                               for i in range(W)]
        a, n = ref.speculative(f(t, weights(target[b], np.float32(tp[0])), tp), f(d, weights(drafter[b], np.float32(dp[0])), dp),
                               ii[b], iu[b], ia[b])
        assert got[b] == (a, n, min(a + 1, W)), (b, got[b], a, n)
    return accepted, nxt, committed


def make(seed, B, W, V, dtype, near=0.5, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    target = spread * torch.randn((B, W, V), generator=g, device="cuda")
    drafter = (target + near * torch.randn((B, W, V), generator=g, device="cuda")).to(dtype)
    u = torch.rand((3, B, W), generator=g, device="cuda")
    return target.to(dtype), drafter, u[0].contiguous(), u[1, :, 0].contiguous(), u[2].contiguous()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V,params", [
    (1, 1, 1, (1.0, 0, 1.0, 0.0)), (3, 2, 7, (0.7, 0, 1.0, 0.0)), (4, 8, 1000, (1.0, 0, 0.9, 0.0)),
    (2, 33, 517, (0.8, 20, 0.95, 0.02)), (2, 4, 32000, (1.0, 0, 0.95, 0.0)), (3, 3, 32001, (0.6, 200, 1.0, 0.0)),
    (2, 2, 40000, (1.3, 1500, 0.99, 0.001)), (3, 5, 300, (0.0, 0, 1.0, 0.0)), (2, 3, 5000, (1.0, 1, 1.0, 0.0)),
    (1, 2, 128257, (1.0, 0, 0.9, 0.0)), (40, 3, 257, (0.9, 0, 1.0, 0.05))])
def test_matches_whole_numbers(B, W, V, params, dtype):
    target, drafter, u, again, u0 = make(V + W, B, W, V, dtype)
    full = lambda x, dt: torch.full((B,), x, dtype=dt, device="cuda")
    ids, _ = das.das_sample(drafter, u0, full(params[0], torch.float32), full(params[1], torch.int32),
                            full(params[2], torch.float32), full(params[3], torch.float32))
    check(target, drafter, ids, u, again, [params] * B)


def test_parameters_of_each_sequence_and_of_the_drafter():
    params = [(0.5, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 5, 1.0, 0.0), (1.5, 0, 0.3, 0.0), (1.0, 0, 1.0, 0.3),
              (float("nan"), 3, float("nan"), float("nan")), (1.0, -2, 2.0, -1.0)]
    draft = [(1.0, 0, 1.0, 0.0)] * 3 + [(0.0, 0, 1.0, 0.0)] + [(2.0, 40, 0.9, 0.0)] * 3
    target, drafter, u, again, _ = make(5, 7, 4, 333, torch.float32)
    ids = torch.randint(0, 333, (7, 4), device="cuda", dtype=torch.int32)
    ids[:, 0] = drafter[:, 0].argmax(-1).int()
    clean = [tuple(0.0 if x != x and i != 2 else 1.0 if x != x else x for i, x in enumerate(p)) for p in params]
    got = check(target, drafter, ids, u, again, clean, draft)
    col = lambda ps, i, dt: torch.tensor([x[i] for x in ps], dtype=dt, device="cuda")
    kinds = (torch.float32, torch.int32, torch.float32, torch.float32)
    raw = das.das_speculative_accept(target, drafter, ids, u, again, *(col(params, i, k) for i, k in enumerate(kinds)),
                                     *(col(draft, i, k) for i, k in enumerate(kinds)))
    assert all(torch.equal(a, b) for a, b in zip(got, raw))   # NaN parameters: as documented for das_sample


def test_ids_outside_the_vocabulary_and_numbers_outside_the_range():
    target, drafter, u, again, _ = make(6, 4, 3, 50, torch.float32)
    ids = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    ids[0, 0], ids[1, 0], ids[2, 1] = -1, 50, 2 ** 31 - 1
    u[3] = torch.tensor([-1.0, float("nan"), 2.0])
    accepted, nxt, committed = das.das_speculative_accept(target, drafter, ids, u, again)
    assert accepted.tolist()[:2] == [0, 0] and accepted[2] <= 1 and ((nxt >= 0) & (nxt < 50)).all()
    assert accepted[3] <= 1                                  # NaN accepts nothing
    for x in (float("nan"), -3.0, 1.0, 5.0):
        n = das.das_speculative_accept(target, drafter, torch.full_like(ids, -1), u, torch.full((4,), x, device="cuda"))[1]
        assert ((n >= 0) & (n < 50)).all()


def test_rows_without_logits_infinities_and_equal_rows():
    target, drafter, u, again, _ = make(7, 6, 2, 40, torch.float32)
    target[0, 0] = -torch.inf                                # nothing to draw from
    drafter[1, 0] = torch.nan                                # the drafter had nothing: p > 0 accepts
    target[2, 0, 3] = target[2, 0, 9] = torch.inf            # both with half of the weight
    drafter[3, 0, 5] = torch.inf
    drafter[4] = target[4]                                    # the same distribution: accepted
    target[5, 0, :20] = torch.nan
    ids = torch.tensor([[1, 2], [3, 4], [3, 1], [5, 6], [7, 8], [30, 2]], dtype=torch.int32, device="cuda")
    accepted, nxt, committed = das.das_speculative_accept(target, drafter, ids, u, again)
    assert accepted[0] == 0 and nxt[0] == -1 and committed[0] == 1
    assert accepted[1] >= 1 and accepted[4] == 2 and nxt[4] == 8 and committed[4] == 2
    assert accepted[2] > 0 or nxt[2].item() in (3, 9)
    if accepted[5] == 0:
        assert nxt[5] >= 20
    sure = torch.zeros_like(u) + 0.999999
    refused = das.das_speculative_accept(target, drafter, torch.full_like(ids, 39), sure, again)
    assert refused[1][2].item() in (3, 9)                     # the target's row 2 has weight at these alone


def test_padded_and_unaligned_rows_and_given_outputs():
    B, W, V = 3, 4, 1003
    target, drafter, u, again, u0 = make(8, B, W, V, torch.bfloat16)
    ids, _ = das.das_sample(drafter, u0)
    want = check(target, drafter, ids, u, again, [(1.0, 0, 1.0, 0.0)] * B)
    pad = lambda x, n: torch.cat([x, torch.full((B, W, n), 99.0, dtype=x.dtype, device="cuda")], -1)[..., :V]
    outs = [torch.full((B,), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
    got = das.das_speculative_accept(pad(target, 5), pad(drafter, 2), ids, u, again, accepted=outs[0],
                                     next_token=outs[1], committed=outs[2])
    assert all(a is b for a, b in zip(got, outs)) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_longest_rows():
    """Rows past a cluster's shared memory, which a CTA each reads from memory."""
    target, drafter, u, again, u0 = make(9, 2, 2, 400009, torch.float32)
    ids, _ = das.das_sample(drafter, u0)
    check(target, drafter, ids, u, again, [(1.0, 0, 1.0, 0.0), (0.8, 50, 0.95, 0.0)])


def test_first_tokens_follow_the_target():
    """Of 40000 sequences with one proposal each, what is emitted is distributed as the target: a token's count is
    within 5 standard deviations (60 tokens: one in 30000 runs would not be)."""
    B, V = 40000, 60
    g = torch.Generator(device="cuda").manual_seed(10)
    target, drafter = (1.5 * torch.randn(V, generator=g, device="cuda") for _ in range(2))
    u = torch.rand((3, B, 1), generator=g, device="cuda")
    rows = lambda x: x.expand(B, 1, V).contiguous()
    ids, _ = das.das_sample(rows(drafter), u[0])
    accepted, nxt, _ = das.das_speculative_accept(rows(target), rows(drafter), ids, u[1], u[2, :, 0].contiguous())
    emitted = torch.where(accepted > 0, ids[:, 0], nxt)
    p = torch.softmax(target.double(), 0)
    n = torch.bincount(emitted, minlength=V).double()
    assert ((n - B * p).abs() <= 5 * torch.sqrt(B * p * (1 - p)) + 1).all()
    q = torch.softmax(drafter.double(), 0)
    mean = torch.minimum(p, q).sum()
    assert abs(accepted.double().mean() - mean) <= 5 * torch.sqrt(mean * (1 - mean) / B)


def test_empty_batch_other_stream_and_graph():
    target, drafter, u, again, u0 = make(11, 3, 4, 5000, torch.bfloat16)
    ids, _ = das.das_sample(drafter, u0)
    e = das.das_speculative_accept(target[:0], drafter[:0], ids[:0], u[:0], again[:0])
    assert [x.shape[0] for x in e] == [0, 0, 0]
    want = das.das_speculative_accept(target, drafter, ids, u, again)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = das.das_speculative_accept(target, drafter, ids, u, again, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = das.das_speculative_accept(target, drafter, ids, u, again)
    for _ in range(3):
        again.copy_(torch.rand(3, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = das.das_speculative_accept(target, drafter, ids, u, again)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [900, 33000, 70001])
def test_ties_at_the_cut(V, dtype):
    """Few different logits: top-k and top-p end among thousands of equal ones, and proposals are drawn of them."""
    B, W = 6, 3
    g = torch.Generator(device="cuda").manual_seed(V)
    target, drafter = (torch.randint(-3, 3, (B, W, V), generator=g, device="cuda").float().div(2).to(dtype) for _ in range(2))
    target[3:], drafter[3:] = target[3:] / 64 * 0, 0.0        # all equal, -0 among them
    target[4, :, ::2] = -0.0
    u, again, u0 = (torch.rand(s, generator=g, device="cuda") for s in ((B, W), (B,), (B, W)))
    for params in ((1.0, 300, 1.0, 0.0), (0.7, 300, 0.6, 0.0), (1.0, 0, 0.35, 0.0), (1.0, 700, 0.9, 0.2), (1.3, 0, 0.99, 0.1),
                   (1.0, 0, 1.0, 0.6)):
        full = lambda i, dt: torch.full((B,), params[i], dtype=dt, device="cuda")
        ids, _ = das.das_sample(drafter, u0, full(0, torch.float32), full(1, torch.int32), full(2, torch.float32),
                                full(3, torch.float32))
        check(target, drafter, ids, u, again, [params] * B)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_candidates_of_every_number(dtype):
    """Numbers of the largest logits around what is sorted (512) and listed (2048 to a part of the row), with equal ones among
    them and few others near; infinite ones among and beside them."""
    V = 20000
    for n, k in ((500, 400), (513, 500), (600, 512), (2040, 512), (2100, 512), (9000, 512), (30, 511)):
        g = torch.Generator(device="cuda").manual_seed(n)
        target = torch.randn((2, 2, V), generator=g, device="cuda") - 20
        where = torch.randperm(V, generator=g, device="cuda")[:n]
        target[:, :, where] = torch.randint(0, 8, (2, 2, n), generator=g, device="cuda").float() / 4
        target[1, 1, where[::3]] = torch.inf
        drafter = target.roll(1, -1)
        u, again, u0 = (torch.rand(s, generator=g, device="cuda") for s in ((2, 2), (2,), (2, 2)))
        for params in ((1.0, k, 1.0, 0.0), (0.9, k, 0.7, 0.3)):
            full = lambda i, dt: torch.full((2,), params[i], dtype=dt, device="cuda")
            ids, _ = das.das_sample(drafter.to(dtype), u0, full(0, torch.float32), full(1, torch.int32),
                                    full(2, torch.float32), full(3, torch.float32))
            check(target.to(dtype), drafter.to(dtype), ids, u, again, [params] * 2)


def test_the_largest_logits_and_temperatures():
    """Temperatures whose quotients go the plain way, logits past the counted bins, rows of one logit above -inf."""
    target, drafter, u, again, u0 = make(12, 5, 2, 3000, torch.bfloat16, spread=300.0)
    target[4, :, 1:], drafter[4, :, :-1] = -torch.inf, -torch.inf
    params = [(1e-30, 0, 0.9, 0.0), (1e25, 0, 0.9, 0.0), (float(np.float32(1.9999999)), 0, 0.9, 0.0), (300.0, 50, 0.9, 0.01),
              (1.0, 10, 0.9, 0.1)]
    ids = torch.stack([drafter[b].float().argmax(-1) for b in range(5)]).int()
    check(target, drafter, ids, u, again, params)


def test_two_streams_at_once():
    """Calls that run beside each other share nothing."""
    cases = [make(13 + i, 4, 4, 32000, torch.float32) for i in range(2)]
    ids = [das.das_sample(c[1], c[4])[0] for c in cases]
    want = [das.das_speculative_accept(*c[:2], i, *c[2:4], top_k=torch.full((4,), 100, dtype=torch.int32, device="cuda"))
            for c, i in zip(cases, ids)]
    k = torch.full((4,), 100, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, (c, s) in enumerate(zip(cases, streams)):
            got[i].append(das.das_speculative_accept(*c[:2], ids[i], *c[2:4], top_k=k, stream=s))
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        assert all(torch.equal(a, b) for r in runs for a, b in zip(w, r))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 9001, 40003])
def test_nan_and_infinities_among_the_logits(V, dtype):
    """NaN counts as -inf wherever it stands, whole groups and ends of rows among them, and -0 as 0."""
    target, drafter, u, again, u0 = make(14 + V, 4, 3, V, dtype)
    g = torch.Generator(device="cuda").manual_seed(V)
    for x in (target, drafter):
        some = torch.rand(x.shape, generator=g, device="cuda")
        x[some < 0.2], x[some > 0.9] = torch.nan, -torch.inf
        x[(some > 0.5) & (some < 0.55)] = -0.0
        x[..., :9], x[..., -7:] = torch.nan, torch.nan
        x[2, :, 20:40] = torch.nan
    target[3, :, 12:45:4] = torch.inf
    for params in ((0.9, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 40, 0.95, 0.01)):
        full = lambda i, dt: torch.full((4,), params[i], dtype=dt, device="cuda")
        ids, _ = das.das_sample(drafter, u0, full(0, torch.float32), full(1, torch.int32), full(2, torch.float32),
                                full(3, torch.float32))
        check(target, drafter, ids, u, again, [params] * 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 3001, 40003, 128257])
def test_refused_between_equal_rows(V, dtype):
    """A proposal that is no token, where drafter and target are the same: nothing is left of the target beside the drafter's,
    to the last bit, and the draw is das_sample's from the target's row."""
    B, W = 6, 2
    target, _, u, again, _ = make(20 + V, B, W, V, dtype)
    target[3] = target[3].round()                             # many equal logits
    target[4, :, ::3], target[4, :, 5] = torch.nan, -torch.inf
    target[5, :, 7:9] = torch.inf
    ids = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    for params in ((1.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (0.9, 30, 0.95, 0.01), (1.0, 1200, 1.0, 0.0),
                   (0.0, 0, 1.0, 0.0)):
        check(target, target.clone(), ids, u, again, [params] * B)
        full = lambda i, dt: torch.full((B,), params[i], dtype=dt, device="cuda")
        sampling = full(0, torch.float32), full(1, torch.int32), full(2, torch.float32), full(3, torch.float32)
        drawn, _ = das.das_sample(target[:, :1], again[:, None], *sampling)
        accepted, nxt, _ = das.das_speculative_accept(target, target, ids, u, again, *sampling)
        assert not accepted.any() and torch.equal(nxt, drawn[:, 0])


def test_refused_between_equal_longest_rows():
    target, _, u, again, _ = make(21, 2, 1, 400009, torch.float32)
    ids = torch.full((2, 1), -1, dtype=torch.int32, device="cuda")
    check(target, target, ids, u, again, [(1.0, 0, 1.0, 0.0), (0.8, 500, 0.95, 0.0)])


@pytest.mark.parametrize("V", [40, 40003])
def test_refused_at_rows_without_logits_and_with_infinities(V):
    """Refusals that are certain (no token's number is -1), of every kind of row, alone in a CTA and over a cluster."""
    target, drafter, u, again, _ = make(22, 6, 2, V, torch.float32)
    drafter[0, 0] = torch.nan                                 # the drafter had nothing
    target[1, 0, 3] = target[1, 0, V - 1] = torch.inf         # both with half of the weight
    drafter[2, 0, 5] = torch.inf
    target[3, 0, :V // 2] = torch.nan
    drafter[4, 0, V // 3:] = -torch.inf
    target[5, 0, 1:] = -torch.inf                             # one token alone
    ids = torch.full((6, 2), -1, dtype=torch.int32, device="cuda")
    for params in ((1.0, 0, 1.0, 0.0), (0.8, 12, 0.9, 0.02)):
        accepted, nxt, _ = check(target, drafter, ids, u, again, [params] * 6)
        assert not accepted.any() and nxt[1].item() in (3, V - 1) and nxt[3] >= V // 2 and nxt[5] == 0
    target[0, 0] = -torch.inf                                 # nothing to draw from, and from neither
    target[1, 0], drafter[1, 0] = torch.nan, torch.nan
    accepted, nxt, committed = das.das_speculative_accept(target, drafter, ids, u, again)
    assert nxt[:2].tolist() == [-1, -1] and accepted[:2].tolist() == [0, 0] and committed[:2].tolist() == [1, 1]
