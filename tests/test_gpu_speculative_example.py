"""The speculative example: norm and rotation, attention over the 4-bit cache, acceptance, pages and the commit together,
on ragged sequences that end at different steps."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2609_34538_gb300 as das
from tests import paged4_ref as ref
from tests.test_gpu_paged4 import assert_close, f64

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_speculative.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_speculative", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("W", [1, 4, 7])
def test_decoding_keeps_its_books(example, W):
    prompts, new = [list(range(3, 3 + n)) for n in (5, 130, 1, 64)], [70, 9, 40, 1]
    tokens, dec, accepts = example.decode(prompts, new, W=W)
    assert [len(t) for t in tokens] == new
    assert all(0 <= t < dec.model.vocab for row in tokens for t in row)
    assert all(0 <= a <= W for a in accepts) and any(accepts)
    # every sequence has ended: all pages are free, each once
    assert dec.length.tolist() == [0] * 4 and dec.free_count.item() == dec.free.numel()
    assert sorted(dec.free.tolist()) == list(range(dec.free.numel()))
    assert dec.flag.item() == 0 and das.workspace_status(dec.ws) == 0


def test_the_same_numbers_give_the_same_tokens(example):
    run = lambda seed: example.decode([[1, 2, 3], [9] * 70], [30, 30], seed=seed)[0]
    assert run(3) == run(3) and run(3) != run(4)


@pytest.mark.parametrize("head_dim", [64, 128])
def test_a_step_against_the_formulas(example, head_dim):
    """The first layer of a step, over a cache that prompts have filled at every depth: what attention gave of the projection's
    rows, against norm, rotation and attention in 64 bits over what the commits have to have stored."""
    model = example.LoopedModel(head_dim=head_dim, seed=2)
    prompts, W = [list(range(n)) for n in (70, 3, 149)], 5
    dec = example.Decoder(model, 3, pages=9, max_pages=3, block=16)
    fresh = []
    store = dec.store
    dec.store = lambda k, v, n: (fresh.append((f64(k), f64(v), n.tolist())), store(k, v, n))
    anchor = dec.prefill(prompts)
    n = torch.tensor([W, W - 2, W], dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, 512, (3, W), dtype=torch.int32, device="cuda")
    tokens[:, 0] = anchor
    seen = {}
    attend = dec.attend(n)
    def look(layer, depth, q, k, v):
        out = attend(layer, depth, q, k, v)
        seen.setdefault((layer, depth), [x.clone() for x in (q, k, v, out)])
        return out
    model.forward(tokens, dec.length, n, look)
    # the cache, of the tokens that were stored in turn
    zero = [np.zeros(t.shape, np.uint8) for t in (dec.cache.k, dec.cache.k_scale, dec.cache.v, dec.cache.v_scale)]
    one, table, at = np.ones(zero[0].shape[:2] + zero[0].shape[3:4]), dec.table.tolist(), [0, 0, 0]
    for k, v, grow in fresh:
        slots, start = [], [0]
        for b, g in enumerate(grow):
            slots += [table[b][t // 64] * 64 + t % 64 for t in range(at[b], at[b] + g)]
            at[b] += g
            start.append(len(slots))
        zero = ref.append(*zero, one, one, k, v, slots, start)
    assert at == [len(p) - 1 for p in prompts] == dec.length.tolist()
    for b in range(3):
        for j in range(-(-at[b] // 64)):
            live = min(64, at[b] - 64 * j)
            assert np.array_equal(dec.cache.k[:, :, table[b][j], :, :live].cpu().numpy(), zero[0][:, :, table[b][j], :, :live])
    # the rows of the first layer
    rows = f64((model.E[tokens.long()] @ model.Wqkv[0]).to(torch.bfloat16).view(3, W, -1, head_dim))
    place = np.array(at)[:, None] + np.arange(W)
    angle = ref.angles(place, model.inv_freq.cpu().numpy())
    q, k, v, out = seen[0, 1]
    live = np.arange(W)[None] < n.cpu().numpy()[:, None]
    for got, x, w in ((q, rows[:, :, :8], model.q_norm[0]), (k, rows[:, :, 8:10], model.k_norm[0])):
        want, size = ref.norm_rope(x, f64(w), 1e-6, angle, False)
        assert (np.abs(f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 3e-6 * size)[live].all()
    assert np.array_equal(f64(v)[live], rows[:, :, 10:][live])
    K, V = ref.keys(zero[0][0, 0], zero[1][0, 0], one[0, 0]), ref.values(zero[2][0, 0], zero[3][0, 0], one[0, 0])
    clean = lambda x: np.where(live[..., None, None], f64(x), 0.0)
    o, l, dev = ref.attention(K, V, np.array(table), np.array(at), n.cpu().numpy(), clean(q), clean(k), clean(v))
    lse = np.where(np.isneginf(l), -np.inf, l)
    assert_close(f64(out), o, lse, l, dev)
    assert dec.flag.item() == 0 and das.workspace_status(dec.ws) == 0
