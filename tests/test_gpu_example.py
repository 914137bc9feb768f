"""The paged sampling example: the calls together, on ragged sequences that end at different steps."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_sampling.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_sampling", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("W", [1, 4, 7])
def test_decoding_keeps_its_books(example, W):
    import paper_2609_34538_gb300 as das
    prompts, new = [list(range(3, 3 + n)) for n in (5, 130, 1, 64)], [70, 9, 40, 1]
    tokens, logprobs, dec, accepts = example.decode(prompts, new, W=W)
    assert [len(t) for t in tokens] == new and [len(l) for l in logprobs] == new
    assert all(0 <= t < dec.model.vocab for row in tokens for t in row)
    assert all(l <= 0 for row in logprobs for l in row)
    assert all(0 <= a <= W for a in accepts)
    # every sequence has ended: all pages are free, each once
    assert dec.length.tolist() == [0] * 4 and dec.free_count.item() == dec.free.numel()
    assert sorted(dec.free.tolist()) == list(range(dec.free.numel()))
    assert dec.flag.item() == 0 and das.workspace_status(dec.ws) == 0


def test_the_same_numbers_give_the_same_tokens(example):
    a = example.decode([[1, 2, 3], [9] * 70], [30, 30], seed=3)
    b = example.decode([[1, 2, 3], [9] * 70], [30, 30], seed=3)
    assert a[0] == b[0] and a[1] == b[1]
    assert a[0] != example.decode([[1, 2, 3], [9] * 70], [30, 30], seed=4)[0]


def test_a_sequence_does_not_depend_on_its_neighbours(example):
    """Greedy decoding of one sequence alone and beside others (other pages, the same numbers)."""
    model = example.LoopedModel(seed=5)
    alone = example.decode([[7, 8, 9]], [25], W=2, temperature=0.0, model=model)[0][0]
    beside = example.decode([[4] * 100, [7, 8, 9], [1]], [3, 25, 60], W=2, temperature=0.0, model=model)[0][1]
    # products of other batch sizes round apart, so that a near tie may part the continuations later
    assert alone[:3] == beside[:3]
