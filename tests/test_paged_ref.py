"""The paged-cache references on cases small enough to check by hand (no GPU)."""
import numpy as np

from tests import paged_ref as ref


def test_e4m3_rounds_to_nearest_even_and_saturates():
    assert ref.TABLE[126] == 448 and np.isnan(ref.TABLE[127])
    assert ref.TABLE[1] == 2.0 ** -9 and ref.TABLE[8] == 2.0 ** -6
    x = np.array([0.0, 1e9, -1e9, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -11])
    assert list(ref.TABLE[ref.to_e4m3(x)]) == [0, 448, -448, 16, 20, 0, 2.0 ** -8, 0]
    assert list(ref.to_e4m3(ref.TABLE[:127])) == list(range(127))


def test_scale_is_the_least_power_of_two():
    assert ref.scale_of(448.0) == 1 and ref.scale_of(449.0) == 2 and ref.scale_of(224.0) == 0.5
    assert ref.scale_of(0.0) == 2.0 ** -40 and ref.scale_of(3e38) == 2.0 ** 120


def test_page_assign_gives_back_then_takes():
    table = np.array([[0, 1, 9], [2, 9, 9]])
    n, t, free, count, slots, start, flag = ref.page_assign([100, 63], [-100, 3], table, [3], 1, 8)
    assert n == [0, 66] and list(t[1]) == [2, 1, 9] and free == [3, 0] and flag == 0
    assert slots == [2 * 64 + 63, 64, 65] and start == [0, 0, 3]


def test_sample_row_orders_filters():
    x = np.array([0.0, 1.0, 1.0, -np.inf])
    e = np.where(x == 1, 1.0, np.where(np.isinf(x), 0.0, 0.25))
    assert ref.sample_row(x, e, 1.0, 0, 1.0, 0.0, 0.999)[0] == 2
    assert ref.sample_row(x, e, 1.0, 0, 1.0, 0.0, 0.1)[0] == 0
    assert ref.sample_row(x, e, 1.0, 0, 0.4, 0.0, 0.999)[0] == 1   # one of the two equal ones is enough
    assert ref.sample_row(x, e, 0.0, 0, 1.0, 0.0, 0.999)[0] == 1
    assert ref.sample_row(np.full(3, -np.inf), x[:3], 1.0, 0, 1.0, 0.0, 0.5)[0] == -1


def test_attention_of_one_key_is_its_value():
    k = np.full((1, 1, 64, 64), 8, np.uint8)
    v = np.arange(64, dtype=np.uint8)[None, None, None, :].repeat(64, 2)
    s = np.ones((1, 1))
    q = np.ones((1, 1, 1, 64))
    out, lse = ref.attention(k, s, v, 2 * s, np.zeros((1, 1), int), [1], [1], q, q * -1e4, q, scale=1.0)
    assert np.allclose(out[0, 0, 0], 2 * ref.TABLE[:64]) and np.isclose(lse[0, 0, 0], 64 * 2.0 ** -6)
