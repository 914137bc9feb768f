"""The references of the 4-bit cache against each other and against hand-made values, on the CPU."""
import numpy as np

from tests import paged4_ref as ref


def test_scale_bytes():
    assert ref.SCALES[0] == 0 and ref.SCALES[1] == 2.0 ** -17 and ref.SCALES[8] == 2.0 ** -14
    assert ref.SCALES[0xa7] == 60 and np.isnan(ref.SCALES[0xff])
    for b in range(256):
        f16 = np.array([b << 7], dtype=np.uint16).view(np.float16)[0]
        assert np.float64(f16) == ref.SCALES[b] or np.isnan(f16) and np.isnan(ref.SCALES[b])


def test_quantised_values_are_near():
    rng = np.random.default_rng(0)
    x = rng.normal(0, 1, (50, 128)) * 2.0 ** rng.integers(-6, 6, (50, 1))
    c, s = ref.quantise(x, 0.5)
    y = (c.astype(np.float64) - 8) * np.repeat(ref.SCALES[s], 32, -1) * 0.5
    m = np.abs(x.reshape(50, 4, 32)).max(-1)
    # half a step of a scale that is at most 1/16 off m / 7, and the largest may be clipped by 1/16
    assert np.all(np.abs(y - x) <= np.repeat(m, 32, -1) * (17 / 16 / 14) + 1e-12)


def test_hand_made_groups():
    x = np.zeros((6, 32))
    x[1, 3], x[1, 4], x[1, 5], x[1, 6] = 7.0, 2.5, -3.5, 0.5      # scale 1: ties go to even
    x[2, 0], x[2, 1] = 1e9, -1.0                                    # saturated: scale 60
    x[3, 0], x[3, 1] = np.nan, 7.0
    x[4, 0], x[4, 1] = -np.inf, 7.0
    x[5, 0] = 2.0 ** -30                                            # below half the least scale
    c, s = ref.quantise(x, 1.0)
    assert s[:, 0].tolist() == [0, 120, 0xa7, 0xff, 120, 0] and ref.SCALES[120] == 1
    assert c[0].tolist() == [8] * 32 and c[1, 3:7].tolist() == [15, 10, 4, 8]
    assert c[2, :2].tolist() == [15, 8] and c[3, :2].tolist() == [8, 15] and c[4, :2].tolist() == [1, 15]
    assert c[5].tolist() == [8] * 32


def test_append_and_decode_meet():
    rng = np.random.default_rng(1)
    z = lambda *s: rng.integers(0, 256, s).astype(np.uint8)
    k, ks, v, vs = z(1, 1, 2, 1, 64, 32), z(1, 1, 2, 1, 64, 2), z(1, 1, 2, 1, 8, 64, 4), z(1, 1, 2, 1, 2, 64)
    kn, vn, one = rng.normal(0, 1, (1, 1, 1, 5, 1, 64)), rng.normal(0, 1, (1, 1, 1, 5, 1, 64)), np.ones((1, 1, 1))
    slots = [64 + 61, 64 + 62, 64 + 63, 0, 1]
    k2, ks2, v2, vs2 = ref.append(k, ks, v, vs, one, one, kn, vn, slots, [0, 5])
    got_k, got_v = ref.keys(k2, ks2, one[0, 0]), ref.values(v2, vs2, one[0, 0])
    for j, s in enumerate(slots):
        c, b = ref.quantise(kn[0, 0, 0, j, 0], 1.0)
        assert np.array_equal(got_k[0, 0, s // 64, 0, s % 64], (c - 8.0) * np.repeat(ref.SCALES[b], 32))
        c, b = ref.quantise(vn[0, 0, 0, j, 0], 1.0)
        assert np.array_equal(got_v[0, 0, s // 64, 0, s % 64], (c - 8.0) * np.repeat(ref.SCALES[b], 32))
    same = np.ones(128, bool)
    same[slots] = False
    old, new = (ref.values(a, np.full_like(vs, 120), one[0, 0])[0, 0, :, 0].reshape(128, 64) for a in (v, v2))
    assert np.array_equal(old[same], new[same])


def test_rotation_keeps_sizes_and_turns():
    x = np.random.default_rng(2).normal(0, 1, (1, 3, 2, 64))
    freq = np.float32(10000.0 ** (-np.arange(16) / 16))
    a = ref.angles(np.array([[0, 1, 1 << 30]]), freq)
    assert np.allclose(a[0, 1], freq, rtol=1e-12)
    for interleaved in (False, True):
        y, _ = ref.norm_rope(x, None, None, a, interleaved)
        assert np.array_equal(y[:, 0], x[:, 0]) and np.array_equal(y[..., 32:], x[..., 32:])
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1))


def test_speculative_draws_follow_the_target():
    """Summed over all proposals and numbers, what is emitted first is distributed as the target."""
    p, q = np.float32([0.5, 0.25, 0.25, 0.0]), np.float32([0.25, 0.5, 0.125, 0.125])
    one = lambda x: (x, [int(t * 2 ** 32) for t in x], 2 ** 32)
    got, n = np.zeros(4), 64
    for y in range(4):
        for a in (np.arange(n) + 0.5) / n:
            for b in (np.arange(n) + 0.5) / n:
                k, tok = ref.speculative([one(p)], [one(q)], [y], [a], b)
                got[tok] += q[y] / n / n
    assert np.allclose(got, p, atol=1.0 / n)
