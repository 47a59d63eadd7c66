"""Pins of the 4-bit format's oracle: written-out values, brute force over the grid, ties."""
import numpy as np

from oracle import kv4_oracle as k4


def test_scale_codes_are_fp16_patterns():
    want = (np.arange(248, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)   # (248 and above: infinity, NaN)
    assert np.array_equal(k4.SCALES[:248], want)
    assert k4.SCALES[k4.N_SCALES - 1] == k4.MAX_SCALE and k4.N_SCALES == 227


def test_written_out_group():
    x = np.zeros(128)
    x[:16] = [6, -6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, 0.26, 4.9, 5.1, -3.4, 0.0, 1.0]   # scale 1
    code, s = k4.encode(x)
    assert s[0] == 15 << 3 and not s[1:].any()
    want = [6, -6, 4, 4, 2, 2, 1, 1, 0, 0, 0.5, 4, 6, -3, 0, 1]
    assert np.array_equal(k4.decode(code, s)[:16], want)
    assert not code[16:].any()


def test_nearest_by_brute_force():
    rng = np.random.default_rng(0)
    for grid in (k4.E2M1, k4.SCALES[:k4.N_SCALES]):
        x = np.concatenate([np.abs(rng.standard_normal(2000)) * 3, rng.random(200) * grid[-1] * 1.2, grid, (grid[1:] + grid[:-1]) / 2])
        got = k4.nearest(x, grid)
        d = np.abs(grid[None] - x[:, None])
        assert np.array_equal(d[np.arange(len(x)), got], d.min(1))
        tie = (d == d.min(1, keepdims=True)).sum(1) == 2
        assert tie.sum() >= len(grid) - 1 and not (got[tie] % 2).any()


def test_error_of_a_group_is_bounded():
    """A code is off by at most a sixth of its value's binade step; the scale's own rounding (2^-4) clips at most that much."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((500, 128)) * 10.0 ** rng.uniform(-2, 3, (500, 1))
    y = k4.decode(*k4.encode(x))
    amax = np.abs(x).reshape(500, 8, 16).max(-1).repeat(16, -1)
    assert (np.abs(y - x) <= amax * (1 / 6 + 1 / 16)).all()


def test_values_are_bf16_numbers_and_fp16_numbers():
    v = (k4.E2M1[:, None] * k4.SCALES[None, :k4.N_SCALES]).ravel()
    assert np.array_equal(v, v.astype(np.float16).astype(np.float64))
    bits = v.astype(np.float32).view(np.uint32)
    assert not (bits & 0xffff).any()


def test_pack_round_trip():
    c = np.random.default_rng(2).integers(0, 16, (3, 5, 128)).astype(np.uint8)
    assert np.array_equal(k4.unpack(k4.pack(c)), c)
    assert k4.pack(c)[0, 0, 0] == c[0, 0, 0] + 16 * c[0, 0, 1]


def test_saturation_and_nan():
    x = np.zeros(128)
    x[0], x[1], x[16], x[17] = np.inf, 3.0, np.nan, 1.0
    y = k4.decode(*k4.encode(x))
    assert y[0] == k4.MAX_VALUE and y[1] == 0.0 and y[16] == 0.0 and abs(y[17] - 1.0) <= 1 / 16
