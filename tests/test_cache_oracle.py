"""The oracle of the cache calls against closed forms and independent ways to
the same numbers (CPU)."""
import math

import numpy as np
import pytest

import oracle.cache_ref as R


def test_e2m1_values_and_midpoints():
    """Every level encodes to itself, every midpoint to its even neighbour."""
    block = np.zeros(32)
    block[0] = 6.0
    block[1:9] = R.E2M1
    block[9:16] = (R.E2M1[1:] + R.E2M1[:-1]) / 2
    block[16:24] = -R.E2M1
    codes, byte = R.mxfp4_encode(block)
    assert byte == 127
    assert list(codes[1:9]) == list(range(8))
    assert list(codes[9:16]) == [0, 2, 2, 4, 4, 6, 6]
    assert list(codes[16:24] & 7) == list(range(8))
    row = R.mxfp4_pack(codes, byte, 32)
    assert np.array_equal(R.mxfp4_decode(row, 32)[1:9], R.E2M1)


@pytest.mark.parametrize("top,exponent,held", [
    (4.0, 0, 4.0), (6.0, 0, 6.0), (7.0, 0, 6.0), (7.001, 1, 8.0), (7.999, 1, 8.0), (8.0, 1, 8.0),
    (1.0, -2, 1.0), (3.5, -1, 3.0), (3.51, 0, 4.0)])
def test_block_exponent(top, exponent, held):
    """7 units is where clipping to 6 costs as much as the coarser grid."""
    block = np.zeros(32)
    block[5] = top
    codes, byte = R.mxfp4_encode(block)
    assert byte == 127 + exponent
    assert R.mxfp4_decode(R.mxfp4_pack(codes, byte, 32), 32)[5] == held


def test_block_error_is_at_most_half_a_step():
    g = np.random.default_rng(5)
    x = g.standard_normal((400, 32)) * np.exp(3 * g.standard_normal((400, 1)))
    codes, byte = R.mxfp4_encode(x)
    y = R.mxfp4_decode(R.mxfp4_pack(codes, byte, 32), 32)
    unit = 2.0 ** (byte.astype(int) - 127)[:, 0]
    assert np.all(np.abs(x - y).max(-1) <= unit * (1 + 1e-12))  # steps of 2 units at most
    small = np.abs(x) <= 2 * unit[:, None]
    assert np.all((np.abs(x - y) / unit[:, None])[small] <= 0.25 + 1e-12)


def test_zero_tiny_and_nan_blocks():
    codes, byte = R.mxfp4_encode(np.zeros(32))
    assert byte == 1 and not codes.any()
    _, byte = R.mxfp4_encode(np.full(32, 2.0 ** -140))
    assert byte == 1
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[40] = bad
        codes, byte = R.mxfp4_encode(x)
        y = R.mxfp4_decode(R.mxfp4_pack(codes, byte, 48), 64)
        assert np.all(y[:32] == 1) and np.all(np.isnan(y[32:]))


def test_quick_encode_is_the_oracle():
    from cache_harness import quick_encode
    g = np.random.default_rng(6)
    x = (g.standard_normal((60, 96)) * np.exp(2 * g.standard_normal((60, 1)))).astype(np.float32)
    x[3, 5], x[4, 40], x[5] = np.nan, np.inf, 0
    x[6, :8] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    a, b = R.mxfp4_encode(x)
    c, d = quick_encode(x)
    assert np.array_equal(b, d)
    keep = np.repeat(b != 255, 32, -1)
    assert np.array_equal(a[keep], c[keep])


def test_rotation_closed_forms():
    """Quarter turns, lengths kept, relative positions, transpose = inverse."""
    x = np.zeros((1, 1, 32))
    x[..., 0] = 1
    c, s = np.zeros((1, 16)), np.ones((1, 16))
    assert R.rotate(x, c, s, False)[0, 0, 16] == 1
    assert R.rotate(x, c, s, True)[0, 0, 1] == 1
    g = np.random.default_rng(7)
    a, b = g.standard_normal((2, 1, 1, 32))
    ang = R.rope_angles(400, 32, 10000.0)

    def turn(v, p, il):
        return R.rotate(v, np.cos(ang[p])[None], np.sin(ang[p])[None], il)[0, 0]
    for il in (False, True):
        assert np.isclose(turn(a, 371, il) @ turn(b, 355, il), turn(a, 16, il) @ turn(b, 0, il))
        y = turn(a, 371, il)[None, None]
        back = R.rotate(y, np.cos(ang[371])[None], np.sin(ang[371])[None], il, transpose=True)
        assert np.allclose(back, a)


def test_frequencies():
    f = R.rope_frequencies(128, 10000.0)
    assert f[0] == 1 and np.isclose(f[63], 10000 ** (-126 / 128))
    assert np.allclose(R.rope_frequencies(128, 10000.0, "linear", 4.0), f / 4)
    # NTK: the first pair stays, the last is stretched by the factor exactly
    n = R.rope_frequencies(128, 10000.0, "ntk", 8.0)
    assert n[0] == 1 and np.isclose(n[63], f[63] / 8)
    # both mixes keep the fast pairs and stretch the slow ones
    for mode, low, high in (("bands", 1.0, 4.0), ("yarn", 1.0, 32.0)):
        m = R.rope_frequencies(128, 500000.0, mode, 8.0, 8192, low, high)
        p = R.rope_frequencies(128, 500000.0)
        turns = 8192 * p / (2 * math.pi)
        assert np.allclose(m[turns > 1.5 * high], p[turns > 1.5 * high])
        assert np.allclose(m[turns < low / 1.5], p[turns < low / 1.5] / 8)
        assert np.all(m <= p * (1 + 1e-12)) and np.all(m >= p / 8 * (1 - 1e-12))


def test_attend_closed_forms():
    """Equal keys average the values; a loud key picks its value; causality."""
    g = np.random.default_rng(8)
    v = g.standard_normal((5, 2, 8))
    q = g.standard_normal((2, 4, 8))
    out, lse, _, _ = R.attend(q, np.zeros((5, 2, 8)), v, 2, 1.0)
    assert np.allclose(out[0, 1], v[:4, 0].mean(0)) and np.allclose(out[1, 2], v[:, 1].mean(0))
    assert np.allclose(lse, np.log([[4, 5]] * 4))
    k = np.zeros((5, 2, 8))
    k[2, 0] = 200 * q[1, 0] / (q[1, 0] @ q[1, 0])
    out, lse, _, _ = R.attend(q, k, v, 2, 1.0)
    assert np.allclose(out[1, 0], v[2, 0]) and np.isclose(lse[0, 1], 200)
    out, lse, _, _ = R.attend(q, k, v, 2, 1.0, ok=np.zeros(5, bool))
    assert not out.any() and np.all(lse == -np.inf)
