"""The oracle of packed pages against the definitions in plain words: nearest values, ties, the least exponent, the
bytes' places, and the windows of rows."""
import numpy as np
import pytest

from oracle import packed as op


@pytest.mark.parametrize("seed", range(4))
def test_block_is_nearest(seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(32) * 2.0 ** rng.integers(-100, 100)
    code, s = op.block(x)
    e, amax = s - 127, np.abs(x).max()
    assert amax <= 7 * 2.0 ** e and amax > 7 * 2.0 ** (e - 1)
    y = op.value(code, np.uint8(s))
    grid = np.concatenate([op.VALUES, -op.VALUES]) * 2.0 ** e
    assert (np.abs(x - y) == np.abs(x[:, None] - grid).min(1)).all()


@pytest.mark.parametrize("x,want", [(0.25, 0.0), (0.26, 0.5), (0.75, 1.0), (0.74, 0.5), (1.25, 1.0), (1.75, 2.0),
                                    (2.5, 2.0), (3.5, 4.0), (5.0, 4.0), (5.01, 6.0), (7.0, 6.0)])
def test_ties_go_to_the_even_code(x, want):
    b = np.zeros(32)
    b[0], b[1], b[2] = 7.0, x, -x
    code, s = op.block(b)
    assert s == 127
    y = op.value(code, np.uint8(s))
    assert y[1] == want and y[2] == -want and (code[2] == code[1] + 8)


def test_limits():
    assert op.block(np.zeros(32))[1] == 2 and op.block(np.full(32, 1e-300))[1] == 2
    big = np.full(32, float(np.float32(3.4e38)))
    code, s = op.block(big)
    assert s == 252 and op.value(code, np.uint8(s))[0] == 6 * 2.0 ** 125
    for odd in (np.inf, -np.inf, np.nan):
        b = np.ones(32)
        b[7] = odd
        code, s = op.block(b)
        assert s == 255 and not code.any() and np.isnan(op.value(code, np.uint8(s))).all()


@pytest.mark.parametrize("p,d", [(32, 32), (64, 128), (96, 64), (32, 96)])
def test_bytes_go_where_the_layout_says(p, d):
    rng = np.random.default_rng(p + d)
    k, v = rng.standard_normal((2, p, d))
    b = op.encode_plane(k, v)
    assert b.size == op.plane_bytes(p, d) and b.dtype == np.uint8
    n, s = p * d // 2, p * d // 32
    for t, c in ((0, 0), (31, 1), (p - 1, d - 1), (17, 30)):
        code, e = op.block(k[t, c // 32 * 32:c // 32 * 32 + 32])
        assert (b[t * d // 2 + c // 2] >> 4 * (c & 1)) & 15 == code[c % 32]
        assert b[n + t // 32 * d + c // 32 * 32 + t % 32] == e
        code, e = op.block(v[t // 32 * 32:t // 32 * 32 + 32, c])
        assert (b[n + s + (t // 8 * d + c) * 4 + t % 8 // 2] >> 4 * (t & 1)) & 15 == code[t % 32]
        assert b[2 * n + s + t // 32 * d + c] == e
    dk, dv = op.decode_plane(b, p, d)
    assert np.abs(dk - k).max() <= np.abs(k).max() / 7 * 2 and np.abs(dv - v).max() <= np.abs(v).max() / 7 * 2
    assert (op.encode_plane(dk, dv) == b).mean() > 0.5  # (a value of 6 alone fixes its block's exponent)
    dk2, dv2 = op.decode_plane(op.encode_plane(dk, dv), p, d)
    assert (dk2 == dk).mean() > 0.9 and (dv2 == dv).mean() > 0.9


def test_windows():
    assert op.visible(5, 0b1, 1, 0, 0) == [0, 1, 2, 3, 4, 5]
    assert op.visible(5, 0b1, 1, 2, 2) == [0, 1, 4, 5]
    assert op.visible(5, 0b1, 1, 0, 1) == [5]
    assert op.visible(5, 0b1, 1, 4, 2) == [0, 1, 2, 3, 4, 5]
    assert op.visible(2, 0b10101, 5, 3, 1) == [0, 1, 2, 6]  # sees 0, 1, 2, 4, 6
    assert op.visible(0, 0b0, 3, 3, 1) == []
