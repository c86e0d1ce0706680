"""The layer operators' oracle against hand-worked blocks, enumeration and differences (CPU)."""
import numpy as np
import pytest

from oracle import layers as ol


def test_int8_block_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [3.0, -1.0, 3.99, 0.03125, 0.046875, -0.015625]    # largest 3.99: e = 1, steps of 1/32
    codes, scales = ol.pack("int8", x)
    assert codes.shape == (1, 1, 128) and scales.shape == (1, 1, 4)
    assert scales[0, 0].tolist() == [128, 0, 0, 0]
    # 3.99 * 32 = 127.68 -> 128, held to 127; 1.5 -> 2 and -0.5 -> -0 (ties to even)
    assert codes[0, 0, :7].tolist() == [96, -32, 127, 1, 2, 0, 0] and not codes[0, 0, 7:].any()


def test_fp4_block_by_hand():
    x = np.zeros((1, 40))
    x[0, :9] = [4.0, 7.9, 5.0, 5.01, 2.5, 3.5, 0.25, -0.75, -0.2]    # e = 2, scale 1
    x[0, 32:34] = [0.0, 1e-3]
    codes, scales = ol.pack("fp4", x)
    n = np.stack([codes[0, 0] & 15, codes[0, 0] >> 4], 1).reshape(-1)
    assert n[:9].tolist() == [6, 7, 6, 7, 4, 6, 0, 8 + 2, 8]          # 4 6 4 6 2 4 0 -1 -0
    assert scales[0, 0].tolist() == [127, -10 - 2 + 127, 0, 0]        # 1e-3 lies over 2^-10
    v = ol.unpack("fp4", codes, scales, 40)
    assert v[0, :9].tolist() == [4, 6, 4, 6, 2, 4, 0, -1, 0]


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_packing_is_nearest_of_all_codes(fmt):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 96)) * np.exp(rng.standard_normal((20, 96)))
    x = x.astype(np.float32).astype(np.float64)
    v = ol.kept(fmt, x)
    for r in range(20):
        for b in range(3):
            blk = x[r, 32 * b:32 * b + 32]
            p = 2.0 ** np.floor(np.log2(np.abs(blk).max()))
            grid = np.arange(-127, 128) * p / 64 if fmt == "int8" else ol.GRID * p / 4
            d = np.abs(blk[:, None] - grid)
            np.testing.assert_array_equal(np.abs(blk - v[r, 32 * b:32 * b + 32]), d.min(1))


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_packing_again_changes_nothing(fmt):
    x = np.random.default_rng(2).standard_normal((7, 133))
    v = ol.kept(fmt, x)
    np.testing.assert_array_equal(ol.kept(fmt, v), v)
    assert np.abs(v - x).max() <= np.abs(x).max() * (2.0 ** -6 if fmt == "int8" else 0.25)


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
def test_ends_of_the_range(fmt):
    tiny, huge = 2.0 ** -149, (2 - 2.0 ** -23) * 2.0 ** 127
    x = np.zeros((4, 32))
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = tiny, huge, np.nan, -np.inf
    x[2, 1] = x[3, 1] = 1.0
    codes, scales = ol.pack(fmt, x)
    assert scales[:, 0, 0].tolist() == [0, 254 if fmt == "int8" else 252, 255, 255]
    v = ol.unpack(fmt, codes, scales, 32)
    assert np.isnan(v[2:]).all() and v[0, 0] == 0 and np.isfinite(v[1]).all() and v[1, 0] > 0.75 * huge


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_slopes_by_differences(kind):
    x = np.linspace(-8, 8, 401)
    h = 1e-5
    d = (ol.act(kind, x + h) - ol.act(kind, x - h)) / (2 * h)
    # error of the difference: h^2 |f'''| / 6 + 1e-16 |f| / h, both below 1e-9
    np.testing.assert_allclose(ol.act_slope(kind, x), d, atol=1e-9)


def test_linear_gradients_by_differences():
    # the products are bilinear: a difference over one step is exact but for rounding
    rng = np.random.default_rng(3)
    x, w, dy = rng.standard_normal((5, 40)), rng.standard_normal((6, 40)), rng.standard_normal((5, 6))
    xk = ol.kept("int8", x)
    dw, db = ol.linear_backward_weight(dy, x)
    dx = ol.linear_backward_input(dy, w)

    def loss(x_, w_, b_):
        return float((dy * (x_ @ w_.T + b_)).sum())
    zero = np.zeros(6)
    for i, j in [(0, 0), (5, 39), (3, 17)]:
        e = np.zeros_like(w)
        e[i, j] = 1
        assert abs(loss(xk, w + e, zero) - loss(xk, w, zero) - dw[i, j]) < 1e-11
    for i, j in [(0, 0), (4, 39), (2, 31)]:
        e = np.zeros_like(x)
        e[i, j] = 1
        assert abs(loss(x + e, w, zero) - loss(x, w, zero) - dx[i, j]) < 1e-11
    for i in range(6):
        assert abs(loss(x, w, np.eye(6)[i]) - loss(x, w, zero) - db[i]) < 1e-11
