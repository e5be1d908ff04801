"""Pins of the 8-bit oracle against hand-worked values and torch's float8 types (CPU)."""
import numpy as np
import pytest

from oracle import q8 as O

torch = pytest.importorskip("torch")


def test_grid_by_hand():
    # e4m3: 3 digits, least normal 2^-6, step of the subnormals 2^-9; ties to even.
    y = [1.0, 1.0625, 1.0624, 1.0626, 1.1875, 448.0, 2 ** -9, 2 ** -10, 1.5 * 2 ** -9, -17.0, np.inf, np.nan]
    want = [1.0, 1.0, 1.0, 1.125, 1.25, 448.0, 2 ** -9, 0.0, 2 * 2 ** -9, -16.0, np.nan, np.nan]
    np.testing.assert_array_equal(O.to_grid(y, "e4m3"), want)
    np.testing.assert_array_equal(O.to_grid([1.125, 1.375, 57344.0, -np.inf, 2 ** -17], "e5m2"),
                                  [1.0, 1.5, 57344.0, -np.inf, 0.0])


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_grid_matches_the_float8_types(fmt, dtype):
    most = O.FORMATS[fmt][0]
    rng = np.random.default_rng(3)
    y = np.concatenate([rng.standard_normal(4000) * np.exp2(rng.integers(-16, 7, 4000)), np.linspace(-2, 2, 4097)])
    y = np.clip(y, -most, most).astype(np.float32)
    got = torch.from_numpy(y).to(dtype).to(torch.float64).numpy()
    np.testing.assert_array_equal(O.to_grid(y, fmt), got)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_scale_is_the_smallest_power_that_holds_the_block(fmt):
    most = O.FORMATS[fmt][0]
    for j in (-100, -8, 0, 5, 90):
        for f, extra in ((1.0, 0), (1.0 + 2 ** -20, 1), (0.5 + 2 ** -20, 0), (0.5, -1)):
            x = np.zeros((1, 130))
            x[0, 7] = -f * most * 2.0 ** j
            x[0, 9] = np.nan
            q, e = O.quantise(x, fmt)
            assert e.tolist() == [[j + extra, 0]]
            assert np.abs(q[0, 7]) <= most and np.isnan(q[0, 9])


def test_dequantise_and_combine_by_hand():
    q = np.ones((2, 129))
    e = np.array([[1, -2], [0, 3]])
    h = O.dequantise(q, e)
    assert h[0, 127] == 2 and h[0, 128] == 0.25 and h[1, 128] == 8
    out, norms = O.combine(h, np.array([[1, -1], [0, 1], [2, 7]]), np.array([[0.5, 9.0], [2.0, 1.0], [1.0, 1.0]]),
                           x=np.full((3, 129), 10.0), gate=np.array([[2.0] * 129, [3.0] * 129]), seq=2)
    assert out[0, 0] == 11 and out[0, 128] == 18 and out[1, 0] == 20 and (out[2] == 10).all()
    np.testing.assert_allclose(norms[1], [np.sqrt(128 * 4 + 0.0625), np.sqrt(128 + 64)])
    assert norms[0, 1] == 0 and (norms[2] == 0).all()


def test_grouped_matmul_is_a_product_per_group():
    rng = np.random.default_rng(1)
    a, b, bias = rng.standard_normal((7, 5)), rng.standard_normal((6, 5)), rng.standard_normal((3, 2))
    out, done, _ = O.matmul(a, b, [1, 4, 4, 99], 2, bias)
    np.testing.assert_allclose(out[1:4], a[1:4] @ b[:2].T + bias[0])
    np.testing.assert_allclose(out[4:], a[4:] @ b[4:].T + bias[2])
    assert done.tolist() == [False] + [True] * 6
    z = torch.linspace(-5, 5, 101, dtype=torch.float64)
    for act, approx in (("gelu", "none"), ("gelu_tanh", "tanh")):
        np.testing.assert_allclose(O.gelu(z.numpy(), act == "gelu_tanh"),
                                   torch.nn.functional.gelu(z, approximate=approx).numpy(), rtol=1e-12, atol=1e-12)
