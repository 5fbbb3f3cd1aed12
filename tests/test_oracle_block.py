"""Pins of the oracle of an MoE block's training step: MX8, the norm, the gated
activation and the weights' gradient."""
import numpy as np
import pytest

from oracle import block, mx4, mx8


def test_mx8_grid_is_that_of_e4m3():
    import torch
    codes = torch.arange(127, dtype=torch.uint8)
    assert (mx8.GRID == codes.view(torch.float8_e4m3fn).double().numpy()).all()
    assert mx8.GRID[-1] == 448 and (np.diff(mx8.GRID) > 0).all()


def test_mx8_takes_the_nearest_and_the_smallest_scale():
    g = np.random.default_rng(0)
    X = g.standard_normal((40, 64)) * np.exp(20 * g.standard_normal((40, 1)))
    codes, scales = mx8.quantize(X)
    V = mx8.dequantize(codes, scales)
    step = np.ldexp(1.0, scales.astype(int) - 127).repeat(32, -1)
    top = np.abs(X).reshape(40, 2, 32).max(-1)
    unit = np.ldexp(1.0, scales.astype(int) - 127)
    assert (top <= 448 * unit).all() and (top > 224 * unit).all()
    near = np.abs(np.abs(X / step)[..., None] - mx8.GRID).min(-1)  # by looking at every value
    assert np.allclose(np.abs(X - V) / step, near, rtol=0, atol=1e-12)
    assert (np.abs(X - V) <= np.maximum(np.abs(X) * 2.0 ** -4, step * 2.0 ** -10)).all()


@pytest.mark.parametrize("x,scale,value", [
    (0.0, 0, 0.0), (448.0, 127, 448.0), (449.0, 128, 448.0), (2.0 ** -133, 0, 2.0 ** -133), (1.0, 119, 1.0),
    (np.inf, 255, np.nan), (np.nan, 255, np.nan),
])
def test_mx8_edges(x, scale, value):
    X = np.zeros((1, 32))
    X[0, 3] = x
    codes, scales = mx8.quantize(X)
    assert scales[0, 0] == scale
    assert np.array_equal(mx8.dequantize(codes, scales)[0, 3], value, equal_nan=True)


def test_mx8_ties_go_to_the_even_code():
    for i in range(126):
        X = np.zeros((1, 32))
        X[0, 0], X[0, 1] = 448.0, (mx8.GRID[i] + mx8.GRID[i + 1]) / 2
        assert mx8.quantize(X)[0][0, 1] == i + i % 2


def difference(f, x, dx, eps=1e-6):
    """d f along dx by a central difference."""
    return (f(x + eps * dx) - f(x - eps * dx)) / (2 * eps)


def test_norm_gradient_is_that_of_differences():
    g = np.random.default_rng(1)
    v, w, dy, dsum = g.standard_normal((5, 16)), g.standard_normal(16), g.standard_normal((5, 16)), \
        g.standard_normal((5, 16))
    y, inv = block.rms_norm(v, w, 0.1)
    assert np.allclose((y / w) ** 2 @ np.ones(16) / 16, (v * v).mean(1) / ((v * v).mean(1) + 0.1))
    dx, dw = block.rms_norm_grad(v, w, inv, dy, dsum)
    along, wlong = g.standard_normal(v.shape), g.standard_normal(16)
    loss = lambda v, w: (block.rms_norm(v, w, 0.1)[0] * dy).sum() + (v * dsum).sum()  # noqa: E731
    assert np.isclose(difference(lambda t: loss(t, w), v, along), (dx * along).sum(), rtol=1e-7)
    assert np.isclose(difference(lambda t: loss(v, t), w, wlong), (dw * wlong).sum(), rtol=1e-7)


def test_glu_gradient_is_that_of_differences():
    g = np.random.default_rng(2)
    gu, dh, along = 2 * g.standard_normal((7, 12)), g.standard_normal((7, 6)), g.standard_normal((7, 12))
    grad = mx8.glu_grad(gu, dh)
    assert np.isclose(difference(lambda t: (mx8.glu(t) * dh).sum(), gu, along), (grad * along).sum(), rtol=1e-7)


def test_weight_gradient_is_that_of_differences():
    g = np.random.default_rng(3)
    E, N, K, S = 3, 5, 4, 11
    offsets, rows = np.array([1, 4, 4, 9]), g.integers(-1, 7, S)
    W, X, dY = g.standard_normal((E, N, K)), g.standard_normal((6, K)), g.standard_normal((S, N))
    dW = block.weight_grad(dY, X, E, offsets, rows)
    along = g.standard_normal(W.shape)
    loss = lambda w: (mx4.product(w, X, offsets, rows) * dY).sum()  # noqa: E731
    assert np.isclose(difference(loss, W, along), (dW * along).sum(), rtol=1e-7)
    assert (dW[1] == 0).all()
