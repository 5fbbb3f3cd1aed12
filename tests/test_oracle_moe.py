"""The fp64 oracle of the MoE layer's operators: the format's definition, the
router's rules, and every gradient against differences."""
import numpy as np
import pytest

from oracle import mx4, route


def test_mx4_values_of_one_block():
    x = np.zeros(32)
    x[:12] = [6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.2, 4]
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [127]  # floor(log2 6) - 2 = 0
    assert mx4.dequantize(codes, scales)[:12].tolist() == [6, -6, 0, 1, 1, 2, 2, 4, 4, 6, 0, 4]
    assert codes[0] == 0xF7  # entry 0 in the low half


@pytest.mark.parametrize("scale", [2.0 ** -140, 2.0 ** -126, 2.0 ** -3, 1.0, 2.0 ** 100])
def test_mx4_error_is_bounded(scale):
    g = np.random.default_rng(5)
    x = (g.standard_normal((7, 96)) * scale).astype(np.float32).astype(np.float64)
    codes, scales = mx4.quantize(x)
    v = mx4.dequantize(codes, scales)
    top = np.abs(x).reshape(7, -1, 32).max(-1).repeat(32, -1)
    unit = np.maximum(2.0 ** (np.floor(np.log2(top)) - 2), 2.0 ** -127)
    # half a step of the top binade (1 unit), and up to 2 units where 8 > |x| / unit > 6 is cut
    assert (np.abs(v - x) <= np.where(np.abs(x) > 6 * unit, 2, 1) * unit).all()
    again = mx4.quantize(v)  # a fixed point, unless the cut lowered the top's binade (it cannot)
    assert (mx4.dequantize(*again) == v).all()


def test_mx4_blocks_that_are_lost_or_empty():
    x = np.ones((1, 128))
    x[0, 3], x[0, 40], x[0, 64:96] = np.nan, -np.inf, 0.0
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [[255, 255, 0, 125]]
    v = mx4.dequantize(codes, scales)[0]
    assert np.isnan(v[:64]).all() and (v[64:96] == 0).all() and (v[96:] == 1).all()


def test_route_rules():
    x = np.array([[1, 3, 3, -np.inf], [-np.inf] * 4, [-np.inf, 2, -np.inf, -np.inf], [0, 0, 0, 0], [9, 8, 7, 6]], float)
    r = route.route(x, 2, valid=[1, 1, 1, 1, 0])
    assert r["experts"].tolist() == [[1, 2], [-1, -1], [1, -1], [0, 1], [-1, -1]]
    assert np.allclose(r["weights"], [[.5, .5], [0, 0], [1, 0], [.5, .5], [0, 0]])
    assert r["counts"].tolist() == [1, 3, 1, 0, 3] and r["offsets"].tolist() == [0, 1, 4, 5, 5]
    assert r["rows"].tolist() == [3, 0, 2, 3, 0, 1, 1, 2, 4, 4]
    assert (r["slots"].reshape(-1)[np.argsort(r["slots"].reshape(-1))] == np.arange(10)).all()


def test_balance_is_one_where_experts_are_used_alike():
    x = np.eye(8)[np.arange(64) % 8] * 1e-9
    r = route.route(x, 1)
    assert abs(r["losses"][0] - 1) < 1e-8


@pytest.mark.parametrize("renorm", [True, False])
def test_route_gradient_against_differences(renorm):
    g = np.random.default_rng(3)
    T, E, k = 5, 7, 3
    x = g.standard_normal((T, E)) * 2
    x[1, 2] = -np.inf
    valid = np.array([1, 1, 0, 1, 1])
    dw, dl = g.standard_normal((T, k)), np.array([0.7, -0.3])
    base = route.route(x, k, valid, renorm)

    def f(y):
        # the counts are constants: the balance loss is linear in p with them
        r = route.route(y, k, valid, renorm)
        assert (r["experts"] == base["experts"]).all()
        return (r["weights"] * dw).sum() + (r["losses"] * dl).sum()

    d = route.route_grad(x, base, dw, dl, renorm)
    for t in range(T):
        for e in range(E):
            if not np.isfinite(x[t, e]):
                assert d[t, e] == 0
                continue
            h = 1e-6
            up, dn = x.copy(), x.copy()
            up[t, e] += h
            dn[t, e] -= h
            assert abs((f(up) - f(dn)) / (2 * h) - d[t, e]) < 1e-8


def test_product_and_combine_gradients_against_differences():
    g = np.random.default_rng(4)
    W = mx4.dequantize(*mx4.quantize(g.standard_normal((3, 8, 32))))
    off = np.array([0, 2, 2, 5])
    X, dY = g.standard_normal((6, 32)), g.standard_normal((6, 8))  # (slot 5 has no expert)
    d = mx4.product_grad(W, dY, off)
    h = 1e-5
    for s, c in [(0, 0), (1, 31), (4, 7), (5, 3)]:
        up, dn = X.copy(), X.copy()
        up[s, c] += h
        dn[s, c] -= h
        diff = ((mx4.product(W, up, off) - mx4.product(W, dn, off)) * dY).sum() / (2 * h)
        assert abs(diff - d[s, c]) < 1e-8
    slots, w = np.array([[3, 0], [1, -1], [2, 4]]), g.standard_normal((3, 2))
    Z, dO = g.standard_normal((6, 4)), g.standard_normal((3, 4))
    dZ, dw = route.combine_grad(Z, slots, w, dO)
    f = lambda z, v: (route.combine(z, slots, v) * dO).sum()  # noqa: E731
    for s in range(6):
        e = np.zeros_like(Z)
        e[s, 1] = h
        assert abs((f(Z + e, w) - f(Z - e, w)) / (2 * h) - dZ[s, 1]) < 1e-8
    for t in range(3):
        for j in range(2):
            e = np.zeros_like(w)
            e[t, j] = h
            assert abs((f(Z, w + e) - f(Z, w - e)) / (2 * h) - dw[t, j]) < 1e-8
