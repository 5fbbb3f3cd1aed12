"""CPU tests of the C ABI of the MoE layer's calls: what they refuse, before any
device work, and with which status."""
import os

import pytest

pkg = pytest.importorskip("paper_2606_00079_amd")

OK, ARG, SHAPE, DTYPE = 0, 1, 2, 3
F32, BF16 = 0, 1
P = 4096  # an aligned address that is never read
BAD = P + 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.LIB_PATH):
        pytest.skip("libbitsmoe.so not built")
    return pkg.lib()


def refused(lib, status, name, *args):
    assert getattr(lib, name)(*args) == status, (name, args, lib.bitsmoe_last_error())
    assert lib.bitsmoe_last_error()


ROUTE = dict(logits=P, lt=BF16, T=4, E=8, ld=8, k=2, valid=None, renorm=1, experts=P, weights=P, counts=P,
             offsets=P, rows=P, slots=P, lse=P, losses=P, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"logits": None}), (ARG, {"experts": None}), (ARG, {"counts": None}), (ARG, {"losses": None}),
    (ARG, {"T": -1}), (ARG, {"E": 0}), (ARG, {"k": 0}), (ARG, {"logits": BAD}), (ARG, {"slots": BAD}),
    (DTYPE, {"lt": 2}), (DTYPE, {"lt": -7}), (SHAPE, {"k": 9}), (SHAPE, {"E": 4097, "ld": 4097}),
    (SHAPE, {"E": 100, "ld": 100, "k": 65}), (SHAPE, {"ld": 7}), (SHAPE, {"T": 1 << 30}),
])
def test_route(lib, status, change):
    refused(lib, status, "bitsmoe_route", *{**ROUTE, **change}.values())


GRAD = dict(logits=P, lt=BF16, T=4, E=8, ld=8, k=2, renorm=1, experts=P, weights=P, counts=P, lse=P, dweights=None,
            dlosses=None, dlogits=P, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"logits": None}), (ARG, {"weights": None}), (ARG, {"dlogits": None}), (ARG, {"dweights": BAD}),
    (DTYPE, {"lt": 5}), (SHAPE, {"k": 9}), (SHAPE, {"ld": 4}),
])
def test_route_grad(lib, status, change):
    refused(lib, status, "bitsmoe_route_grad", *{**GRAD, **change}.values())


@pytest.mark.parametrize("status,args", [
    (ARG, (None, BF16, 2, 64, 64, P, P, None)), (ARG, (P, BF16, 2, 64, 64, BAD, P, None)),
    (ARG, (P, BF16, -1, 64, 64, P, P, None)), (ARG, (P, BF16, 2, 0, 64, P, P, None)),
    (DTYPE, (P, 3, 2, 64, 64, P, P, None)), (SHAPE, (P, BF16, 2, 48, 64, P, P, None)),
    (SHAPE, (P, BF16, 2, 64, 32, P, P, None)), (SHAPE, (P, BF16, 2, 64, 68, P, P, None)),
    (SHAPE, (P, F32, 2, 64, 66, P, P, None)), (SHAPE, (P, F32, 1 << 36, 64, 64, P, P, None)),
])
def test_mx4_quantize(lib, status, args):
    refused(lib, status, "bitsmoe_mx4_quantize", *args)


@pytest.mark.parametrize("status,args", [
    (ARG, (None, P, 2, 64, P, BF16, None)), (ARG, (P, P, 2, 64, BAD, BF16, None)),
    (DTYPE, (P, P, 2, 64, P, 9, None)), (SHAPE, (P, P, 2, 33, P, BF16, None)),
])
def test_mx4_dequantize(lib, status, args):
    refused(lib, status, "bitsmoe_mx4_dequantize", *args)


PRODUCT = dict(codes=P, scales=P, E=2, N=16, K=64, X=P, xt=BF16, x_rows=4, ldx=64, offsets=P, rows=P, S=8, glu=0, Y=P,
               yt=BF16, ldy=16, stream=None)
BOTH = [
    (ARG, {"codes": None}), (ARG, {"scales": None}), (ARG, {"Y": None}), (ARG, {"E": 0}), (ARG, {"N": 0}),
    (ARG, {"K": -32}), (ARG, {"S": -1}), (ARG, {"offsets": None}), (ARG, {"Y": BAD}), (ARG, {"rows": BAD}),
    (DTYPE, {"yt": 4}), (SHAPE, {"K": 48}), (SHAPE, {"E": 70000}), (SHAPE, {"ldy": 15}),
    (SHAPE, {"rows": None}),  # eight slots of four rows
    (SHAPE, {"N": (1 << 24) + 1, "ldy": 1 << 25}), (SHAPE, {"S": 1 << 31}),
]


@pytest.mark.parametrize("status,change", BOTH + [
    (ARG, {"X": None}), (ARG, {"X": BAD}), (DTYPE, {"xt": F32}), (SHAPE, {"ldx": 32}), (SHAPE, {"ldx": 68}),
    # few slots an expert, and more workgroups than a launch takes
    (SHAPE, {"E": 65535, "N": 1 << 24, "ldy": 1 << 24, "S": 60000, "K": 32, "ldx": 64}),
])
def test_mx4_product(lib, status, change):
    refused(lib, status, "bitsmoe_mx4_product", *{**PRODUCT, **change}.values())


@pytest.mark.parametrize("status,change", BOTH + [(ARG, {"xcodes": None}), (ARG, {"xscales": None})])
def test_mx4_product_q(lib, status, change):
    a = {k: v for k, v in PRODUCT.items() if k not in ("X", "xt", "ldx")}
    a = {"codes": P, "scales": P, "E": 2, "N": 16, "K": 64, "xcodes": P, "xscales": P, **a}
    order = ["codes", "scales", "E", "N", "K", "xcodes", "xscales", "x_rows", "offsets", "rows", "S", "glu", "Y", "yt",
             "ldy", "stream"]
    a.update(change)
    refused(lib, status, "bitsmoe_mx4_product_q", *(a[k] for k in order))


PGRAD = dict(codes=P, scales=P, E=2, N=16, K=64, dY=P, dyt=BF16, lddy=16, offsets=P, S=8, dX=P, xt=F32, ldx=64,
             stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"codes": None}), (ARG, {"dY": None}), (ARG, {"dX": None}), (ARG, {"offsets": None}), (ARG, {"dY": BAD}),
    (DTYPE, {"dyt": F32}), (DTYPE, {"xt": 2}), (SHAPE, {"N": 12}), (SHAPE, {"lddy": 8}), (SHAPE, {"lddy": 20}),
    (SHAPE, {"ldx": 32}), (SHAPE, {"K": 40}),
])
def test_mx4_product_grad(lib, status, change):
    refused(lib, status, "bitsmoe_mx4_product_grad", *{**PGRAD, **change}.values())


@pytest.mark.parametrize("status,args", [
    (ARG, (None, BF16, 4, P, P, 2, 2, 64, P, None)), (ARG, (P, BF16, 4, None, P, 2, 2, 64, P, None)),
    (ARG, (P, BF16, 4, P, P, 2, 0, 64, P, None)), (ARG, (P, BF16, 4, P, BAD, 2, 2, 64, P, None)),
    (DTYPE, (P, 7, 4, P, P, 2, 2, 64, P, None)), (SHAPE, (P, BF16, 4, P, P, 2, 2, 60, P, None)),
    (SHAPE, (P, BF16, 4, P, P, 2, 65, 64, P, None)),
])
def test_combine(lib, status, args):
    refused(lib, status, "bitsmoe_combine", *args)


@pytest.mark.parametrize("status,args", [
    (ARG, (None, BF16, 4, P, P, P, 2, 2, 64, P, P, None)),   # dweights wanted, no rows to read
    (ARG, (P, BF16, 4, P, P, None, 2, 2, 64, P, P, None)), (ARG, (P, BF16, 4, P, P, P, 2, 2, 64, None, P, None)),
    (DTYPE, (P, 7, 4, P, P, P, 2, 2, 64, P, P, None)), (SHAPE, (P, F32, 4, P, P, P, 2, 2, 12, P, P, None)),
    (SHAPE, (P, F32, 4, P, P, P, 1 << 24, 2, 8, P, P, None)),
])
def test_combine_grad(lib, status, args):
    refused(lib, status, "bitsmoe_combine_grad", *args)


def test_nothing_to_do_is_no_error(lib):
    """No rows: nothing is enqueued, and no buffer is needed."""
    n = None
    assert lib.bitsmoe_mx4_quantize(n, BF16, 0, 64, 64, n, n, n) == OK
    assert lib.bitsmoe_mx4_dequantize(n, n, 0, 64, n, BF16, n) == OK
    assert lib.bitsmoe_mx4_product(n, n, 2, 16, 64, n, BF16, 0, 64, P, n, 0, 0, n, BF16, 16, n) == OK
    assert lib.bitsmoe_mx4_product_q(n, n, 2, 16, 64, n, n, 0, P, n, 0, 0, n, BF16, 16, n) == OK
    assert lib.bitsmoe_mx4_product_grad(n, n, 2, 16, 64, n, BF16, 16, P, 0, n, BF16, 64, n) == OK
    assert lib.bitsmoe_combine(n, BF16, 0, n, n, 0, 2, 64, n, n) == OK
    assert lib.bitsmoe_combine_grad(n, BF16, 0, n, n, n, 0, 2, 64, n, n, n) == OK
    assert lib.bitsmoe_route_grad(n, BF16, 0, 8, 8, 2, 1, n, n, n, n, n, n, n, n) == OK
    assert lib.bitsmoe_last_error() == b""


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 64)
    for call in (lambda: pkg.route(x, 2), lambda: pkg.mx4_quantize(x), lambda: pkg.combine(x, torch.zeros(1, 2))):
        with pytest.raises(TypeError):
            call()
