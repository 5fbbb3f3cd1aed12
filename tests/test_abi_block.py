"""CPU tests of the C ABI of an MoE block's training calls: what they refuse,
before any device work, and with which status."""
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


@pytest.mark.parametrize("status,args", [
    (ARG, (None, BF16, 2, 64, 64, P, P, None)), (ARG, (P, BF16, 2, 64, 64, BAD, P, None)),
    (ARG, (P, BF16, 2, 64, 64, P, None, None)), (ARG, (P, BF16, -1, 64, 64, P, P, None)),
    (ARG, (P, BF16, 2, 0, 64, P, P, None)), (DTYPE, (P, 3, 2, 64, 64, P, P, None)),
    (SHAPE, (P, BF16, 2, 48, 64, P, P, None)), (SHAPE, (P, BF16, 2, 64, 32, P, P, None)),
    (SHAPE, (P, BF16, 2, 64, 68, P, P, None)), (SHAPE, (P, F32, 1 << 36, 64, 64, P, P, None)),
])
def test_mx8_quantize(lib, status, args):
    refused(lib, status, "bitsmoe_mx8_quantize", *args)


@pytest.mark.parametrize("status,args", [
    (ARG, (None, P, 2, 64, P, BF16, None)), (ARG, (P, P, 2, 64, BAD, BF16, None)),
    (DTYPE, (P, P, 2, 64, P, 9, None)), (SHAPE, (P, P, 2, 33, P, BF16, None)),
])
def test_mx8_dequantize(lib, status, args):
    refused(lib, status, "bitsmoe_mx8_dequantize", *args)


NORM = dict(X=P, xt=BF16, ldx=64, R=P, ldr=64, W=P, wt=F32, T=4, d=64, eps=1e-6, Sum=P, Y=P, codes=P, scales=P, inv=P,
            stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"X": None}), (ARG, {"W": None}), (ARG, {"inv": None}), (ARG, {"Sum": None}), (ARG, {"codes": None}),
    (ARG, {"scales": None}), (ARG, {"Y": BAD}), (ARG, {"R": BAD}), (ARG, {"T": -1}), (ARG, {"d": 0}),
    (ARG, {"eps": 0.0}), (ARG, {"eps": 1e-60}), (ARG, {"eps": -1.0}), (ARG, {"eps": float("nan")}), (ARG, {"eps": float("inf")}),
    (DTYPE, {"xt": 2}), (DTYPE, {"wt": -1}), (SHAPE, {"d": 60, "ldx": 64, "ldr": 64}),
    (SHAPE, {"d": 40}), (SHAPE, {"d": 32800, "ldx": 32800, "ldr": 32800}), (SHAPE, {"ldx": 56}), (SHAPE, {"ldr": 68}),
    (SHAPE, {"T": 1 << 36}),
])
def test_rms_norm(lib, status, change):
    refused(lib, status, "bitsmoe_rms_norm", *{**NORM, **change}.values())


NORM_GRAD = dict(Sum=P, xt=BF16, ldsum=64, W=P, wt=F32, inv=P, dY=P, lddy=64, dSum=P, lddsum=64, valid=None, T=40, d=64, dX=P, dW=P,
                 work=P, work_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"Sum": None}), (ARG, {"W": None}), (ARG, {"inv": None}), (ARG, {"dY": None}), (ARG, {"dX": None}),
    (ARG, {"work": None}), (ARG, {"work_bytes": 255}), (ARG, {"dX": BAD}), (ARG, {"work": BAD}), (ARG, {"d": -8}),
    (DTYPE, {"xt": 7}), (DTYPE, {"wt": 7}), (SHAPE, {"d": 36}), (SHAPE, {"ldsum": 63}), (SHAPE, {"lddy": 32}),
    (SHAPE, {"lddsum": 66}),
])
def test_rms_norm_grad(lib, status, change):
    refused(lib, status, "bitsmoe_rms_norm_grad", *{**NORM_GRAD, **change}.values())


def test_rms_norm_grad_workspace(lib):
    size = lib.bitsmoe_rms_norm_grad_workspace
    assert size(0, 64) == size(1, 64) == size(-1, 64) == size(5, 0) == size(5, 1 << 40) == 0
    assert size(1 << 20, 32768) % (32768 * 4) == 0 and size(1 << 20, 32768) > 0
    assert size(5, 4096) == 5 * 4096 * 4


GLU = dict(GU=P, gut=F32, S=4, N=64, ld=128, H=P, codes=P, scales=P, stream=None)
GLU_GRAD = dict(codes=P, scales=P, dH=P, dht=F32, S=4, N=64, lddh=64, dGU=P, H=None, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"GU": None}), (ARG, {"H": None}), (ARG, {"codes": BAD}), (ARG, {"S": -1}), (ARG, {"N": 0}),
    (DTYPE, {"gut": 4}), (SHAPE, {"N": 48}), (SHAPE, {"ld": 64}), (SHAPE, {"ld": 130}), (SHAPE, {"N": 1 << 30}),
    (SHAPE, {"S": 1 << 36}),
])
def test_glu_mx8(lib, status, change):
    refused(lib, status, "bitsmoe_glu_mx8", *{**GLU, **change}.values())


@pytest.mark.parametrize("status,change", [
    (ARG, {"codes": None}), (ARG, {"dH": None}), (ARG, {"dGU": None}), (ARG, {"H": BAD}), (ARG, {"S": -1}),
    (DTYPE, {"dht": 4}), (SHAPE, {"N": 16}), (SHAPE, {"lddh": 32}), (SHAPE, {"lddh": 66}),
])
def test_glu_mx8_grad(lib, status, change):
    refused(lib, status, "bitsmoe_glu_mx8_grad", *{**GLU_GRAD, **change}.values())


PRODUCT = dict(W=P, t=BF16, E=2, N=16, K=64, X=P, x_rows=4, ldx=64, offsets=P, rows=P, S=8, glu=0, Y=P, yt=BF16, ldy=16,
               stream=None)
BOTH = [
    (ARG, {"W": None}), (ARG, {"E": 0}), (ARG, {"N": 0}), (ARG, {"K": -32}), (ARG, {"S": -1}), (ARG, {"offsets": None}),
    (ARG, {"W": BAD}), (DTYPE, {"t": F32}), (SHAPE, {"K": 36}), (SHAPE, {"E": 70000}), (SHAPE, {"S": 1 << 31}),
]


@pytest.mark.parametrize("status,change", BOTH + [
    (ARG, {"X": None}), (ARG, {"Y": None}), (ARG, {"Y": BAD}), (ARG, {"rows": BAD}), (ARG, {"x_rows": -1}),
    (DTYPE, {"yt": 4}), (SHAPE, {"ldy": 15}), (SHAPE, {"ldx": 56}), (SHAPE, {"ldx": 68}),
    (SHAPE, {"rows": None}),  # eight slots of four rows
    (SHAPE, {"N": (1 << 24) + 1, "ldy": 1 << 25}),
])
def test_expert_product(lib, status, change):
    refused(lib, status, "bitsmoe_expert_product", *{**PRODUCT, **change}.values())


PRODUCT_GRAD = dict(W=P, t=BF16, E=2, N=16, K=64, dY=P, lddy=16, offsets=P, S=8, dX=P, xt=BF16, ldx=64, stream=None)


@pytest.mark.parametrize("status,change", BOTH + [
    (ARG, {"dY": None}), (ARG, {"dX": None}), (DTYPE, {"xt": 4}), (SHAPE, {"N": 12}), (SHAPE, {"lddy": 8}),
    (SHAPE, {"lddy": 20}), (SHAPE, {"ldx": 63}),
])
def test_expert_product_grad(lib, status, change):
    refused(lib, status, "bitsmoe_expert_product_grad", *{**PRODUCT_GRAD, **change}.values())


WEIGHT = dict(dY=P, t=BF16, lddy=16, E=2, N=16, K=64, X=P, x_rows=4, ldx=64, offsets=P, rows=P, S=8, dW=P, wt=F32,
              work=None, work_bytes=0, stream=None)
WEIGHT_Q = dict(dY=P, t=BF16, lddy=16, E=2, N=16, K=64, xcodes=P, xscales=P, x_rows=4, offsets=P, rows=P, S=8, dW=P,
                wt=F32, work=None, work_bytes=0, stream=None)
OURS = [b for b in BOTH if "W" not in b[1]] + [
    (ARG, {"dY": None}), (ARG, {"dW": None}), (ARG, {"dW": None, "S": 0}), (ARG, {"rows": BAD}), (DTYPE, {"wt": 4}),
    (SHAPE, {"N": 12}), (SHAPE, {"lddy": 8}), (SHAPE, {"rows": None}), (SHAPE, {"lddy": 1 << 31}),
    (ARG, {"S": 4096, "E": 1, "work": P, "work_bytes": 4096}), (ARG, {"work": BAD, "work_bytes": 1 << 40}),
]


@pytest.mark.parametrize("status,change", OURS + [(ARG, {"X": None}), (SHAPE, {"ldx": 32}), (SHAPE, {"ldx": 68})])
def test_expert_weight_grad(lib, status, change):
    refused(lib, status, "bitsmoe_expert_weight_grad", *{**WEIGHT, **change}.values())


@pytest.mark.parametrize("status,change", OURS + [(ARG, {"xcodes": None}), (ARG, {"xscales": BAD}), (SHAPE, {"K": 40})])
def test_expert_weight_grad_q(lib, status, change):
    refused(lib, status, "bitsmoe_expert_weight_grad_q", *{**WEIGHT_Q, **change}.values())


def test_expert_weight_grad_workspace(lib):
    size = lib.bitsmoe_expert_weight_grad_workspace
    assert size(128, 1536, 2048, 32768) == size(1, 128, 2048, 0) == size(0, 8, 8, 8) == size(1, 8, 8, 100) == 0
    assert size(1, 128, 2048, 4096) % (128 * 2048 * 4) == 0 and size(1, 128, 2048, 4096) > 128 * 2048 * 4
    assert size(1, 128, 2048, 1 << 30) <= 64 << 20


def test_nothing_to_do(lib):
    """Sizes of zero return at once, with no pointer read."""
    none = {k: None for k in ("X", "R", "W", "Sum", "Y", "codes", "scales", "inv", "GU", "H", "dH", "dGU", "dY", "dX")}

    def call(name, args, **change):
        a = {**args, **{k: v for k, v in none.items() if k in args}, **change}
        assert getattr(lib, name)(*a.values()) == OK, lib.bitsmoe_last_error()

    call("bitsmoe_rms_norm", NORM, T=0)
    call("bitsmoe_rms_norm_grad", NORM_GRAD, T=0, dW=None)
    call("bitsmoe_glu_mx8", GLU, S=0)
    call("bitsmoe_glu_mx8_grad", GLU_GRAD, S=0)
    call("bitsmoe_expert_product", PRODUCT, S=0)
    call("bitsmoe_expert_product_grad", PRODUCT_GRAD, S=0)
