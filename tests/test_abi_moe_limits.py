"""CPU tests of the C ABI of the MoE layer's calls at the edge of their limits:
refused before any device work, or nothing to do."""
import os

import pytest

pkg = pytest.importorskip("paper_2606_00079_amd")

OK, ARG, SHAPE, DTYPE = 0, 1, 2, 3
F32, BF16 = 0, 1
P = 4096  # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pkg.LIB_PATH):
        pytest.skip("libbitsmoe.so not built")
    return pkg.lib()


@pytest.mark.parametrize("S", [(1 << 31) - 256, (1 << 31) - 17, (1 << 31) - 16, (1 << 31) - 1])
def test_products_refuse_slots_whose_tiles_would_end_past_31_bits(lib, S):
    """A tile of 128 slots that begins at one of the last has an end above 2^31 - 1."""
    x_rows = S
    assert lib.bitsmoe_mx4_product(P, P, 2, 2048, 512, P, BF16, x_rows, 512, P, P, S, 0, P, BF16, 2048, None) == SHAPE
    assert lib.bitsmoe_mx4_product_q(P, P, 2, 2048, 1024, P, P, x_rows, P, P, S, 0, P, BF16, 2048, None) == SHAPE
    assert lib.bitsmoe_mx4_product_grad(P, P, 2, 512, 2048, P, BF16, 512, P, S, P, BF16, 2048, None) == SHAPE
    assert lib.bitsmoe_last_error()


def test_route_workspace(lib):
    """Room for the sums of more than one run of rows; none up to 16 rows, or 128 of up to 512 experts."""
    size = lib.bitsmoe_route_workspace
    assert size(0, 8) == size(-3, 8) == size(100, 0) == size(100, 4097) == size(1 << 31, 8) == 0
    assert size(16, 4096) == size(128, 512) == 0
    for T, E in [(17, 513), (129, 1), (129, 512), (4096, 128), (16384, 256), (32769, 60), (1 << 20, 4096)]:
        run = min(max(-(-T // 256), 16), 128)
        runs = -(-T // run)
        assert size(T, E) >= 2 * 4 * E * (runs + 1) + 8 * runs, (T, E)


@pytest.mark.parametrize("work,room", [(None, 1 << 30), (P, 100), (P + 4, 1 << 30)])
def test_route_refuses_a_workspace_that_is_none(lib, work, room):
    """Missing, too small, misaligned."""
    assert lib.bitsmoe_route_ws(P, BF16, 300, 8, 8, 2, None, 1, P, P, P, P, P, P, P, P, work, room, None) == ARG
    assert b"workspace" in lib.bitsmoe_last_error()


def test_route_with_a_workspace_checks_the_rest_as_well(lib):
    a = [P, BF16, 300, 8, 8, 2, None, 1, P, P, P, P, P, P, P, P, P, 1 << 30, None]
    for at, value, status in [(0, None, ARG), (1, 5, DTYPE), (2, -1, ARG), (4, 7, SHAPE), (5, 9, SHAPE), (8, None, ARG),
                              (13, P + 4, ARG)]:
        assert lib.bitsmoe_route_ws(*a[:at], value, *a[at + 1:]) == status, at


ALL = dict(Z=P, zt=BF16, S=4, slots=P, weights=P, dY=P, T=2, k=2, d=64, dZ=P, dweights=P, work=None, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, {"Z": None}), (ARG, {"slots": None}), (ARG, {"dY": None}), (ARG, {"dZ": None}), (ARG, {"T": 0, "dZ": None}),
    (ARG, {"T": 8193}),  # more than 16384 slots, and no workspace
    (ARG, {"T": 8193, "work": P + 4}), (DTYPE, {"zt": 7}), (SHAPE, {"d": 12}), (SHAPE, {"k": 65}),
    (SHAPE, {"T": 1 << 24, "work": P}),
])
def test_combine_grad_all(lib, status, change):
    assert lib.bitsmoe_combine_grad_all(*{**ALL, **change}.values()) == status, change
    assert lib.bitsmoe_last_error()


def test_combine_grad_all_of_nothing(lib):
    n = None
    assert lib.bitsmoe_combine_grad_all(n, BF16, 0, n, n, n, 0, 2, 64, n, n, n, n) == OK
    assert lib.bitsmoe_last_error() == b""
