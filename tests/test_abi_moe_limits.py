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
