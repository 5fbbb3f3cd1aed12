"""An MoE block's training step with rows that do not count, and weights that hold
no numbers.  What a mask leaves out is given to the bit: no bounds."""
import numpy as np
import pytest

from conftest import gpu_available

pytestmark = pytest.mark.gpu

if not gpu_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import torch  # noqa: E402

import paper_2606_00079_amd as bm  # noqa: E402

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def randn(g, *shape, dtype="bf16", scale=1.0):
    return dev((g.standard_normal(shape) * scale).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 64), (6, 64), (40, 1032), (9, 4096), (1100, 512), (5, 16416)])
@pytest.mark.parametrize("weight", ["inf", "-inf", "nan"])
def test_norm_gradient_of_masked_rows_is_that_of_the_sum(dtype, T, d, weight):
    """dx of a row that does not count is dsum (0 without it), whatever the weights hold."""
    g = np.random.default_rng([T, d, 31])
    v, dY, ds = (randn(g, T, d, dtype=dtype) for _ in range(3))
    w, valid = randn(g, d, dtype="f32"), dev(g.random(T) < 0.6)
    valid[0] = False
    w[3], w[d - 1] = float(weight), float(weight)
    inv = bm.rms_norm(v, w).inv
    dX, dw = bm.rms_norm_grad(v, w, inv, dY, dsum=ds, valid=valid)
    assert torch.equal(dX[~valid], ds[~valid])
    assert torch.isfinite(dw).all()
    if weight == "nan":
        assert torch.isnan(dX[valid]).all()
    dX, again = bm.rms_norm_grad(v, w, inv, dY, valid=valid)
    assert not dX[~valid].any() and torch.equal(dw, again)
