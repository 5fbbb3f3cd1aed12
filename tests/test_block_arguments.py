"""CPU tests of what the functions that run an MoE block's operators together
refuse, before any device work."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2606_00079_amd")

from paper_2606_00079_amd import pipeline  # noqa: E402

T, E, k, N, K = 6, 4, 2, 32, 64


def layer(x_rows=T, logit_rows=T, kept=None, train=True):
    bf16 = torch.bfloat16
    ex = pipeline.Experts(torch.zeros((E, 2 * N, K), dtype=bf16), torch.zeros((E, K, N), dtype=bf16))
    return pipeline.experts_layer(torch.zeros((x_rows, K), dtype=bf16), torch.zeros((logit_rows, E)), ex, k,
                                  train=train, kept=kept)


@pytest.mark.parametrize("rows,cols", [(T - 1, K), (T + 1, K), (T, K + 32), (0, K)])
def test_kept_tokens_of_another_shape(rows, cols):
    """Rows that are not there would be left out of the weights' gradient without a word."""
    kept = (torch.zeros((rows, cols), dtype=torch.uint8), torch.zeros((rows, cols // 32), dtype=torch.uint8))
    with pytest.raises(ValueError, match="kept"):
        layer(kept=kept)


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("x_rows,logit_rows", [(T, T - 1), (T, T + 1), (T, 0), (0, T)])
def test_logits_of_other_rows(x_rows, logit_rows, train):
    """Slots of rows that are not there would give zeros without a word."""
    with pytest.raises(ValueError, match="logits"):
        layer(x_rows, logit_rows, train=train)
