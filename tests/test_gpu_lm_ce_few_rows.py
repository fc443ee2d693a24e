"""fp32 LM head, one to five rows: both gradients in one pass over a wide weight, and as products where it is narrower."""
import pytest
import torch

from tests.loss_util import gen
from tests.test_gpu_lm_ce import check, head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 512), (1, 1001, 516), (1, 130, 508), (2, 63, 1028), (2, 4099, 1024), (2, 300, 1020), (3, 300, 1540), (3, 65, 1536), (3, 301, 1532),
                                          (4, 257, 2048), (4, 4, 2052), (4, 2049, 2044), (4, 3, 16384), (1, 5001, 16380), (5, 257, 2560)])
def test_either_side_of_every_width(rows, vocab, d):
    y, w, tokens, mask = head(rows, vocab, d, "fp32", seed=rows + d)
    mask[:] = 1
    check(y, w, tokens, mask, scale=0.5)
    check(y, w, tokens, mask, scale=0.5, want_dw=False)
    check(y, w, tokens, mask, torch.randn(rows, device=y.device, generator=gen(2)), scale=-2.0)
    mask[rows - 1] = 0
    y[rows - 1] = float("nan")
    check(y, w, tokens, mask)
