"""Arguments of the experts' wrappers and of ``ExpertLayer``: calls without work, shapes
that do not fit, streams and devices.
"""
import pytest
import torch

from paper_2512_05831_amd import experts as ex
from test_gpu_expert_product import blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("shape", [(3, 0, 200), (0, 5, 200), (0, 0, 16), (2, 0, 1)])
def test_stacks_without_rows(shape, block_rows, device):
    q, s = ex.quantize_fp8(torch.empty(shape, device=device), block_rows=block_rows)
    m, rows, cols = shape
    assert q.shape == shape and q.dtype == torch.float8_e4m3fn
    assert s.shape == (m, rows if block_rows == 1 else blocks(rows), blocks(cols))
