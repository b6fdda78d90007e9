"""Attention over a 4-bit cache with the table's capacity as the bound of the lengths: workspace and results by exactly those arguments."""
import pytest
import torch

from tests.test_gpu_kv4_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_ctx", [0, -1])
@pytest.mark.parametrize("width", [20, 60, 500])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 0, 5]])
def test_no_bound(max_ctx, width, new):
    case = Case(8, 2, 128, [300, 17, 250], new)
    case.table = torch.nn.functional.pad(case.table, (0, width - case.table.shape[1]), value=-1)
    case.run(max_ctx=max_ctx)
    case.check()
    assert case.status.item() == 0
