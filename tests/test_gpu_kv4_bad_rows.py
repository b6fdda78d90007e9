"""Attention over a 4-bit cache where no sequence has a row that can be computed: the call says so, whether keys are split or not."""
import pytest
import torch

from tests.test_gpu_kv4_attn import Case

pytestmark = pytest.mark.gpu
BAD_POSITION = 2


def _case(new, extra_rows=0):
    case = Case(8, 2, 128, [190, 100], new, extra_rows=extra_rows)
    case.table = torch.nn.functional.pad(case.table, (0, 256 - case.table.shape[1]), value=-1)
    return case


@pytest.mark.parametrize("max_ctx", [200, 4096])
@pytest.mark.parametrize("indptr", [[10, 12, 15], [-7, -5, -2], [5, 3, 1], [1 << 30, (1 << 30) + 2, (1 << 30) + 5]])
def test_no_sequence_has_its_rows(max_ctx, indptr):
    case = _case([2, 3])
    case.indptr = torch.tensor(indptr, dtype=torch.int32, device="cuda")
    case.run(max_ctx=max_ctx)
    assert case.status.item() == BAD_POSITION
    assert (case.out.float() == 5).all() and (case.lse == 5).all()


@pytest.mark.parametrize("max_ctx", [200, 4096])
def test_no_rows_at_all(max_ctx):
    """Nothing to compute is no error, but for a length beyond the call's bound."""
    case = _case([0, 0], 3)
    for ctx, status in ((190, 0), (5000, BAD_POSITION)):
        case.ctx[0] = ctx
        case.run(max_ctx=max_ctx, max_new=2)
        assert case.status.item() == status
        assert (case.out.float() == 5).all() and (case.lse == 5).all()
