"""A turn over a 4-bit cache in which some sequences have no new tokens: lengths of theirs are no lengths of the call."""
import pytest
import torch

from tests.test_gpu_kv4_prefill import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (16, 1, 128)])
@pytest.mark.parametrize("ctx,new", [([5000, 100], [0, 1]),                          # units that fit a CTA
                                     ([100, 4000, 3000, 700], [1, 0, 0, 1]),          # units that are cut
                                     ([9000, 2000, 16], [0, 1, 0]), ([20, 600, 513], [1, 0, 0])])
def test_an_idle_sequence_longer_than_the_others(hq, hkv, d, ctx, new):
    case = Case(hq, hkv, d, ctx, new, seed=len(ctx))
    case.run()
    case.check()
    assert case.status.item() == 0


def test_an_idle_sequence_among_many_rows():
    case = Case(32, 8, 128, [300, 5000, 200], [90, 0, 40])
    case.run()
    out, lse = case.bf16()
    torch.cuda.synchronize()
    assert case.status.item() == 0
    assert torch.equal(case.out.view(torch.int16), out.view(torch.int16)) and torch.equal(case.lse, lse)
