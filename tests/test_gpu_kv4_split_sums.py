"""Attention over a 4-bit cache whose keys are split: pieces in which the largest score, however large, occurs a different number of times.

Queries with one dim each, whose scores are exact but for a factor that all of a row share: tolerances as there (test_gpu_kv4_large_scores.py)."""
import numpy as np
import pytest
import torch

from oracle import efim_kv4_oracle as orc
from tests.test_gpu_kv4_attn import Case
from tests.test_gpu_kv4_large_scores import _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 8, 64), (16, 1, 128), (28, 2, 64)])
@pytest.mark.parametrize("new", [(1, 1), (2, 4)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 12, 2.0 ** 20, 2.0 ** 27, 2.0 ** 40])
def test_equal_largest_scores(hq, hkv, d, new, size):
    case = Case(hq, hkv, d, [5000, 700], new, seed=hq)
    keep = torch.nn.functional.one_hot(torch.randint(d, case.q.shape[:2], generator=torch.Generator().manual_seed(d)), d).bool().cuda()
    case.q.copy_(torch.where(keep, case.q.sign() * (1 + case.q.abs()) * size, 0))
    case.run()
    assert case.status.item() == 0 and case.ws is not None
    for q, k, v, out, lse in _rows(case):
        (want,), (want_lse,), (size_of,), _ = orc.attend(q[None], k, v, [len(k)], d ** -0.5)
        assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -15) * size_of + 2.0 ** -36 * np.abs(v).sum(0)).all()
        assert abs(lse - want_lse) <= 2.0 ** -21 * abs(want_lse) + 2.0 ** -15
