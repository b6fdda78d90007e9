"""Attention over a 4-bit cache with finite queries whose scores are large: 2^20 to 2^40.

Queries with one dim each: products are exact, and so are scores but for the factor that all of a row share (2^-22, of differences that count up to
2^5: 2^-17 of a weight).  What is left is the single-token form's tolerance without its scores' part: the weight's rounding 2^-11, the result's 2^-8.
Full queries: a score is off by at most 2^-16 E, E the largest sum of magnitudes (see the single-token form), plus 2^-22 of itself for the references
that warps and pieces take; keys whose scores lie further than twice that and 40 below the largest have no weight, and the result lies
between the smallest and the largest of the others' values, each held to the same roundings."""
import numpy as np
import pytest
import torch

from oracle import efim_kv4_oracle as orc
from tests.test_gpu_kv4_attn import Case, _f64

pytestmark = pytest.mark.gpu
SHAPES = [(32, 8, 128), (28, 4, 128), (8, 8, 64), (24, 1, 64), (16, 1, 128)]


def _rows(case):
    """(query row in fp64, its keys and values, its result and lse)"""
    hq, hkv, d = case.shape
    k_pool, v_pool = case.held()
    q, out, lse, row = _f64(case.q), _f64(case.out), case.lse.double().cpu().numpy(), 0
    for s, (c, n) in enumerate(zip(case.ctx, case.new)):
        pages = case.table[s, :-(-c // 16)].numpy()
        for i in range(n):
            for h in range(hq):
                k, v = (x[pages, h * hkv // hq].reshape(-1, d)[:c - n + i + 1] for x in (k_pool, v_pool))
                yield q[row, h], k, v, out[row, h], lse[row, h]
            row += 1


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("new", [(1, 1, 1), (3, 1, 5)])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 27, 2.0 ** 33, 2.0 ** 40])
def test_one_dim(hq, hkv, d, new, size):
    case = Case(hq, hkv, d, [300, 40, 500], new, seed=hq)
    keep = torch.nn.functional.one_hot(torch.randint(d, case.q.shape[:2], generator=torch.Generator().manual_seed(d)), d).bool().cuda()
    case.q.copy_(torch.where(keep, case.q.sign() * (1 + case.q.abs()) * size, 0))
    case.run()
    assert case.status.item() == 0
    for q, k, v, out, lse in _rows(case):
        (want,), (want_lse,), (size_of,), _ = orc.attend(q[None], k, v, [len(k)], d ** -0.5)
        assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -15) * size_of + 2.0 ** -36 * np.abs(v).sum(0)).all()
        assert abs(lse - want_lse) <= 2.0 ** -21 * abs(want_lse)


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("new", [(1, 1, 1), (3, 1, 5)])
@pytest.mark.parametrize("ctx", [(300, 40, 500), (2500, 9, 700)])
@pytest.mark.parametrize("size", [2.0 ** 18, 2.0 ** 25, 2.0 ** 31, 2.0 ** 38])
def test_all_dims(hq, hkv, d, new, ctx, size):
    case = Case(hq, hkv, d, ctx, new, seed=hq, q_size=size)
    case.run()
    assert case.status.item() == 0 and torch.isfinite(case.out.float()).all() and torch.isfinite(case.lse).all()
    for q, k, v, out, lse in _rows(case):
        s = k @ q * d ** -0.5
        off = 2.0 ** -16 * (np.abs(k) @ np.abs(q)).max() * d ** -0.5 + 2.0 ** -22 * np.abs(s).max()
        near = v[s >= s.max() - 2 * off - 40]
        room = (2.0 ** -8 + 2.0 ** -11) * np.abs(near).max(0) + 2.0 ** -36 * np.abs(v).sum(0)
        assert (out >= near.min(0) - room).all() and (out <= near.max(0) + room).all()
        assert abs(lse - s.max()) <= off + np.log(len(k)) + 1


def test_small_and_large_scores_in_one_tile():
    """A row's bits are its own: beside rows of large scores as beside others."""
    case, clean = (Case(16, 1, 128, [700, 90], [2, 3], seed=6) for _ in range(2))
    case.q[:, ::3] *= 2.0 ** 30
    case.run()
    clean.run()
    same = torch.ones(16, dtype=torch.bool)
    same[::3] = False
    assert torch.equal(case.out[:, same].view(torch.int16), clean.out[:, same].view(torch.int16))
    assert torch.isfinite(case.out.float()).all()
