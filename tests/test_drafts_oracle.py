"""Pins of the oracle of drafted steps (CPU): closed forms, hand examples, and the rule's point - what is emitted is distributed as
the target."""
import math

import numpy as np
import pytest

from oracle import efim_drafts_oracle as orc


def test_norm_closed_forms():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    assert np.allclose(orc.qk_norm(x, None, 0.0), x / 2.5, rtol=1e-15)          # root mean square sqrt(25 / 4)
    w = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(orc.qk_norm(x, w, 0.0, 1.0), x / 2.5 * (w + 1), rtol=1e-15)
    assert np.array_equal(orc.qk_norm(np.zeros((1, 4)), w, 1e-6), np.zeros((1, 4)))
    y = np.random.default_rng(0).standard_normal((5, 64))
    assert np.allclose((orc.qk_norm(y, None, 0.0) ** 2).mean(-1), 1.0, rtol=1e-12)
    assert np.allclose(orc.qk_norm(7 * y, None, 0.0), orc.qk_norm(y, None, 0.0), rtol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_the_complex_product(interleaved):
    rng = np.random.default_rng(1)
    y, angle = rng.standard_normal((3, 8)), rng.uniform(-9, 9, 4)
    got, size = orc.rotate(y, np.concatenate([np.cos(angle), np.sin(angle)]), interleaved)
    pairs = [(2 * f, 2 * f + 1) if interleaved else (f, f + 4) for f in range(4)]
    for f, (a, b) in enumerate(pairs):
        z = (y[:, a] + 1j * y[:, b]) * np.exp(1j * angle[f])
        assert np.allclose(got[:, a], z.real, atol=1e-14) and np.allclose(got[:, b], z.imag, atol=1e-14)
    assert (size >= np.abs(got) - 1e-15).all()


def test_lookup_by_hand():
    #             0  1  2  3  4  5  6  7  8
    h = [5, 6, 7, 1, 6, 7, 2, 6, 7]
    assert orc.draft_lookup(h, 1, 3, 2) == [2, 6]             # "6 7" before place 6 (later than the one before place 3)
    assert orc.draft_lookup(h + [1], 1, 3, 3) == [6, 7, 2]    # "6 7 1" is longer than "1" alone
    assert orc.draft_lookup([4, 9, 4], 1, 4, 5) == [9, 4, 9, 4, 9]
    assert orc.draft_lookup([3, 3, 3, 3], 1, 2, 3) == [3, 3, 3]
    assert orc.draft_lookup([1, 2, 3], 1, 4, 2) is None
    assert orc.draft_lookup([1, 2, 1], 2, 4, 2) is None       # one token agrees, two are asked for
    assert orc.draft_lookup([], 1, 2, 2) is None and orc.draft_lookup([1], 1, 2, 2) is None


@pytest.mark.parametrize("dense", [False, True])
def test_emitted_first_token_is_distributed_as_the_target(dense):
    """First token that a step with one draft emits, over many draws: each frequency within 5 standard deviations of p."""
    rng = np.random.default_rng(3)
    v, draws = 6, 40000
    p_logits = rng.standard_normal(v)
    p = orc.distribution(p_logits, 0.8)
    q = orc.distribution(rng.standard_normal(v), 1.0) if dense else None
    counts = np.zeros(v)
    for _ in range(draws):
        draft = int(rng.choice(v, p=q)) if dense else int(rng.integers(v))     # a certain draft may be any token
        acc, nxt, logs, _ = orc.verify([0, draft], [p_logits, np.zeros(v)], rng.random(2), rng.exponential(size=v),
                                       None if q is None else [q, q], 0.8)
        first = draft if acc else nxt
        counts[first] += 1
        assert abs(logs[0] - math.log(p[first])) < 1e-12 and len(logs) == acc + 1
    assert (np.abs(counts / draws - p) < 5 * np.sqrt(p * (1 - p) / draws)).all()


def test_verification_by_hand():
    e = [1.0, 1.0, 1.0]
    p = [[0.5, 0.3, 0.2], [0.1, 0.1, 0.8], [0.2, 0.7, 0.1]]
    q = [[0.2, 0.6, 0.2], [0.3, 0.3, 0.4], None]
    assert orc.verify([9, 0, 2], p, [0.99, 0.99, 0], e, q, probs=True)[:2] == (2, 1)
    assert orc.verify([9, 1, 2], p, [0.6, 0.0, 0], e, q, probs=True)[:2] == (0, 0)         # 0.36 >= 0.3; only token 0 is left
    assert orc.verify([9, 1, 2], p, [0.4, 0.0, 0], e, q, probs=True)[:2] == (2, 1)         # 0.24 < 0.3
    assert orc.verify([9, 0, 1], p, [0.4, 0.1, 0], e, None, probs=True)[:2] == (1, 2)      # a certain draft: 0.1 >= 0.1; without it 2
    assert orc.verify([9, 0], [[0, 0], [0, 0]], [0, 0], None)[:2] == (1, 0)                # greedy, the lowest of equals
    assert orc.verify([9, 1], [[0, 0], [0, 0]], [0, 0], None)[:2] == (0, 0)
    inf = math.inf
    assert orc.verify([9], [[-inf, -inf]], [0], [1, 1])[:2] == (0, -1)
    assert orc.verify([9], [[-inf, 2]], [0], [1, 1])[:3] == (0, 1, [0.0])
    assert orc.verify([9], [[inf, 2, inf]], [0], [5, 1, 1])[:2] == (0, 2)
    assert orc.verify([9], [[math.nan, 2]], [0], [1, 1])[:2] == (0, -1)
    assert orc.verify([], [], [], [1])[:2] == (0, -1)
    same = [[0.25, 0.75], [1.0, 0.0]]
    assert orc.verify([9, 1], same, [1.0, 0], [1, 1], same, probs=True)[:2] == (0, 1)      # p = q leaves nothing: p itself
