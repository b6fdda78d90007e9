"""Equals in efim_verify_drafts: the lowest place among equal maxima (greedy), and among equal results of the race, wherever the
places stand - in one vector, in lanes, warps, CTAs or pieces of a row - and in both forms of the call.  Whole numbers, equal."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import Step

pytestmark = pytest.mark.gpu
ONE, TWO = dict(bf16=30000, f32=15001, probs=15000), dict(bf16=70000, f32=70001, probs=70000)      # places: one kernel, two kernels
APART = [1, 2, 3, 4, 7, 8, 9, 31, 32, 256, 248, 512, 1024, 2040, 2048, 4096, 8192, 10048, 16384, 20000]


def _places(rng, vocab):
    """Two to five places, the distances between them those of vectors, lanes, warps, CTAs and pieces."""
    while True:
        at = int(rng.integers(0, vocab)) + np.concatenate([[0], rng.choice(APART, rng.integers(1, 5))]).cumsum()
        at = at[at < vocab]
        if len(at) > 1:
            return at.tolist()


def _step(batch, vocab, kind, dense, greedy, layout, seed):
    """Sequences of two rows.  Row r's equals: step.equal[r]."""
    stride, offset = (vocab, 0) if layout == "packed" else (vocab + 3, 1)
    step = Step([2] * batch, vocab, kind, dense, None, seed, stride, offset, greedy)
    rng = np.random.default_rng(seed)
    step.equal = [_places(rng, vocab) for _ in range(2 * batch)]
    step.target[:] = -20.0
    for row, at in zip(step.target, step.equal):
        row[at] = 1.5
    if kind == "probs":
        step.target = (np.exp(step.target.astype(np.float64)) / 32.0).astype(np.float32)
    if not greedy:
        step.noise = np.maximum(step.noise, 0.01).astype(np.float32)
    return step


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [3, 36])
@pytest.mark.parametrize("layout", ["packed", "apart"])
@pytest.mark.parametrize("form", [ONE, TWO])
def test_equal_maxima(form, layout, batch, kind):
    """Every second sequence drafts the lowest of the equals, which is accepted, the others the next one, which is not."""
    for seed in range(4):
        step = _step(batch, form[kind], kind, False, True, layout, 50 + seed)
        for s in range(batch):
            step.tokens[2 * s + 1] = step.equal[2 * s][s % 2]
        assert step.check() == (batch + 1) // 2
        assert step.next.tolist() == [step.equal[2 * s + 1 - s % 2][0] for s in range(batch)]
    step.target[:] = 0.25                               # a row of nothing but equals
    step.tokens[:] = 0
    assert step.check() == batch and step.next.tolist() == [0] * batch


@pytest.mark.parametrize("kind", ["bf16", "f32", "probs"])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("batch", [3, 36])
@pytest.mark.parametrize("layout", ["packed", "apart"])
@pytest.mark.parametrize("form", [ONE, TWO])
def test_equal_results_of_the_race(form, layout, batch, dense, kind):
    """Equal probabilities over equal random numbers.  A third of the sequences accept their draft and race over the last row; the
    others' is refused: one that is none of the equals, or the lowest of them, which then does not run if it was certain."""
    for seed in range(2):
        step = _step(batch, form[kind], kind, dense, False, layout, 70 + seed)
        want = []
        for s in range(batch):
            first, last = step.equal[2 * s], step.equal[2 * s + 1]
            other = next(j for j in range(step.vocab) if j not in first)
            step.tokens[2 * s + 1] = [first[-1], other, first[0]][s % 3]
            step.uniform[2 * s] = 0.0 if s % 3 == 0 else 0.999
            if dense:                                   # (p - q)+ is the same at the equals
                step.q[2 * s] = 0
                step.q[2 * s, first] = 2.0 ** -6
                step.q[2 * s, step.tokens[2 * s + 1]] = 1.0 if s % 3 else 2.0 ** -6
            step.noise[s, last if s % 3 == 0 else first] = 0.5
            left = last if s % 3 == 0 else first[1:] if s % 3 == 2 else first
            want.append(left[0])
        step.run()
        assert int(step.status.item()) == 0
        assert step.accepted.tolist() == [int(s % 3 == 0) for s in range(batch)]
        assert step.next.tolist() == want == [step.want(s)[1] for s in range(batch)]
    step.target[:] = 2.0 ** -20 if kind == "probs" else 0.5          # everything equal
    step.noise[:] = 0.75
    if dense:
        step.q[:] = 0
        step.q[:, 0] = 1.0
    step.tokens[:] = 0
    step.uniform[:] = 0.999
    step.run()
    assert step.accepted.tolist() == [0] * batch and step.next.tolist() == [1] * batch


def test_inputs_have_equals():
    """What the two tests above put into rows."""
    step = _step(3, ONE["bf16"], "bf16", False, True, "packed", 50)
    for row, at in zip(step.target, step.equal):
        assert len(at) > 1 and np.flatnonzero(row == row.max()).tolist() == sorted(at) == at
