"""The calls of a drafted step at the sizes where 32-bit arithmetic ends."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from tests.test_gpu_verify import Step

pytestmark = pytest.mark.gpu


def test_more_than_2_to_31_threads():
    """2^24 rows and some, a CTA each (2^32 threads and some), over a workspace of ones: what the CTAs meet in is cleared all the
    same, and nothing else is.  Three hundred sequences: two kernels."""
    step = Step([2] * 300, 64, "bf16", False, seed=31)
    step.tokens[599], step.uniform[598] = step.target[598].argmin(), 0.999          # the last sequence stops at its first row
    step.temperature[299] = 0.8
    step.run()
    want = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
    assert int(want[0].sum()) > 75 and int(want[0][299]) == 0
    indptr, tokens, target, accepted, following = step.main
    rows = (1 << 24) + 700

    def longer(x):
        return torch.cat([x, torch.zeros((rows - len(x),) + x.shape[1:], dtype=x.dtype, device="cuda")])
    indptr[-1] = rows
    target = longer(target)
    need = efim.efim_verify_workspace_bytes(300, target)
    assert need > 0
    guard = torch.full((4096 + need + 4096,), 255, dtype=torch.uint8, device="cuda")
    step.args.update(uniform=longer(step.args["uniform"]), workspace=guard[4096:4096 + need])
    for t in (accepted, following, step.out):
        t.fill_(-5)
    efim.efim_verify_drafts(indptr, longer(tokens), target, accepted, following, **step.args)
    torch.cuda.synchronize()
    assert int(step.status.item()) == 0
    for x, y in zip(want, (accepted, following, step.out, step.logs)):
        assert torch.equal(x, y)
    assert bool((guard[:4096] == 255).all()) and bool((guard[4096 + need:] == 255).all())


@pytest.mark.parametrize("vocab", [300000, 300001])
@pytest.mark.parametrize("dense", [False, True])
def test_races_that_others_raise(dense, vocab):
    """One sequence, as many CTAs as there can be on one race, with results that rise along the row and fall along it: CTAs begin
    while others have raised the best already.  Whatever each of them saw, the result is the definition's, every time."""
    for flip in (False, True):
        step = Step([1], vocab, "f32", False, None, seed=37)
        if dense:                                       # two rows: the first refuses its draft
            step = Step([2, 1], vocab, "f32", True, None, seed=37)
            step.tokens[1] = step.target[0].argmin()
            step.q[0] *= 0.5
            step.q[0, step.tokens[1]] = 0.5
            step.uniform[0] = 0.999
        step.target[:] = np.random.default_rng(41).uniform(-1, 1, step.target.shape)
        place = np.arange(vocab)[::-1] if flip else np.arange(vocab)
        step.noise[:] = 1.0 / (1.0 + place) * np.random.default_rng(43).uniform(0.9, 1.1, step.noise.shape)
        step.check()
        want = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
        for _ in range(50):
            step.again()
        torch.cuda.synchronize()
        for x, y in zip(want, (step.accepted, step.next, step.out, step.logs)):
            assert torch.equal(x, y)
