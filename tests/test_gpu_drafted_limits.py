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


def _look(history, num_drafts, length=None, lo=1, hi=4):
    drafts = torch.full((1, num_drafts), -9, dtype=torch.int32, device="cuda")
    n = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    length = torch.tensor([history.shape[1] if length is None else length], dtype=torch.int32, device="cuda")
    efim.efim_draft_lookup(history, length, lo, hi, drafts, n, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return drafts, int(n.item())


@pytest.mark.parametrize("offset", [0, 1])
def test_the_longest_history(offset):
    """2^31 - 1 tokens, aligned and not; the place to be found is one of the first, or the last of all."""
    size = (1 << 31) - 1
    buf = torch.zeros(size + offset, dtype=torch.int32, device="cuda")
    history = buf[offset:].view(1, size)
    history[0, 3], history[0, 4], history[0, size - 1] = 5, 9, 5
    drafts, n = _look(history, 4)
    assert n == 4 and drafts.tolist() == [[9, 0, 0, 0]]
    for back in (2, 3, 4):                              # of one to three tokens behind the last vector
        history[0, size - back] = 5
        drafts, n = _look(history, 4, hi=1)
        assert n == 4 and drafts.tolist() == [(([0] * (back - 2) + [5]) * 4)[:4]]
        history[0, size - back] = 0


def test_the_most_drafts():
    history = torch.tensor([[7, 8, 8, 8]], dtype=torch.int32, device="cuda")
    drafts, n = _look(history, (1 << 31) - 1)
    assert n == (1 << 31) - 1 and bool((drafts == 8).all())
    drafts, n = _look(history, (1 << 31) - 1, length=1)
    assert n == 0 and bool((drafts == -1).all())


@pytest.mark.parametrize("vocab", [2000, 70000])
def test_the_longest_output(vocab):
    """2^31 - 1 places for what a sequence goes on with, in both forms."""
    step = Step([3], vocab, "bf16", False, seed=47).run()
    width = (1 << 31) - 1
    out = torch.full((1, width), -9, dtype=torch.int32, device="cuda")
    step.args.update(out_tokens=out, out_logprobs=None)
    step.again()
    torch.cuda.synchronize()
    n = int(step.accepted[0]) + 1
    assert out[0, :n].tolist() == step.out[0, :n].tolist() and bool((out[0, n:] == -1).all())


@pytest.mark.parametrize("vocab", [2000, 70000])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_no_rows_at_all(kind, vocab):
    """Nothing is read of a call without rows but the (empty) row ranges: not the random numbers, whose address and rows are not
    looked at either."""
    import ctypes
    from paper_2505_21889_b200 import binding as B
    indptr = torch.zeros(3, dtype=torch.int32, device="cuda")
    accepted, following = torch.full((2, 2), -9, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    few = torch.ones(8, device="cuda")
    lib = efim.load_library()
    size = lib.efim_verify_workspace_bytes(2, 0, vocab, kind)
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    desc = B._VerifyDesc(batch=2, total_rows=0, vocab=vocab, target_kind=kind, d_row_indptr=indptr.data_ptr(),
                         d_noise=few.data_ptr() + 2, noise_stride=1 << 40)
    assert lib.efim_verify_drafts(ctypes.byref(desc), accepted.data_ptr(), following.data_ptr(), None, None, 0,
                                  ws.data_ptr() if size else None, size, status.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert accepted.tolist() == [0, 0] and following.tolist() == [-1, -1] and int(status.item()) == 0


@pytest.mark.parametrize("vocab", [3000, 70000])
@pytest.mark.parametrize("operand", ["target", "draft_probs", "noise"])
def test_rows_far_apart(operand, vocab):
    """2^30 elements from one row to the next, so that the third is past 2^31 of them, for one operand at a time: the same bits as
    packed."""
    step = Step([3, 1, 2, 3], vocab, "bf16", True, seed=23).run()
    assert int(step.accepted.sum()) >= 2
    want = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
    rows = step.main[2] if operand == "target" else step.args[operand]
    buf = torch.empty((len(rows) - 1 << 30) + vocab, dtype=rows.dtype, device="cuda")
    far = buf.as_strided(rows.shape, (1 << 30, 1))
    far.copy_(rows)
    if operand == "target":
        step.main = step.main[:2] + (far,) + step.main[3:]
    else:
        step.args[operand] = far
    for t in (step.accepted, step.next, step.out):
        t.fill_(-5)
    step.again()
    torch.cuda.synchronize()
    for x, y in zip(want, (step.accepted, step.next, step.out, step.logs)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [3000, 70000])
def test_small_probabilities_that_are_left(vocab, kind):
    """(p - q)+ leaves one place of a probability between 2^-124 and 2^-40, 2e-5 of which is more than its q.  An fp32 probability there is
    within 1.1e-5 of p: two roundings of an exponent below 128 (126 * 2^-24 and 2^-18), times ln 2, and 1e-6 for the exponential, the
    sum and the division."""
    step = Step([2] * 40, vocab, kind, True, None, seed=53)
    rng = np.random.default_rng(59)
    step.target[:] = rng.uniform(-85.0, -28.0, step.target.shape)
    step.target[:, [5, 9]] = 0.0
    if kind == "bf16":
        step.target = torch.from_numpy(step.target).bfloat16().float().numpy()
    places = rng.integers(10, vocab, 40)
    for s, j in enumerate(places):
        p = np.exp(step.target[2 * s].astype(np.float64))
        p /= p.sum()
        step.q[2 * s] = 1.01 * p
        step.q[2 * s, j] = p[j] * (1 - 2e-5)
        step.q[2 * s, 5], step.q[2 * s, 9] = 1.0, 0.6
        step.tokens[2 * s + 1], step.uniform[2 * s] = 5, 0.999
    step.run()
    assert int(step.status.item()) == 0 and step.accepted.tolist() == [0] * 40
    assert step.next.tolist() == places.tolist()
