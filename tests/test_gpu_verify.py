"""efim_verify_drafts against the float64 definition: the same decisions wherever they are further than 1e-5 from going the other
way (fp32 probabilities of these rows are within 2e-6), which all of these inputs are - asserted, with the oracle's margin.

Tolerance of a log-probability: (x - max) / T below 100 in size, two roundings (1.2e-5); the logarithm of a sum of up to 1e5
exponentials with 2^-22 each and at most 512 additions in a chain (3e-5, all roundings one way): 5e-5."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_drafts_oracle as orc

pytestmark = pytest.mark.gpu
BAD_POSITION, BAD_TOKEN, NO_TOKEN = 2, 8, 16
LOG_TOL, MARGIN = 5e-5, 1e-5
WIDE = 70000                                            # rows of more than 64 KB: two kernels


class Step:
    """Rows with one likely token, drafts that mostly are that token, or draws of a distribution near the target's."""

    def __init__(self, rows, vocab, kind="bf16", dense=False, temperature="mixed", seed=0, stride=None, offset=0, greedy=False):
        rng = np.random.default_rng([seed, vocab, sum(rows)])
        b, r = len(rows), sum(rows)
        self.rows, self.vocab, self.kind, self.dense = rows, vocab, kind, dense
        self.indptr = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        logits = (2.5 * rng.standard_normal((r, vocab))).astype(np.float32)
        likely = rng.integers(0, vocab, r)
        lift = np.log(vocab) + 3.1 + rng.uniform(-1, 3, r)
        logits[np.arange(r), likely] = lift
        if kind == "bf16":
            logits = torch.from_numpy(logits).bfloat16().float().numpy()
        self.target = logits
        if kind == "probs":
            self.target = np.stack([orc.distribution(x, 1.0) for x in logits]).astype(np.float32) if r else logits
        drawn = np.where(rng.random(r) < 0.85, likely, rng.integers(0, vocab, r))
        self.q = None
        if dense:
            near = logits + 0.5 * rng.standard_normal((r, vocab))
            self.q = np.stack([orc.distribution(x, 1.0) for x in near]).astype(np.float32) if r else near.astype(np.float32)
            drawn = np.array([(x / rng.exponential(size=vocab)).argmax() for x in self.q], np.int64)
        self.tokens = np.roll(drawn, 1).astype(np.int32)
        self.uniform = rng.random(r).astype(np.float32)
        self.noise = None if greedy else rng.exponential(size=(b, vocab)).astype(np.float32)
        self.temperature = None
        if temperature == "mixed" and kind != "probs":
            self.temperature = rng.uniform(0.6, 1.0, b).astype(np.float32)
            self.temperature[rng.random(b) < 0.2] = 0.0
        self.stride, self.offset = stride or vocab, offset

    def _matrix(self, x, dtype=torch.float32):
        """On the device, rows `stride` apart, the first `offset` values behind an aligned address; NaN around them."""
        if x is None:
            return None
        buf = torch.full((self.offset + self.stride * len(x) + 8,), float("nan"), dtype=dtype, device="cuda")
        view = buf[self.offset:].as_strided(x.shape, (self.stride, 1))
        view.copy_(torch.from_numpy(x))
        return view

    def run(self, out=True, stream=None):
        dev = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
        b = len(self.rows)
        self.accepted, self.next = (torch.full((b,), -99, dtype=torch.int32, device="cuda") for _ in range(2))
        width = max(self.rows + [1]) + 2
        self.out = torch.full((b, width), -99, dtype=torch.int32, device="cuda") if out else None
        self.logs = torch.full((b, width), float("nan"), device="cuda") if out else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.args = dict(uniform=dev(self.uniform), noise=self._matrix(self.noise), draft_probs=self._matrix(self.q),
                         temperature=dev(self.temperature), target_is_probs=self.kind == "probs", out_tokens=self.out,
                         out_logprobs=self.logs, status=self.status, stream=stream)
        self.main = (dev(self.indptr), dev(self.tokens),
                     self._matrix(self.target, torch.bfloat16 if self.kind == "bf16" else torch.float32), self.accepted, self.next)
        self.again()
        torch.cuda.synchronize()
        return self

    def again(self):
        efim.efim_verify_drafts(*self.main, **self.args)

    def want(self, s):
        a, b = self.indptr[s], self.indptr[s + 1]
        return orc.verify(self.tokens[a:b], self.target[a:b], self.uniform[a:b], None if self.noise is None else self.noise[s],
                          None if self.q is None else self.q[a:b], 1.0 if self.temperature is None else float(self.temperature[s]),
                          self.kind == "probs")

    def check(self, status=0):
        self.run()
        assert int(self.status.item()) == status
        total = 0
        for s in range(len(self.rows)):
            acc, nxt, logs, margin = self.want(s)
            assert margin > MARGIN, (s, margin)
            assert (int(self.accepted[s]), int(self.next[s])) == (acc, nxt), (s, margin)
            emitted = self.tokens[self.indptr[s] + 1:self.indptr[s] + 1 + acc].tolist() + [nxt]
            width = self.out.shape[1]
            assert self.out[s].tolist() == emitted + [-1] * (width - len(emitted)), s
            got = self.logs[s].cpu().numpy()
            assert np.abs(got[:len(logs)] - logs).max() <= LOG_TOL, (s, got, logs)
            assert (got[len(logs):] == 0).all()
            total += acc
        return total


@pytest.mark.parametrize("kind", ["bf16", "f32", "probs"])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("vocab", [1, 5, 37, 1000, 4099, 40000])
def test_ragged_rows(kind, dense, vocab):
    """Numbers of drafts from none on, also sequences without rows; one CTA a sequence up to eight."""
    n = Step([1, 0, 5, 2, 9, 1, 3, 17, 0, 4], vocab, kind, dense, seed=11).check()
    assert n > 0


@pytest.mark.parametrize("batch,vocab", [(20, 16384), (90, 8200), (300, 2500), (700, 300)])
@pytest.mark.parametrize("dense", [False, True])
def test_sizes_of_the_batch(batch, vocab, dense):
    rng = np.random.default_rng(batch)
    n = Step(rng.integers(1, 5, batch).tolist(), vocab, "bf16", dense, seed=3).check()
    assert n > batch // 4


@pytest.mark.parametrize("kind", ["bf16", "f32", "probs"])
@pytest.mark.parametrize("vocab,stride,offset", [(9999, 9999, 0), (9999, 10007, 1), (10000, 10002, 3), (10000, 10008, 0), (8192, 8192, 5)])
def test_rows_at_any_place(kind, vocab, stride, offset):
    """Alignments of every operand; what stands between the rows is not read."""
    Step([3, 1, 6], vocab, kind, True, seed=5, stride=stride, offset=offset).check()
    Step([3, 1, 6], vocab, kind, False, seed=6, stride=stride, offset=offset).check()


@pytest.mark.parametrize("kind,vocab,stride,offset,dense", [("bf16", 131072, 131072, 0, False), ("bf16", 131072, 131072, 0, True),
                                                            ("f32", 70001, 70001, 0, False), ("bf16", 99999, 100001, 3, False)])
def test_many_rows(kind, vocab, stride, offset, dense):
    """Rows of more than 64 KB; some sequences of many more rows than the others, some of none."""
    rng = np.random.default_rng(vocab)
    rows = rng.integers(0, 6, 100).tolist() + [17, 0, 1, 40]
    step = Step(rows, vocab, kind, dense, seed=29, stride=stride, offset=offset)
    # a sequence that accepts everything, past the average number of rows
    a = int(step.indptr[-2])
    step.tokens[a + 1:] = step.target[a:-1].argmax(1)
    step.uniform[a:] = 1e-7
    if dense:
        step.q[a:] = 1.0 / vocab
    n = step.check()
    assert n > 100 and int(step.accepted[-1]) == 39
    first = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
    for _ in range(3):
        step.again()
    torch.cuda.synchronize()
    for x, y in zip(first, (step.accepted, step.next, step.out, step.logs)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("vocab", [30000, WIDE])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_greedy(kind, vocab):
    """No noise at all: every sequence greedy, ties to the lowest place (bf16 logits have many)."""
    step = Step([4, 1, 7, 2], vocab, kind, False, None, seed=9, greedy=True)
    step.target = np.round(step.target)
    lowest = step.target.argmax(1)
    step.tokens[1:] = lowest[:-1]
    step.tokens[7] = 17                                 # the second draft of the third sequence is another one
    assert step.check() == 3 + 1 + 1


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,place", [(2000, 7), (WIDE, WIDE - 3)])
def test_statuses_and_rows_without_a_token(vocab, place, kind):
    step = Step([3, 3, 3, 2, 1], vocab, kind, False, None, seed=2)
    step.tokens[[1, 2]] = step.target[[0, 1]].argmax(1)
    step.uniform[:] = 1e-6
    step.target[2] = -np.inf                            # sequence 0's last row
    step.target[4, place] = np.nan                          # sequence 1's second
    step.tokens[4] = step.target[3].argmax()
    step.tokens[7] = vocab                              # sequence 2's first draft
    step.target[10, 5] = np.inf                         # sequence 3's second
    step.target[10, 9] = np.inf
    step.tokens[10] = step.target[9].argmax()
    step.target[11] = -np.inf
    step.target[11, 1234] = -3.0
    step.run()
    assert int(step.status.item()) == BAD_TOKEN | NO_TOKEN
    assert step.accepted.tolist() == [2, 1, 0, 1, 0]
    want = [step.want(s) for s in range(5)]
    assert step.next.tolist() == [w[1] for w in want] and want[0][1] == want[1][1] == -1 and want[4][1] == 1234
    assert want[3][1] in (5, 9) and abs(float(step.logs[3, 1]) - np.log(0.5)) < 1e-6 and float(step.logs[4, 0]) == 0
    for s, w in enumerate(want):
        assert np.abs(step.logs[s, :len(w[2])].cpu().numpy() - w[2]).max() <= LOG_TOL


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5000, WIDE])
@pytest.mark.parametrize("value", [-3.0e38, -1e9])
def test_masks_of_low_finite_values(value, vocab, kind):
    step = Step([2, 1], vocab, kind, False, None, seed=4)
    for row in range(3):
        keep = [11 + row, 17, 4000]
        masked = np.full(vocab, value, np.float32)
        masked[keep] = [1.0, 2.0, 0.5]
        step.target[row] = masked
    step.check()
    step.target[:] = value                              # nothing but the mask: all equal
    step.run()
    assert int(step.status.item()) == 0 and abs(float(step.logs[1, 0]) + np.log(vocab)) < LOG_TOL


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [3000, WIDE])
def test_small_temperatures_and_infinite_masks(vocab, kind):
    step = Step([3, 1, 2], vocab, kind, False, None, seed=13)
    step.target[:, 100:] = -np.inf
    step.tokens[1:] = step.target.argmax(1)[:-1]
    step.temperature = np.array([1e-30, 1e-6, 1e-39], np.float32)
    step.run()
    assert int(step.status.item()) == 0 and step.accepted.tolist() == [2, 0, 1]
    assert step.next.tolist() == step.target.argmax(1)[[2, 3, 5]].tolist()
    assert np.abs(step.logs.cpu().numpy()).max() < 1e-6


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [3000, WIDE])
def test_infinite_temperature(vocab, kind):
    """The limit: all that has a probability has the same."""
    step = Step([2, 1], vocab, kind, False, None, seed=15)
    step.target[:, 100:] = -np.inf
    step.tokens[1] = 200                                # masked: refused
    step.temperature = np.array([np.inf, np.inf], np.float32)
    step.run()
    assert int(step.status.item()) == 0 and step.accepted.tolist() == [0, 0]
    assert step.next.tolist() == step.noise[:, :100].argmin(1).tolist()
    assert np.abs(step.logs[:, 0].cpu().numpy() + np.log(100)).max() < LOG_TOL


@pytest.mark.parametrize("vocab", [3000, WIDE])
def test_probabilities_of_nothing(vocab):
    """Rows of zeros; NaN has no probability."""
    step = Step([2, 1, 1], vocab, "probs", False, seed=27)
    step.target[:] = 0
    step.target[2, [5, vocab - 1]] = [np.nan, 0.25]
    step.target[3, 8] = 1.0
    step.run()
    assert int(step.status.item()) == NO_TOKEN and step.accepted.tolist() == [0, 0, 0]
    assert step.next.tolist() == [-1, vocab - 1, 8]
    assert np.abs(step.logs[:, 0].cpu().numpy() - [0, np.log(0.25), 0]).max() < 1e-6


@pytest.mark.parametrize("vocab", [700, WIDE])
def test_a_draft_that_leaves_nothing(vocab):
    """q = p: every draft below u = 1 is accepted; one that is refused all the same falls back on p."""
    step = Step([2, 2], vocab, "probs", True, seed=21)
    step.q = step.target.copy()
    step.uniform[:] = [1.0, 0, 0.999, 0]
    step.run()                                          # (1 * q < p is exact, so the margin of 0 is none)
    assert step.accepted.tolist() == [0, 1] == [step.want(s)[0] for s in (0, 1)]
    assert step.next.tolist() == [step.want(s)[1] for s in (0, 1)] and int(step.status.item()) == 0


@pytest.mark.parametrize("vocab", [500, WIDE])
def test_row_ranges_outside_the_rows(vocab):
    step = Step([2, 3], vocab, "f32", False, seed=1)
    step.run()
    step.indptr[:] = [0, 2, 9]
    step.run()
    assert int(step.status.item()) == BAD_POSITION and step.accepted.tolist()[1] == 0 and step.next.tolist()[1] == -1
    assert step.out[1].tolist() == [-1] * step.out.shape[1]


@pytest.mark.parametrize("vocab", [20000, WIDE])
def test_optional_outputs_and_repeats(vocab):
    step = Step([4, 1, 8], vocab, "bf16", True, seed=17).run()
    want = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
    for _ in range(3):
        for t in (step.accepted, step.next, step.out):
            t.fill_(-5)
        step.again()
        torch.cuda.synchronize()
        for x, y in zip(want, (step.accepted, step.next, step.out, step.logs)):
            assert torch.equal(x, y)                    # the same bits
    bare = Step([4, 1, 8], vocab, "bf16", True, seed=17).run(out=False)
    assert torch.equal(bare.accepted, want[0]) and torch.equal(bare.next, want[1])
    narrow = torch.full((3, 2), -9, dtype=torch.int32, device="cuda")
    step.args.update(out_tokens=narrow, out_logprobs=None)
    step.again()
    torch.cuda.synchronize()
    assert torch.equal(narrow, want[2][:, :2])


def test_other_streams_and_graphs():
    step = Step([4, 2, 6], 9000, "bf16", True, seed=19).run()
    want = [t.clone() for t in (step.accepted, step.next, step.out, step.logs)]
    step.out.fill_(-5)
    # a call that needs a workspace takes one on torch's current stream, so it runs there or brings its own
    wide = Step([2, 3], 50000, "bf16", False, seed=2).run()
    other = torch.cuda.Stream()
    was = wide.out.clone()
    wide.args["stream"] = other
    with pytest.raises(ValueError):
        wide.again()
    other.wait_stream(torch.cuda.current_stream())
    wide.args["workspace"] = torch.empty(efim.efim_verify_workspace_bytes(2, wide.main[2]), dtype=torch.uint8, device="cuda")
    other.wait_stream(torch.cuda.current_stream())
    wide.out.fill_(-5)
    other.wait_stream(torch.cuda.current_stream())
    wide.again()
    other.synchronize()
    assert torch.equal(wide.out, was)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.again()
    side.synchronize()
    assert torch.equal(step.out, want[2])
    step.out.fill_(-5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.again()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(step.out, want[2]) and torch.equal(step.logs, want[3])


def test_offsets_past_32_bits():
    """Rows 2^30 bf16 elements apart, drafts' and random numbers' rows 2^30 floats apart."""
    small = Step([3], 3000, "bf16", True, seed=23).run()
    stride = 1 << 30
    def far(x):
        buf = torch.zeros(stride * (len(x) - 1) + x.shape[1], dtype=x.dtype, device="cuda")
        view = buf.as_strided(x.shape, (stride, 1))
        view.copy_(x)
        return view
    want = [t.clone() for t in (small.accepted, small.next, small.logs)]
    indptr, tokens, target, accepted, nxt = small.main
    small.args.update(draft_probs=far(small.args["draft_probs"]))
    efim.efim_verify_drafts(indptr, tokens, far(target), accepted.fill_(-5), nxt.fill_(-5), **small.args)
    torch.cuda.synchronize()
    for x, y in zip(want, (accepted, nxt, small.logs)):
        assert torch.equal(x, y)
