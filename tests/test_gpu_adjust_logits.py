"""efim_adjust_logits against the float64 definition.

Tolerance, from the arithmetic: a quotient, two products, three sums in fp32, each off by 2^-24 of its result at most, which the sum M of the
terms' magnitudes bounds: 6 * 2^-24 M; and the one rounding to the result's type, 2^-8 (bf16) or 2^-24 (fp32) of it."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_kv4_oracle as orc

pytestmark = pytest.mark.gpu
BAD_POSITION, BAD_TOKEN = 2, 8


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, rows, vocab, lens, dtype=torch.bfloat16, seed=0, pad=0, shift=0, bias=5, mask=True, prompt=True, tokens=True, extra=0):
        rng = np.random.default_rng(seed)
        self.rows, self.vocab, self.lens = list(rows), vocab, list(lens)
        b, r = len(rows), sum(rows) + extra
        x = torch.from_numpy(rng.standard_normal(r * (vocab + pad) + shift) * 3).to(dtype).cuda()
        self.logits = x[shift:].view(r, vocab + pad)[:, :vocab]
        few = rng.integers(0, vocab, (b, 12))
        self.history = np.take_along_axis(few, rng.integers(0, 12, (b, max(lens) + 3)), 1)
        self.prompt = [int(rng.integers(0, n + 1)) for n in lens] if prompt else None
        self.tokens = np.concatenate([rng.choice(few[s], n) for s, n in enumerate(rows)] + [np.zeros(extra)]).astype(int) if tokens else None
        self.repetition, self.presence, self.frequency = (0.5 + rng.random(b)).astype(np.float32), rng.standard_normal(b).astype(np.float32), rng.standard_normal(b).astype(np.float32)
        self.bias = [[(int(rng.integers(0, vocab)), float(np.float32(rng.standard_normal()))) for _ in range(int(rng.integers(0, bias + 1)))] for _ in rows] if bias else None
        self.mask = rng.integers(0, 1 << 32, (r, (vocab + 31) // 32), dtype=np.uint64).astype(np.uint32) if mask else None

    def run(self, in_place=False, out=None, stream=None, **changed):
        self.before = self.logits.clone()
        self.out = self.logits if in_place else torch.full_like(self.before, 7.0) if out is None else out
        self.status = _i32([0])
        args = dict(row_indptr=_i32([0] + np.cumsum(self.rows).tolist()), history=_i32(self.history.tolist()), lengths=_i32(self.lens),
                    prompt_len=_i32(self.prompt) if self.prompt else None, tokens=_i32(self.tokens.tolist()) if self.tokens is not None else None,
                    **{n: torch.from_numpy(getattr(self, n)).cuda() for n in ("repetition", "presence", "frequency")})
        if self.bias is not None:
            flat = [e for entries in self.bias for e in entries]
            args["bias"] = (_i32([0] + np.cumsum([len(e) for e in self.bias]).tolist()), _i32([t for t, _ in flat]),
                            torch.tensor([x for _, x in flat], dtype=torch.float32, device="cuda"))
        if self.mask is not None:
            args["mask"] = torch.from_numpy(self.mask.view(np.int32)).cuda()
        self.args = {**args, **changed}
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        efim.efim_adjust_logits(logits=self.logits, out=None if in_place else self.out, status=self.status, stream=stream, **self.args)

    def check(self, only=None):
        torch.cuda.synchronize()
        step = 2.0 ** -8 if self.logits.dtype == torch.bfloat16 else 2.0 ** -24
        before, got = self.before.double().cpu().numpy(), self.out.double().cpu().numpy()
        row = 0
        for s, n in enumerate(self.rows):
            prompt = self.prompt[s] if self.prompt else 0
            said = self.history[s, prompt:self.lens[s]].tolist()
            for i in range(n):
                if i and self.tokens is not None:
                    said.append(self.tokens[row])
                if only is None or row in only:
                    allowed = None
                    if self.mask is not None:
                        allowed = (self.mask[row][:, None] >> np.arange(32, dtype=np.uint32) & 1).astype(bool).reshape(-1)[:self.vocab]
                    want, size = orc.adjust(before[row], self.history[s, :prompt], said, float(self.repetition[s]), float(self.frequency[s]),
                                            float(self.presence[s]), self.bias[s] if self.bias else [], allowed)
                    with np.errstate(all="ignore"):
                        off = np.abs(got[row] - want) > step * np.abs(want) + 6 * 2.0 ** -24 * size + 1e-40
                    same = (got[row] == want) | (np.isnan(got[row]) & np.isnan(want))
                    bad = ~same & (off | ~np.isfinite(want) | ~np.isfinite(got[row]))
                    assert not bad.any(), (row, np.argwhere(bad)[0], got[row][bad][0], want[bad][0])
                row += 1
        if self.out is not self.logits:
            assert (self.out[row:].float() == 7).all()
        else:
            assert torch.equal(self.out[row:], self.before[row:])


@pytest.mark.parametrize("vocab", [1, 7, 33, 1000, 2048, 2049, 32003, 40000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("in_place", [False, True])
def test_vocabularies(vocab, dtype, in_place):
    case = Case([1, 3, 0, 2], vocab, [20, 1, 5, 40], dtype, seed=vocab, extra=2)
    case.run(in_place)
    case.check()
    assert case.status.item() == 0


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 0), (24, 8), (3, 5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_apart_and_unaligned(pad, shift, dtype):
    case = Case([2, 1], 3000, [9, 300], dtype, pad=pad, shift=shift)
    case.run()
    case.check()
    case.run(in_place=True)
    case.check()


@pytest.mark.parametrize("off", [dict(mask=False), dict(bias=0), dict(prompt=False), dict(tokens=False), dict(mask=False, bias=0)])
def test_parts_left_out(off):
    case = Case([2, 4], 5000, [100, 7], **off)
    case.run()
    case.check()


def test_none_of_the_penalties():
    case = Case([2, 1], 700, [30, 4])
    case.run(repetition=None, presence=None, frequency=None)
    case.repetition, case.presence, case.frequency = np.ones(2), np.zeros(2), np.zeros(2)
    case.check()
    case = Case([2, 1], 700, [30, 4], mask=False)
    case.run(history=None, lengths=None, prompt_len=None, repetition=None, presence=None, frequency=None, bias=None)
    assert torch.equal(case.out, case.logits)


def test_many_sequences():
    rng = np.random.default_rng(0)
    case = Case(rng.integers(0, 4, 700).tolist(), 4500, rng.integers(0, 200, 700).tolist(), seed=2)
    case.run()
    case.check(only={0, 1, 333, 600, 601, 602, sum(case.rows) - 1})


@pytest.mark.parametrize("most,dtype", [(70000, torch.bfloat16), (3, torch.float32)])
def test_long_lists_and_histories(most, dtype):
    """Counts and lists that leave 32-bit words: one token 70,000 times, 40,000 entries, tokens many times among them, the last counts."""
    case = Case([2, 1], 20000, [most, 3], dtype, bias=0)
    case.history[0, :most] = 17
    case.prompt = [1, 0]
    rng = np.random.default_rng(3)
    case.bias = [[(int(t), float(np.float32(x))) for t, x in zip(rng.integers(0, 2000, 40000), rng.standard_normal(40000))], [(5, 1.0), (6, -np.inf), (5, 2.0)]]
    case.frequency = np.array([0.001, 0.5], np.float32)
    case.run()
    case.check()
    assert case.status.item() == 0


@pytest.mark.parametrize("in_place", [False, True])
def test_drafts_of_one_token(in_place):
    """A token that only the drafts bring, several times over; a history that touches more tokens than a slice's list holds."""
    case = Case([7, 3], 40000, [30000, 3], seed=4, bias=0)
    case.history[0, :30000] = np.random.default_rng(1).permutation(40000)[:30000]
    case.history[1] = 5
    case.prompt = [10000, 0]
    case.tokens[:] = [39999] * 3 + [7] * 4 + [39999, 12345, 12345]
    case.run(in_place)
    case.check()
    assert case.status.item() == 0


def test_values_that_are_not_finite():
    case = Case([2], 300, [12], torch.float32, bias=0)
    case.history[0, :4] = [0, 1, 2, 3]
    case.prompt = [0]
    case.logits[0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0])
    case.logits[1, 10:13] = torch.tensor([float("inf"), -float("inf"), float("nan")])
    case.bias = [[(10, -np.inf), (12, 1.0), (11, 3.0)]]
    case.mask[:, 0] |= 0xff
    case.run()
    case.check()
    case.mask[:] = 0
    case.run()
    assert torch.isneginf(case.out).all()


def test_ids_and_lengths_that_do_not_fit():
    case = Case([2, 2], 500, [40, 30], bias=0, mask=False)
    case.history[0, 3], case.history[1, 2], case.tokens[1] = 500, -1, 1 << 30
    case.run()
    assert case.status.item() == BAD_TOKEN
    first = case.out.clone()
    history = case.history.copy()
    lens = list(case.lens)
    case.history[0, 3], case.tokens[1] = 0, 0
    case.run()
    assert not torch.equal(first, case.out) and torch.equal(first[2:], case.out[2:])
    for changed in (dict(lengths=_i32([44, 30])), dict(lengths=_i32([-1, 30])), dict(prompt_len=_i32([41, case.prompt[1]])), dict(prompt_len=_i32([-1, case.prompt[1]]))):
        case.history = np.abs(history) % 500
        case.lens = lens
        case.run(**changed)
        assert case.status.item() == BAD_POSITION, changed
        case.check(only={2, 3})
    # rows beyond what was given, entries beyond the list
    case.run(row_indptr=_i32([0, 2, 9]))
    assert case.status.item() == BAD_POSITION
    case.check()
    case.run(row_indptr=_i32([0, 2, 1]))
    assert case.status.item() == BAD_POSITION and (case.out[2:].float() == 7).all()
    case.run(bias=(_i32([0, 1, 4]), _i32([3, 4]), torch.ones(2, device="cuda")))
    assert case.status.item() == BAD_POSITION
    case.bias = [[(3, 1.0)], []]
    case.check()
    case.run(bias=(_i32([0, 1, 2]), _i32([3, 500]), torch.ones(2, device="cuda")))
    assert case.status.item() == BAD_TOKEN
    case.check()


def test_graph_and_another_stream():
    case = Case([1, 2], 9000, [40, 30])
    case.run(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    case.check()
    first = case.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        efim.efim_adjust_logits(logits=case.logits, out=case.out, status=case.status, **case.args)
    case.out.fill_(7)
    graph.replay()
    assert torch.equal(first.view(torch.int16), case.out.view(torch.int16))


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_far_apart(in_place):
    """Rows 2^30 + 8 elements apart: offsets past 32 bits in bytes and in elements; nothing between the rows is touched."""
    case = Case([2, 3], 1000, [30, 4])
    step = (1 << 30) + 8
    wide = torch.full((4 * step + 1000,), 3.0, dtype=torch.bfloat16, device="cuda")
    far = wide.as_strided((5, 1000), (step, 1))
    far.copy_(case.logits)
    want = torch.empty_like(case.logits)
    case.run(out=want)
    case.check()
    efim.efim_adjust_logits(logits=far, out=None if in_place else (near := torch.empty_like(want)), status=case.status, **case.args)
    assert torch.equal((far if in_place else near).contiguous().view(torch.int16), want.view(torch.int16))
    if not in_place:
        efim.efim_adjust_logits(logits=case.logits, out=far, status=case.status, **case.args)
        assert torch.equal(far.contiguous().view(torch.int16), want.view(torch.int16))
    far.fill_(3.0)
    assert bool((wide[::1021] == 3).all()) and bool((wide[1000:2000] == 3).all()) and case.status.item() == 0
