"""efim_draft_lookup against the definition, place by place: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_drafts_oracle as orc

pytestmark = pytest.mark.gpu


def _run(hist, lens, lo, hi, k, stride=None, offset=0):
    b, top = hist.shape
    stride = stride or top
    buf = torch.full((offset + stride * b + 8,), -7, dtype=torch.int32, device="cuda")
    view = buf[offset:].as_strided((b, top), (stride, 1))
    view.copy_(torch.from_numpy(hist))
    drafts = torch.full((b, k), -99, dtype=torch.int32, device="cuda")
    n = torch.full((b,), -99, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    efim.efim_draft_lookup(view, torch.tensor(lens, dtype=torch.int32, device="cuda"), lo, hi, drafts, n, status)
    torch.cuda.synchronize()
    return drafts.cpu().numpy(), n.cpu().numpy(), int(status.item())


def _check(hist, lens, lo, hi, k, **layout):
    drafts, n, status = _run(hist, lens, lo, hi, k, **layout)
    assert status == 0
    found = 0
    for s in range(len(lens)):
        want = orc.draft_lookup(hist[s, :lens[s]].tolist(), lo, hi, k)
        assert (n[s], drafts[s].tolist()) == ((k, want) if want else (0, [-1] * k)), (s, lens[s])
        found += want is not None
    return found


@pytest.mark.parametrize("vocab", [2, 7, 1000])
@pytest.mark.parametrize("lo,hi,k", [(1, 1, 1), (1, 4, 5), (2, 3, 8), (3, 32, 20)])
def test_ragged_histories(vocab, lo, hi, k):
    rng = np.random.default_rng(vocab + hi)
    lens = [0, 1, 2, 3, 4, 5, 31, 32, 33, 100, 511, 700, 1023]
    hist = rng.integers(0, vocab, (len(lens), 1024)).astype(np.int32)
    assert _check(hist, lens, lo, hi, k) > 0 or (vocab == 1000 and lo > 1)


@pytest.mark.parametrize("batch,top", [(1, 5000), (3, 16384), (5, 17001), (150, 2500), (700, 300), (1, 40000)])
def test_sizes_of_the_batch(batch, top):
    """Every number of CTAs a sequence; what is found stands in any of their parts."""
    rng = np.random.default_rng(top)
    hist = rng.integers(0, 100000, (batch, top)).astype(np.int32)
    lens = rng.integers(top // 2, top + 1, batch).tolist()
    for s, n in enumerate(lens):
        if s % 5 != 4:
            e = int(rng.integers(3, n - 3))
            hist[s, e - 3:e] = hist[s, n - 3:n] = rng.integers(0, 100000, 3)
    assert _check(hist, lens, 1, 3, 4) >= batch * 3 // 5


@pytest.mark.parametrize("stride,offset", [(1001, 0), (1003, 1), (1002, 3), (1024, 2)])
def test_rows_at_any_place(stride, offset):
    rng = np.random.default_rng(stride)
    hist = rng.integers(0, 20, (6, 1001)).astype(np.int32)
    assert _check(hist, [1001, 1000, 7, 999, 2, 64], 1, 8, 6, stride=stride, offset=offset) > 0


def test_repetitions():
    hist = np.stack([np.zeros(400, np.int32), np.tile([1, 2], 200), np.arange(400), np.tile(np.arange(100), 4)]).astype(np.int32)
    assert _check(hist, [400, 399, 400, 400], 1, 32, 9) == 3


@pytest.mark.parametrize("hi", [1, 2, 3, 32])
@pytest.mark.parametrize("batch", [2, 200])
def test_long_repetitions(batch, hi):
    """Every place agrees, or every second, or all but the newest; the longest agreement may be an old one."""
    rows = np.zeros((batch, 9001), np.int32)
    rows[1::4, 1::2] = 3
    rows[2::4] = np.random.default_rng(5).integers(0, 2, rows[2::4].shape)
    rows[3::4] = np.arange(9001)
    rows[3::4, 40:45] = rows[3::4, 8990:8995] = 7, 8, 9, 8, 9
    rows[3::4, 8996:] = 7, 8, 9, 8, 9
    lens = [9001, 9000, 8999, 9001] * (batch // 4) + [9001, 8999, 9001][:batch % 4]
    assert _check(rows, lens, 1, hi, 11, stride=9003, offset=1) == batch


def test_lengths_outside_the_rows():
    hist = np.tile(np.array([[4, 5, 6, 4]], np.int32), (3, 1))
    drafts, n, status = _run(hist, [-3, 9, 4], 1, 2, 2)
    assert status == 2 and n.tolist() == [0, 2, 2] and drafts.tolist() == [[-1, -1], [5, 6], [5, 6]]


def test_offsets_past_32_bits():
    stride = (1 << 31) + 5
    buf = torch.zeros(stride + 64, dtype=torch.int32, device="cuda")
    view = buf.as_strided((2, 50), (stride, 1))
    hist = np.random.default_rng(0).integers(0, 5, (2, 50)).astype(np.int32)
    view.copy_(torch.from_numpy(hist))
    drafts = torch.empty(2, 3, dtype=torch.int32, device="cuda")
    n = torch.empty(2, dtype=torch.int32, device="cuda")
    efim.efim_draft_lookup(view, torch.tensor([50, 50], dtype=torch.int32, device="cuda"), 1, 4, drafts, n)
    torch.cuda.synchronize()
    assert drafts.tolist() == [orc.draft_lookup(h.tolist(), 1, 4, 3) for h in hist]
