"""efim_step_tables and efim_release_pages: whole numbers, which have to be the oracle's."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_kv4_oracle as orc

pytestmark = pytest.mark.gpu
BAD_POSITION, NO_PAGE = 2, 0x20


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, cached, new, width, free, seed=0, room=None, holes=True):
        rng = np.random.default_rng(seed)
        self.cached, self.new, self.free = list(cached), list(new), rng.permutation(100000)[:free].tolist()
        self.table = [[(1000 * s + e) if e < -(-c // 16) or (holes and rng.random() < 0.3) else -1 for e in range(width)]
                      for s, c in enumerate(cached)]
        self.room = sum(new) + 5 if room is None else room

    def run(self, in_place=False, workspace=True, stream=None, capacity=None):
        self.d_free = _i32(self.free + [-7] * ((capacity or len(self.free) + 3) - len(self.free)))
        self.args = dict(cached_len=_i32(self.cached), new_len=_i32(self.new), block_table=_i32(self.table).view(len(self.cached), -1), num_free=_i32([len(self.free)]))
        b = len(self.cached)
        self.out = dict(q_indptr=_i32([9] * (b + 1)), positions=_i32([9] * self.room), sequences=_i32([9] * self.room),
                        slots=torch.full((self.room,), 9, dtype=torch.int64, device="cuda"))
        self.table_out = self.args["block_table"] if in_place else torch.full_like(self.args["block_table"], 9)
        self.count_out = self.args["num_free"] if in_place else _i32([9])
        self.status = _i32([0])
        more = {} if in_place else dict(block_table_out=self.table_out, num_free_out=self.count_out)
        if workspace:
            more["workspace"] = torch.full((efim.efim_step_tables_workspace_bytes(b),), 255, dtype=torch.uint8, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        efim.efim_step_tables(**self.args, free_pages=self.d_free, **self.out, **more, status=self.status, stream=stream)
        self.more = more

    def check(self, status=0):
        torch.cuda.synchronize()
        indptr, table, free, positions, slots, sequences, ran_out = orc.step_tables(self.cached, self.new, self.table, self.free, self.room)
        assert self.out["q_indptr"].tolist() == indptr
        assert self.table_out.tolist() == table
        assert self.count_out.item() == len(free)
        for name, want in (("positions", positions), ("sequences", sequences), ("slots", slots)):
            assert self.out[name].tolist() == want, name
        assert self.status.item() == status | (NO_PAGE if ran_out else 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cached,new", [([0], [1]), ([16], [0]), ([15, 16, 17, 0, 31], [1, 1, 1, 1, 1]), ([0, 0, 5], [0, 0, 0]),
                                        ([100, 0, 1000], [300, 700, 24]), ([7] * 129, [9, 10, 0] * 43)])
def test_lengths(cached, new, in_place):
    case = Case(cached, new, 70, 400)
    case.run(in_place)
    case.check()


@pytest.mark.parametrize("batch,most,width", [(1, 20000, 2000), (300, 40, 33), (2000, 3, 20), (64, 2000, 300)])
@pytest.mark.parametrize("in_place", [False, True])
def test_sizes(batch, most, width, in_place):
    rng = np.random.default_rng(batch)
    new = rng.integers(0, most + 1, batch)
    cached = [int(rng.integers(0, width * 16 - n + 1)) for n in new]
    case = Case(cached, new.tolist(), width, 30000, batch)
    case.run(in_place, workspace=False)
    case.check()


@pytest.mark.parametrize("free", [0, 1, 7])
def test_pages_run_out(free):
    """Sequences in order take what there is; whoever comes later has slots of -1."""
    case = Case([10, 32, 0, 64], [40, 60, 3, 1], 8, free, holes=False)
    case.run()
    case.check()
    assert case.status.item() == NO_PAGE


def test_fewer_rows_than_tokens():
    case = Case([3, 4, 5], [10, 10, 10], 4, 9, room=17)
    case.run()
    case.check(BAD_POSITION)


def test_without_rows():
    case = Case([3, 4, 5], [10, 10, 10], 4, 9)
    case.run()
    out = _i32([0] * 4)
    efim.efim_step_tables(**case.args, free_pages=case.d_free, q_indptr=out, status=case.status)
    assert out.tolist() == case.out["q_indptr"].tolist() and case.args["block_table"].tolist() == case.table_out.tolist()


def test_lengths_that_are_none():
    """Negative lengths count as no tokens; lengths beyond the table fill it."""
    for cached, new, as_cached, as_new in (([5, -1, 7], [3, 4, 2], [5, 0, 7], [3, 0, 2]), ([5, 3, 7], [3, -4, 2], [5, 0, 7], [3, 0, 2]),
                                           ([5, (1 << 31) - 1, 7], [3, (1 << 31) - 1, 2], [5, 0, 7], [3, 0, 2]), ([60, 50, 7], [3, 40, 2], None, None)):
        case = Case([max(0, c) if c < 1000 else 0 for c in cached], [max(0, n) if n < 1000 else 0 for n in new], 4, 20, holes=False)
        case.cached, case.new = cached, new
        case.run()
        if as_cached:
            case.cached, case.new = as_cached, as_new
        case.check(BAD_POSITION)


def test_numbers_of_free_pages_outside_the_stack():
    for number, as_number in ((-3, 0), (50, 12)):
        case = Case([0, 0], [16, 32], 4, 12)
        case.run(capacity=12)
        case.args["num_free"].fill_(number)
        efim.efim_step_tables(**case.args, free_pages=case.d_free, **case.out, **case.more, status=case.status)
        case.free = case.free[:as_number]
        case.check(BAD_POSITION)


def test_graph_and_another_stream():
    case = Case([15, 16, 40], [4, 1, 30], 12, 40)
    case.run(stream=torch.cuda.Stream())
    case.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        efim.efim_step_tables(**case.args, free_pages=case.d_free, **case.out, **case.more, status=case.status)
    case.cached, case.new = [16, 100, 3], [1, 17, 0]
    case.table = [[9] + [-1] * 11, list(range(7)) + [-1] * 5, [3] + [-1] * 11]
    case.args["cached_len"].copy_(_i32(case.cached))
    case.args["new_len"].copy_(_i32(case.new))
    case.args["block_table"].copy_(_i32(case.table))
    case.room = len(case.out["positions"])
    graph.replay()
    case.check()


@pytest.mark.parametrize("batch,width", [(1, 5), (3, 100), (200, 40), (1, 5000)])
def test_release(batch, width):
    rng = np.random.default_rng(width)
    table = np.where(rng.random((batch, width)) < 0.8, rng.integers(0, 10 ** 6, (batch, width)), -1)
    keep = rng.integers(0, width * 16 + 40, batch)
    keep[0] = 0
    free = rng.integers(0, 10 ** 6, 11).tolist()
    want_free, want = list(free), table.copy()
    for s in range(batch):
        for e in range(-(-int(keep[s]) // 16), width):
            if table[s, e] >= 0:
                want_free.append(int(table[s, e]))
                want[s, e] = -1
    d_table, d_free, count, status = _i32(table.tolist()), _i32(free + [0] * (batch * width)), _i32([11]), _i32([0])
    efim.efim_release_pages(_i32(keep.tolist()), d_table, d_free, count, status=status)
    assert status.item() == 0 and count.item() == len(want_free)
    assert d_table.tolist() == want.tolist() and d_free[:len(want_free)].tolist() == want_free


def test_release_without_room_and_negative():
    table, free, count, status = _i32([[1, 2, 3], [4, 5, 6]]), _i32([7, 0, 0, 0]), _i32([1]), _i32([0])
    efim.efim_release_pages(_i32([17, 0]), table, free, count, status=status)
    assert status.item() == NO_PAGE and count.item() == 4
    assert free.tolist() == [7, 3, 4, 5] and table.tolist() == [[1, 2, -1], [-1, -1, 6]]
    status.zero_()
    efim.efim_release_pages(_i32([-1, 48]), table, free, count, status=status)
    assert status.item() == BAD_POSITION and table.tolist() == [[1, 2, -1], [-1, -1, 6]] and count.item() == 4


def test_what_is_given_comes_back():
    case = Case([0, 20, 5], [50, 3, 0], 6, 20, holes=False)
    case.run(in_place=True)
    efim.efim_release_pages(case.args["cached_len"], case.table_out, case.d_free, case.count_out, status=case.status)
    assert case.status.item() == 0 and case.count_out.item() == 20 and case.table_out.tolist() == case.table
    assert sorted(case.d_free[:20].tolist()) == sorted(case.free)
