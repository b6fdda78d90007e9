"""efim_kv4_decode_attn against the float64 definition on what the cache holds.

Tolerance, from the arithmetic.  Scores: products of fp16 numbers are exact, their sum over D <= 128 dims in fp32 is off by at most
128 * 2^-23 of the sum of magnitudes E (2^-23 a step: a tensor core may cut where it does not round), i.e. 2^-16 E; a weight is then off by 2^-16 E,
its exponential by 2^-21 (argument rounded to 2^-24 of at most 2^7 where weights count: 2^-17 in the exponent), and its entry into the
product by 2^-11.  Numerator and denominator each carry the former, the numerator alone the last: (2^-11 + 2 (2^-16 E + 2^-16)) of the weighted mean of
|v|; and the result's own rounding, 2^-8 of it.  Weights below 2^-25 of the largest lie under fp16's normal range as they enter (the largest
at 2^11 or more) and are off by half its smallest step, 2^-25 / 2^11 of the largest weight, which the denominator holds at least once: 2^-36 of
the sum of |v| over the keys (it shows where the heavy keys' values are 0).  lse: 2^-16 E + 2^-15."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_kv4_oracle as orc
from oracle.efim_oracle import bf16_to_f64

pytestmark = pytest.mark.gpu
BAD_PAGE, BAD_POSITION = 1, 2


def _f64(t):
    return bf16_to_f64(t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16))


class Case:
    def __init__(self, hq, hkv, d, ctx, new, seed=0, extra_rows=0, k_scale=0.5, v_scale=0.25, q_size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.shape, self.ctx, self.new, self.extra = (hq, hkv, d), list(ctx), list(new), extra_rows
        pages = [-(-c // 16) for c in ctx]
        n = sum(pages) + 3
        order = torch.randperm(n, generator=g).tolist()
        self.table = torch.full((len(ctx), max(pages + [1]) + 1), -1, dtype=torch.int32)
        for s, m in enumerate(pages):
            self.table[s, :m] = torch.tensor([order.pop() for _ in range(m)])
        codes = [torch.randint(256, (n, hkv, 16, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
        scales = [(torch.rand(n, hkv, 16, d // 16, generator=g) * 2 + 0.3).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
        # what no sequence holds is anything: NaN's scales too
        free = torch.ones(n, 16, dtype=torch.bool)
        for s, c in enumerate(ctx):
            for p in range(c):
                free[self.table[s, p // 16], p % 16] = False
        for x in scales:
            x.permute(0, 2, 1, 3)[free] = 127
        self.cache = efim.Cache4(*(x.cuda() for x in codes + scales), hq, k_scale, v_scale)
        self.q = (q_size * torch.randn(sum(new) + extra_rows, hq, d, generator=g)).bfloat16().cuda()
        self.out = torch.full_like(self.q, 5.0)
        self.lse = torch.full(self.q.shape[:2], 5.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.indptr = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device="cuda")

    def run(self, indptr=True, max_ctx=None, max_new=None, out=None, stream=None, sm_scale=0.0):
        max_ctx = max(self.ctx + [1]) if max_ctx is None else max_ctx
        max_new = max(self.new) if max_new is None else max_new
        args = dict(q_indptr=self.indptr, max_new_len=max_new) if indptr else {}
        size = efim.efim_kv4_decode_workspace_bytes(self.cache, len(self.ctx), max_new if indptr else 1, max_ctx)
        self.ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
        self.d_table, self.d_ctx = self.table.cuda(), torch.tensor(self.ctx, dtype=torch.int32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        efim.efim_kv4_decode_attn(self.cache, len(self.ctx), self.d_ctx, max_ctx, self.d_table, self.q, self.out if out is None else out,
                                  self.lse, sm_scale, workspace=self.ws, status=self.status, stream=stream, **args)

    def held(self):
        c = self.cache
        return (orc.held(c.k_codes.cpu().numpy(), c.k_scales.cpu().numpy(), c.desc.k_scale),
                orc.held(c.v_codes.cpu().numpy(), c.v_scales.cpu().numpy(), c.desc.v_scale))

    def check(self, q=None, only=None, sm_scale=None):
        hq, hkv, d = self.shape
        k_pool, v_pool = self.held()
        q, out, lse = _f64(self.q if q is None else q), _f64(self.out), self.lse.double().cpu().numpy()
        group, worst = hq // hkv, 0.0
        row = 0
        for s, (c, n) in enumerate(zip(self.ctx, self.new)):
            if only is None or s in only:
                pages = self.table[s, :-(-c // 16)].numpy()
                for h in range(hkv):
                    heads = slice(h * group, (h + 1) * group)
                    k, v = (x[pages, h].reshape(-1, d)[:max(c, 0)] for x in (k_pool, v_pool))
                    limits = np.repeat(np.arange(c - n + 1, c + 1), group)
                    want, want_lse, size, reach = orc.attend(q[row:row + n, heads].reshape(-1, d), k, v, limits, sm_scale or d ** -0.5)
                    shape = (n, group)
                    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * (2.0 ** -16 * reach + 2.0 ** -16))[:, None] * size + 2.0 ** -36 * np.abs(v).sum(0) + 1e-37
                    err = np.abs(out[row:row + n, heads].reshape(-1, d) - want)
                    assert (err <= tol).all(), (s, h, float((err / tol).max()))
                    worst = max(worst, float((err / tol).max(initial=0)))
                    got = lse[row:row + n, heads].reshape(-1)
                    none = limits <= 0
                    assert np.isneginf(got[none]).all() and (np.abs(got - want_lse)[~none] <= (2.0 ** -16 * reach + 2.0 ** -15)[~none]).all()
                    assert want.reshape(*shape, d).shape[0] == n
            row += n
        assert (out[row:] == 5).all() and (lse[row:] == 5).all()
        return worst


HEADS = [(32, 8, 128), (28, 4, 128), (8, 8, 64), (16, 1, 128), (9, 3, 64), (24, 1, 64), (48, 2, 128), (5, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("indptr", [False, True])
def test_one_token(hq, hkv, d, indptr):
    """Lengths of zero, one, around a page, of several chunks; with the rows in order or given."""
    case = Case(hq, hkv, d, [1, 0, 15, 16, 17, 300, 700, 2100], [1] * 8, seed=hq)
    case.run(indptr)
    case.check()
    assert case.status.item() == 0


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("new", [(2, 2, 2), (1, 5, 3), (9, 0, 1), (0, 40, 17)])
def test_several_tokens(hq, hkv, d, new):
    case = Case(hq, hkv, d, [50, 800, 17], new, seed=sum(new), extra_rows=3)
    case.run()
    case.check()
    assert case.status.item() == 0


@pytest.mark.parametrize("batch,ctx", [(1, 5000), (3, 9000), (40, 600), (200, 90), (300, 2500)])
def test_plans(batch, ctx):
    """One chunk and many, fewer and more CTAs than are resident; a few sequences are looked at."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(1, ctx + 1, batch).tolist()
    lens[0] = ctx
    case = Case(8, 2, 128, lens, [1] * batch, seed=batch)
    case.run(False)
    case.check(only={0, batch // 2, batch - 1})
    assert case.status.item() == 0


@pytest.mark.parametrize("hq,hkv,d,most", [(28, 4, 128, 9), (8, 2, 64, 5), (16, 2, 128, 2), (48, 2, 128, 3)])
@pytest.mark.parametrize("batch,ctx", [(60, 5000), (7, 20000), (500, 1500)])
def test_pieces(hq, hkv, d, most, batch, ctx):
    """Rows and lengths of all kinds in one call: pieces that hold many units, a part of one, starts alone."""
    rng = np.random.default_rng(batch + hq)
    new = rng.integers(0, most + 1, batch)
    lens = np.maximum((ctx * rng.random(batch) ** 3).astype(int), new)
    lens[batch // 2], new[batch // 2] = ctx, most
    case = Case(hq, hkv, d, lens.tolist(), new.tolist(), seed=batch, extra_rows=2)
    case.run(max_new=most)
    assert case.status.item() == 0
    longest = int(np.argmax(lens))
    case.check(only={0, longest, batch // 2, batch - 1, *rng.integers(0, batch, 4 if batch < 100 else 12).tolist()} - ({longest} if ctx > 6000 else set()))


def test_pages_past_32_bit_offsets():
    """A pool of more than 2^32 bytes of codes: its last pages give what a small pool gives, appended, read back and attended."""
    hq, hkv, d, many = 8, 8, 128, 540000
    g = torch.Generator().manual_seed(2)
    assert many * hkv * 16 * d // 2 > 1 << 32
    results = []
    for pages in (many, 12):
        codes = [torch.empty(pages, hkv, 16, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.empty(pages, hkv, 16, d // 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = efim.Cache4(*codes, *scales, hq)
        g.manual_seed(2)
        qkv = torch.randn(170, 3 * hq * d, generator=g).bfloat16().cuda()
        table = torch.tensor([[pages - 1 - i for i in range(11)]], dtype=torch.int32)
        batch = efim.Batch([3], [170], table.numpy())
        head = efim.Batch([0], [3], table.numpy())
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        q = torch.empty(170, hq, d, dtype=torch.bfloat16, device="cuda")
        efim.efim_kv4_append(cache, head, None, None, None, qkv[:3, hq * d:2 * hq * d], qkv[:3, 2 * hq * d:], None, status)
        efim.efim_kv4_append(cache, batch, None, None, *qkv.split([hq * d] * 3, 1), q, status)
        read = [torch.empty(11, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        efim.efim_kv4_unpack(cache, table[0].cuda(), *read, status)
        read[0].view(11, hkv, 16, d)[10, :, 13:] = read[1].view(11, hkv, 16, d)[10, :, 13:] = 0      # (slots that hold nothing)
        out = torch.empty(1, hq, d, dtype=torch.bfloat16, device="cuda")
        ctx = torch.tensor([173], dtype=torch.int32, device="cuda")
        efim.efim_kv4_decode_attn(cache, 1, ctx, 173, table.cuda(), q[-1:], out, status=status)
        turn = torch.empty_like(q)
        ws = torch.empty(efim.efim_kv4_prefill_workspace_bytes(cache, batch), dtype=torch.uint8, device="cuda")
        efim.efim_kv4_append_prefill_attn(cache, batch, q, turn, workspace=ws, status=status)
        assert status.item() == 0
        results.append([q, *read, out, turn])
        del codes, scales, cache
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_new_tokens_before_the_sequence():
    """More rows than keys: the first ones see nothing."""
    case = Case(4, 2, 64, [3, 2], [5, 2])
    case.run()
    case.check()
    assert case.status.item() == 0 and torch.isneginf(case.lse[:2]).all() and (case.out[:2].float() == 0).all()


def test_chunks_that_some_rows_do_not_see():
    """The last rows begin a chunk that the first ones do not reach."""
    for ctx in (256 + 3, 512 + 1):
        case = Case(4, 1, 128, [ctx], [9])
        case.table = torch.nn.functional.pad(case.table, (0, 125 - case.table.shape[1]), value=-1)
        case.run(max_ctx=2000)
        case.check()


@pytest.mark.parametrize("q_size", [1e-30, 30.0, 1e4])
def test_sizes_of_queries(q_size):
    """Scores of hundreds (one key takes all), and queries whose scores are all alike."""
    case = Case(4, 2, 128, [700, 40], [2, 1], q_size=q_size)
    sm_scale = 0.0 if q_size != 1e4 else 1e-4
    case.run(sm_scale=sm_scale)
    case.check(sm_scale=sm_scale or None)


def test_equal_keys_of_a_long_context():
    """Every weight alike: no bias of the rounded weights against the sum that divides them."""
    case = Case(8, 1, 128, [6000], [1])
    for x in (case.cache.k_codes, case.cache.v_codes):
        x.copy_(x[:1, :, :1].expand_as(x).clone())
    for x in (case.cache.k_scales, case.cache.v_scales):
        x.fill_(0x38)
    case.run(False)
    case.check()


def test_d_out_is_q():
    case = Case(28, 4, 128, [900, 33, 64], [3, 1, 5])
    q = case.q.clone()
    case.run(out=case.q)
    case.out = case.q
    case.check(q=q)


def test_bad_pages():
    """Keys of pages outside the pool are absent; the others count."""
    case = Case(4, 2, 64, [100, 60, 40], [1, 3, 1])
    good = case.table.clone()
    case.table[0, 2], case.table[2, :3] = len(case.cache.k_codes), -5
    case.run()
    assert case.status.item() == BAD_PAGE
    assert (case.out[4].float() == 0).all() and torch.isneginf(case.lse[4]).all()
    case.table = good
    case.check(only={1})
    k_pool, v_pool = case.held()
    keys = [p for p in range(100) if p // 16 != 2]
    for h in range(2):
        k, v = (np.stack([x[good[0, p // 16], h, p % 16] for p in keys]) for x in (k_pool, v_pool))
        want, _, size, reach = orc.attend(_f64(case.q[0, 2 * h:2 * h + 2]), k, v, [84, 84], 64 ** -0.5)
        assert (np.abs(_f64(case.out[0, 2 * h:2 * h + 2]) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -15 * reach.max()) * size).all()


def test_lengths_beyond_the_bounds():
    case = Case(4, 2, 64, [700, 40, 30], [2, 1, 1])
    case.run(max_ctx=256)
    assert case.status.item() == BAD_POSITION
    case.check(only={1, 2})
    assert torch.isfinite(case.out.float()).all()
    case = Case(4, 2, 64, [70, 40, 30], [4, 1, 2])
    case.run(max_new=2)
    assert case.status.item() == BAD_POSITION
    case.check(only={1, 2})
    assert (case.out[2:4].float() == 5).all()                               # rows beyond the bound
    # rows that q does not have
    case = Case(4, 2, 64, [70, 40], [2, 3])
    case.q, case.out, case.lse = case.q[:4], case.out[:4], case.lse[:4]
    case.run()
    assert case.status.item() == BAD_POSITION and (case.out[2:].float() == 5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", [10, 95, 98])
def test_values_that_are_nan(d, where):
    """A NaN reaches the rows that see it, in its sixteen places; the others are as without it."""
    hq = 4
    case, clean = (Case(hq, 2, d, [100, 50], [4, 2], seed=3) for _ in range(2))
    page, slot = case.table[0, where // 16], where % 16
    case.cache.v_scales[page, 1, slot, 2] = 255
    case.run()
    clean.run()
    torch.cuda.synchronize()
    sees = torch.arange(4) + 97 > where
    nan = torch.isnan(case.out.float()).cpu()
    want = torch.zeros_like(nan)
    want[:4, 2:, 32:48] = sees[:, None, None]
    assert torch.equal(nan, want)
    assert torch.equal(case.out.cpu()[~want].view(torch.int16), clean.out.cpu()[~want].view(torch.int16))
    # a key
    case.cache.v_scales.copy_(clean.cache.v_scales)
    case.cache.k_scales[page, 1, slot, 0] = 127
    case.run()
    nan = torch.isnan(case.out.float()).cpu()
    want[:4, 2:] = sees[:, None, None]
    assert torch.equal(nan, want)
    assert torch.equal(case.out.cpu()[~want].view(torch.int16), clean.out.cpu()[~want].view(torch.int16))


def test_queries_that_are_not_finite():
    case, clean = (Case(8, 2, 128, [300, 50], [3, 2], seed=4) for _ in range(2))
    case.q[1, 2, 5], case.q[3, 7, 0] = float("inf"), float("nan")
    case.run()
    clean.run()
    bad = torch.zeros(5, 8, dtype=torch.bool)
    bad[1, 2] = bad[3, 7] = True
    assert torch.equal(torch.isnan(case.out.float()).cpu(), bad[..., None].expand(5, 8, 128))
    assert torch.equal(case.out.cpu()[~bad].view(torch.int16), clean.out.cpu()[~bad].view(torch.int16))


def test_another_stream_and_a_graph():
    case = Case(32, 8, 128, [4000, 70], [1, 1], seed=9)
    case.run(False, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    case.check()
    first = case.out.clone()
    case.out.fill_(5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        efim.efim_kv4_decode_attn(case.cache, 2, case.d_ctx, 4000, case.d_table, case.q, case.out, case.lse, workspace=case.ws, status=case.status)
    for _ in range(2):
        graph.replay()
        assert torch.equal(case.out.view(torch.int16), first.view(torch.int16))
    case.d_ctx.copy_(torch.tensor([2500, 33]))                              # other lengths, the same graph
    case.ctx = [2500, 33]
    graph.replay()
    case.check()
