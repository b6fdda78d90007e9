"""efim_qk_norm_append against the float64 definition.

Tolerance, from the arithmetic: the result is rounded to bf16 once (half an ulp: 2^-8 of the value, 2^-134 below the normal range).  Before
that, in fp32: a sum of 128 squares (16 in a chain, 3 levels of pairs: 20 * 2^-24, halved by the root), the root (2 ulp), two
products and a weight's offset (3 * 2^-24) - below 2^-20 of a normalised value - then two products and a sum: 2^-19 of the pair's
products |a c| + |b s|, and the rounding of what that moves, together below 2^-18 of them."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_drafts_oracle as orc
from oracle.efim_oracle import bf16_to_f64

pytestmark = pytest.mark.gpu
BAD_PAGE, BAD_POSITION = 1, 2


def _bits(t):
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _f64(t):
    return bf16_to_f64(_bits(t))


class Case:
    def __init__(self, hq, hkv, d, cached, new, layout="qkv", weights="bf16", offset=0.0, interleaved=False, rope=True, seed=0,
                 eps=1e-6, scale=1.0, max_position=None):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.d, self.cached, self.new = hq, hkv, d, list(cached), list(new)
        self.eps, self.offset, self.interleaved = eps, offset, interleaved
        t = sum(new)
        pages = [-(-(c + n) // 16) for c, n in zip(cached, new)]
        order = torch.randperm(sum(pages) + 2, generator=g).tolist()
        self.table = np.full((len(new), max(pages + [1])), -1, np.int32)
        for s, n in enumerate(pages):
            self.table[s, :n] = [order.pop() for _ in range(n)]
        q, kv = hq * d, hkv * d
        pad = dict(qkv=0, wide=24)[layout] if layout in ("qkv", "wide") else 0
        x = (scale * torch.randn(t, q + 2 * kv + pad, generator=g)).bfloat16().cuda()
        self.q, self.k, self.v = x[:, :q], x[:, q:q + kv], x[:, q + kv:q + 2 * kv]
        if layout in ("packed", "in place"):
            self.q, self.k, self.v = (y.clone().view(t, -1, d) for y in (self.q, self.k, self.v))
        self.out = self.q if layout == "in place" else torch.full((t, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        shape = (sum(pages) + 2, hkv, 16, d)
        self.k_pool, self.v_pool = (torch.randn(shape, generator=g).bfloat16().cuda() for _ in range(2))
        self.wq = self.wk = None
        if weights:
            dtype = dict(bf16=torch.bfloat16, f32=torch.float32)[weights]
            self.wq, self.wk = ((torch.randn(d, generator=g) * 0.3 + 1 - offset).to(dtype).cuda() for _ in range(2))
        self.rope = efim.Rope(10000.0, d, max_position or max([c + n for c, n in zip(cached, new)] + [1]), interleaved) if rope else None
        self.cache = efim.Cache(self.k_pool, self.v_pool, hq)
        self.batch = efim.Batch(self.cached, self.new, self.table)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, q=True, stream=None):
        norm = efim.QkNorm(self.wq, self.wk, self.eps, self.offset)
        efim.efim_qk_norm_append(self.cache, self.batch, norm, self.rope, self.q if q else None, self.k, self.v,
                                 self.out if q else None, self.status, stream)

    def want(self):
        """-> per token: (query rows, key rows) each with its tolerance, value bits, position, sequence."""
        table = self.rope.table.cpu().numpy() if self.rope else None
        inputs = [_f64(x).reshape(len(x), -1, self.d) for x in (self.q, self.k)]
        values = _bits(self.v).reshape(len(self.v), -1, self.d)
        weights = [None if w is None else w.double().cpu().numpy() for w in (self.wq, self.wk)]
        t, rows = 0, []
        for s, (c, n) in enumerate(zip(self.cached, self.new)):
            for i in range(n):
                both = []
                for x, w in zip(inputs, weights):
                    with np.errstate(all="ignore"):
                        y = orc.qk_norm(x[t], w, self.eps, self.offset)
                    if self.rope is None:
                        y, size = y, np.abs(y)
                    elif c + i < len(table):
                        y, size = orc.rotate(y, table[c + i], self.interleaved)
                    else:
                        y = size = np.zeros_like(y)
                    both.append((y, 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size + 2.0 ** -134))
                rows.append((both[0], both[1], values[t], c + i, s))
                t += 1
        return rows

    def check(self, q=True, skip=lambda s, pos: False):
        before = _bits(self.k_pool).copy(), _bits(self.v_pool).copy()
        rows = self.want()
        self.run(q)
        torch.cuda.synchronize()
        out, kp, vp = _f64(self.out), _bits(self.k_pool), _bits(self.v_pool)
        untouched = np.ones(kp.shape[:1] + kp.shape[2:3], bool)
        for t, ((yq, tq), (yk, tk), v, pos, s) in enumerate(rows):
            if q:
                err = np.abs(out[t].reshape(yq.shape) - yq)
                assert (err <= tq).all(), (t, s, pos, float((err / tq).max()))
            if skip(s, pos):
                continue
            page, slot = self.table[s, pos // 16], pos % 16
            err = np.abs(bf16_to_f64(kp[page, :, slot]) - yk)
            assert (err <= tk).all(), (t, s, pos, float((err / tk).max()))
            assert np.array_equal(vp[page, :, slot], v)
            untouched[page, slot] = False
        for got, was in ((kp, before[0]), (vp, before[1])):
            got, was = np.moveaxis(got, 2, 1), np.moveaxis(was, 2, 1)
            assert np.array_equal(got[untouched], was[untouched])
        return int(self.status.item())


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (4, 4, 64), (16, 1, 64), (9, 3, 128), (1, 1, 64), (5, 1, 128)])
@pytest.mark.parametrize("layout", ["qkv", "wide", "packed", "in place"])
def test_heads_and_layouts(hq, hkv, d, layout):
    assert Case(hq, hkv, d, [0, 15, 37], [1, 18, 4], layout, seed=hq + d).check() == 0


@pytest.mark.parametrize("weights,offset", [("bf16", 0.0), ("f32", 0.0), (None, 0.0), ("bf16", 1.0), ("f32", 1.0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rope", [False, True])
def test_weights_and_pairings(weights, offset, interleaved, rope):
    assert Case(6, 2, 128, [100, 3], [5, 2], weights=weights, offset=offset, interleaved=interleaved, rope=rope, seed=5).check() == 0


@pytest.mark.parametrize("tokens,hq,hkv,d", [(444, 4, 4, 64), (445, 4, 4, 64), (900, 2, 1, 64), (1800, 4, 4, 64), (1790, 2, 2, 128),
                                             (900, 32, 32, 128), (1777, 24, 4, 128),
                                             (9500, 32, 8, 128), (1500, 240, 16, 128), (9600, 72, 8, 64)])
def test_numbers_of_tokens(tokens, hq, hkv, d):
    """Every number of warps a token, one wave and several, ragged over sequences (one of them without new tokens)."""
    rng = np.random.default_rng(tokens)
    cut = np.sort(rng.integers(0, tokens + 1, 6))
    new = np.diff(np.concatenate([[0], cut, [tokens]])).tolist()
    new[3:3] = [0]
    assert Case(hq, hkv, d, rng.integers(0, 50, len(new)).tolist(), new, seed=tokens).check() == 0


@pytest.mark.parametrize("batch", [31, 33, 1025])
def test_many_sequences(batch):
    rng = np.random.default_rng(batch)
    assert Case(4, 2, 64, rng.integers(0, 40, batch).tolist(), rng.integers(0, 3, batch).tolist() + [], seed=batch).check() == 0


def test_keys_and_values_alone():
    assert Case(8, 2, 128, [10, 0], [30, 7], seed=2).check(q=False) == 0


def test_one_row_may_stand_anywhere():
    """A single token's row stride says nothing."""
    c = Case(8, 2, 128, [10], [1], seed=2)
    c.q, c.k, c.v = (x.as_strided(x.shape, (0, 1)) for x in (c.q, c.k, c.v))
    assert c.check() == 0


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1e17, 1e20, 1e37])
def test_sizes_of_values(scale):
    """Squares beyond either end of fp32.  At 1e-30 eps is all there is under the root."""
    assert Case(4, 2, 128, [3], [9], scale=scale, eps=1e-6, seed=8).check() == 0
    assert Case(4, 2, 64, [3], [9], scale=scale, eps=1e-6, rope=False, seed=9).check() == 0


def test_rows_of_zeros_infinities_and_nan():
    c = Case(4, 2, 64, [20], [4], rope=False, seed=3)
    x = c.q.view(4, 4, 64)
    x[0, 1] = 0
    x[1, 2, 7] = float("inf")
    x[2, 3, 9] = float("nan")
    other = c.q.clone()
    c.run()
    torch.cuda.synchronize()
    out = c.out.float().cpu()
    assert (out[0, 1] == 0).all()
    assert out[1, 2, 7].isnan() and (out[1, 2].nan_to_num(0) == 0).all()
    assert out[2, 3].isnan().all()
    keep = torch.ones(4, 4, dtype=torch.bool)
    keep[0, 1] = keep[1, 2] = keep[2, 3] = False
    assert out[keep].isfinite().all()
    # the other heads are what they are without those beside them
    clean = Case(4, 2, 64, [20], [4], rope=False, seed=3)
    clean.run()
    assert torch.equal(clean.out.cpu()[keep].view(torch.int16), c.out.cpu()[keep].view(torch.int16))
    assert torch.equal(other.view(torch.int16), c.q.view(torch.int16))


def test_tokens_without_a_place():
    """A page id outside the pool and a position past the rotary table: their k and v go nowhere, their query rows are written."""
    c = Case(6, 2, 128, [14, 40], [4, 3], seed=4)
    c.table[1, 2] = 10 ** 6
    c.batch = efim.Batch(c.cached, c.new, c.table)
    assert c.check(skip=lambda s, pos: s == 1 and pos // 16 == 2) == BAD_PAGE
    c = Case(6, 2, 128, [14, 40], [4, 3], seed=4, max_position=42)
    assert c.check(skip=lambda s, pos: pos >= 42) == BAD_POSITION
    c = Case(6, 2, 128, [14, 40], [4, 3], seed=4)
    c.batch = efim.Batch(c.cached, c.new, c.table[:, :2])             # the block table ends before the tokens do
    assert c.check(skip=lambda s, pos: pos // 16 >= 2) == BAD_POSITION


def test_offsets_past_32_bits():
    """Pages whose elements lie beyond 2^32 bytes and 2^31 elements of the pools, and token rows beyond 2^31 elements of their buffer."""
    hkv, d, pages = 8, 128, 131072 + 40
    pools = [torch.zeros((pages, hkv, 16, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c = Case(8, hkv, d, [15], [3], seed=6)
    far = np.array([[pages - 2, pages - 1]], np.int32)
    small_k, small_v = c.k_pool, c.v_pool
    c.run()
    cache = efim.Cache(*pools, 8)
    stride = 1 << 30
    buf = torch.zeros(2 * stride + 8 * d + 2 * hkv * d, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((3, 8 * d + 2 * hkv * d), (stride, 1))
    rows.copy_(torch.cat([c.q, c.k, c.v], 1))
    out = torch.empty_like(c.out)
    efim.efim_qk_norm_append(cache, efim.Batch([15], [3], far), efim.QkNorm(c.wq, c.wk), c.rope, rows[:, :8 * d],
                             rows[:, 8 * d:(8 + hkv) * d], rows[:, (8 + hkv) * d:], out, c.status)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and torch.equal(out.view(torch.int16), c.out.view(torch.int16))
    for small, large in ((small_k, pools[0]), (small_v, pools[1])):
        assert torch.equal(large[pages - 2, :, 15], small[int(c.table[0, 0]), :, 15])
        assert torch.equal(large[pages - 1, :, :2], small[int(c.table[0, 1]), :, :2])
        assert not large[pages - 1, :, 2:].any() and not large[:pages - 2].any()


def test_other_streams_and_graphs():
    a, b = (Case(8, 2, 128, [30, 2], [5, 40], seed=7) for _ in range(2))
    a.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run()
    side.synchronize()
    want = [t.clone() for t in (a.out, a.k_pool, a.v_pool)]
    for x, y in zip(want, (b.out, b.k_pool, b.v_pool)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    b.out.fill_(float("nan"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want[0].view(torch.int16), b.out.view(torch.int16))


def test_attention_takes_what_it_writes():
    """Heads of root mean square 1 under weights of one: the norm changes nothing but eps, so the step agrees with efim_kv_append's."""
    import tests.gpu_harness as H
    from tests.test_gpu_parity import _custom
    w = _custom(8, 2, 128, [100, 7], [20, 3], seed=31)
    dw = H.DeviceWorkload(w)
    rng = np.random.default_rng(1)
    for x in (dw.q, dw.k_new):                         # +-1 everywhere
        x.copy_(torch.from_numpy(rng.choice([-1.0, 1.0], tuple(x.shape))).to(x))
    q_raw, k_raw, v_raw = dw.q.clone(), dw.k_new.clone(), dw.v_new.clone()
    dw.gpu_kv_append()
    dw.gpu_prefill()
    want, pool = dw.out.clone(), dw.k_pool.clone()
    q_out = torch.empty_like(q_raw)
    efim.efim_qk_norm_append(dw.cache, dw.batch, efim.QkNorm(None, None, 1e-30), dw.rope, q_raw, k_raw, v_raw, q_out, dw.status)
    assert torch.equal(q_out.view(torch.int16), dw.q.view(torch.int16)) and torch.equal(pool.view(torch.int16), dw.k_pool.view(torch.int16))
    efim.efim_append_prefill_attn(dw.cache, dw.batch, q_out, dw.out, None, 0.0, dw.ws, dw.status)
    torch.cuda.synchronize()
    assert torch.equal(want.view(torch.int16), dw.out.view(torch.int16)) and int(dw.status.item()) == 0
