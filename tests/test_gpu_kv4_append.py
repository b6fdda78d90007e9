"""efim_kv4_append and efim_kv4_unpack.  What the 4-bit append rounds to bf16 on the way is what efim_kv_append or efim_qk_norm_append
leave, bit for bit; from there the blocks are whole numbers, which have to be the oracle's."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_kv4_oracle as orc
from oracle.efim_oracle import bf16_to_f64

pytestmark = pytest.mark.gpu
BAD_PAGE, BAD_POSITION = 1, 2


def _bits(t):
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _f64(t):
    return bf16_to_f64(_bits(t))


class Case:
    def __init__(self, hq, hkv, d, cached, new, norm=None, interleaved=False, rope=True, seed=0, packed=False, k_scale=0.5, v_scale=0.25,
                 size=1.0, max_position=None, spare=0):
        g = torch.Generator().manual_seed(seed)
        self.shape, self.cached, self.new = (hq, hkv, d), list(cached), list(new)
        t = sum(new) + spare
        pages = [-(-(c + n) // 16) for c, n in zip(cached, new)]
        order = torch.randperm(sum(pages) + 2, generator=g).tolist()
        self.table = np.full((len(new), max(pages + [1])), -1, np.int32)
        for s, n in enumerate(pages):
            self.table[s, :n] = [order.pop() for _ in range(n)]
        q, kv = hq * d, hkv * d
        x = (size * torch.randn(t, q + 2 * kv, generator=g)).bfloat16().cuda()
        self.q, self.k, self.v = x[:, :q], x[:, q:q + kv], x[:, q + kv:]
        if packed:
            self.q, self.k, self.v = (y.clone().view(t, -1, d) for y in (self.q, self.k, self.v))
        n = sum(pages) + 2
        codes = [torch.randint(256, (n, hkv, 16, d // 2), generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
        scales = [torch.randint(256, (n, hkv, 16, d // 16), generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
        self.cache = efim.Cache4(*codes, *scales, hq, k_scale, v_scale)
        self.plain = efim.Cache(*(torch.zeros(n, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)), hq)
        self.batch = efim.Batch(self.cached, self.new, self.table)
        self.batch.desc.total_new_tokens = t
        self.rope = efim.Rope(10000.0, d, max_position or max([c + m for c, m in zip(cached, new)] + [1]), interleaved) if rope else None
        weights = [(torch.randn(d, generator=g) * 0.3 + 1).to(torch.float32 if norm == "f32" else torch.bfloat16).cuda() for _ in range(2)]
        self.norm = efim.QkNorm(*weights, 1e-6) if norm else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.out = torch.full((t, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")

    def check(self, queries=True, skip=lambda s, pos: False):
        """Against the bf16 append of the same tokens, quantised by the oracle.  -> the device's status"""
        hq, hkv, d = self.shape
        t = sum(self.new)
        status = torch.zeros_like(self.status)
        self.batch.desc.total_new_tokens = t
        q, k, v = (y[:t] for y in (self.q, self.k, self.v))
        want_q = q.clone().contiguous().view(t, hq, d)
        if self.norm:
            efim.efim_qk_norm_append(self.plain, self.batch, self.norm, self.rope, q, k, v, want_q, status)
        else:
            efim.efim_kv_append(self.plain, self.batch, self.rope, want_q, k.contiguous(), v.contiguous(), status)
        pools = [p.cpu().numpy() for p in (self.cache.k_codes, self.cache.v_codes, self.cache.k_scales, self.cache.v_scales)]
        self.batch.desc.total_new_tokens = len(self.q)
        efim.efim_kv4_append(self.cache, self.batch, self.norm, self.rope, self.q if queries else None, self.k, self.v,
                             self.out if queries else None, self.status)
        torch.cuda.synchronize()
        if queries:
            assert np.array_equal(_bits(self.out[:t]), _bits(want_q))
        assert torch.isnan(self.out[t if queries else 0:].float()).all()     # rows behind the last sequence, or all
        row = 0
        for s, (c, n) in enumerate(zip(self.cached, self.new)):
            for pos in range(c, c + n):
                if not skip(s, pos):
                    page, slot = self.table[s, pos // 16], pos % 16
                    for x, (pool, g) in enumerate(((self.plain.k_pool, self.cache.desc.k_scale), (self.plain.v_pool, self.cache.desc.v_scale))):
                        pools[x][page, :, slot], pools[2 + x][page, :, slot] = orc.quantize(_f64(pool[page, :, slot]), g)
                row += 1
        got = [p.cpu().numpy() for p in (self.cache.k_codes, self.cache.v_codes, self.cache.k_scales, self.cache.v_scales)]
        for x in (0, 1):                                                     # (the codes of a block that is NaN say nothing)
            nan = np.repeat(pools[2 + x] & 127 == 127, 8, axis=-1)
            for name, off in (("scales", got[2 + x] != pools[2 + x]), ("codes", (got[x] != pools[x]) & ~nan)):
                assert not off.any(), (name, x, int(off.sum()), np.argwhere(off)[0])
        return int(self.status.item())


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (4, 4, 64), (16, 1, 64), (9, 3, 128), (1, 1, 64), (5, 1, 128)])
@pytest.mark.parametrize("norm", [None, "bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_heads(hq, hkv, d, norm, packed):
    assert Case(hq, hkv, d, [0, 15, 37], [1, 18, 4], norm, packed=packed, seed=hq + d).check() == 0


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("norm", [None, "bf16"])
@pytest.mark.parametrize("queries", [False, True])
def test_pairings(interleaved, rope, norm, queries):
    assert Case(6, 2, 64, [100, 3], [5, 2], norm, interleaved, rope, seed=5).check(queries) == 0


@pytest.mark.parametrize("tokens,hq,hkv,d", [(444, 4, 4, 64), (2000, 4, 4, 64), (1800, 24, 4, 128), (3000, 2, 2, 128)])
def test_numbers_of_tokens(tokens, hq, hkv, d):
    cut = np.sort(np.random.default_rng(tokens).integers(0, tokens + 1, 6))
    new = np.diff(np.concatenate([[0], cut, [tokens]])).tolist()
    assert Case(hq, hkv, d, [3 * i for i in range(len(new))], new, seed=tokens).check() == 0


@pytest.mark.parametrize("k_scale,v_scale,size", [(1.0, 1.0, 1000.0), (2.0 ** -20, 2.0 ** 30, 1e-3), (2.0 ** 60, 2.0 ** -60, 1.0), (1.0, 64.0, 1e5)])
def test_pool_scales(k_scale, v_scale, size):
    """Values beyond the range of the pool's scale, within and below it."""
    assert Case(4, 2, 128, [5, 0], [20, 3], k_scale=k_scale, v_scale=v_scale, size=size).check() == 0


def test_ties_and_ends():
    """Every pair of a block's largest value and another one of 8 significant bits, ties of scales and codes among them; zeros of both
    signs, infinities, NaN, the smallest and largest numbers."""
    tops = np.arange(128, 256)
    rng = np.random.default_rng(1)
    for exponent in (0, -9, -20, 9):
        x = rng.integers(-255, 256, (128, 2, 64)).astype(np.float64)
        x = np.where(np.abs(x) > tops[:, None, None], x // 4, x)
        x[:, :, ::16] = tops[:, None, None]
        x[:, :, 1::16] = -tops[:, None, None] / 2 ** rng.integers(0, 6, (128, 2, 4))
        case = Case(2, 2, 64, [0], [128], rope=False, packed=True)
        for t in (case.k, case.v):
            t.copy_(torch.from_numpy(x * 2.0 ** exponent).bfloat16())
        assert case.check() == 0
    case = Case(2, 2, 64, [0], [128], rope=False, packed=True)
    flat = case.k.view(-1)
    flat[:8] = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), 3e38, -3e38, 1e-40, -1e-40])
    flat[16:32] = -0.0
    flat[40] = float("nan")
    flat[64:80] = 1e-40
    case.v.copy_(case.k.flip(0))
    assert case.check() == 0
    assert case.cache.k_scales[case.table[0, 0], 0, 0].tolist()[:3] == [126, 1, 127]


def test_rows_behind_the_last_sequence():
    case = Case(4, 2, 128, [7, 0, 3], [2, 0, 0], spare=37)
    assert case.check() == 0
    assert Case(4, 2, 128, [7], [0], spare=3).check() == 0


def test_bad_pages_and_positions():
    for norm in (None, "bf16"):
        case = Case(4, 2, 64, [10, 20, 0], [10, 3, 5], norm, max_position=22, spare=1)
        for table in (case.table, case.batch.d_block_table):
            table[0, 1] = len(case.cache.k_codes)
            table[2, 0] = -1
        lost = lambda s, pos: (s == 0 and pos >= 16) or s == 2 or pos >= 22  # noqa: E731
        pools = [p.clone() for p in (case.cache.k_codes, case.cache.v_scales)]
        efim.efim_kv4_append(case.cache, case.batch, case.norm, case.rope, case.q, case.k, case.v, case.out, case.status)
        assert case.status.item() == BAD_PAGE | BAD_POSITION
        row = 10 + 2
        assert (case.out[row].float() == 0).all() and torch.isnan(case.out[18].float()).all() and not torch.isnan(case.out[:18].float()).any()
        changed = [(p != q).flatten(3).any(3).any(1) for p, q in zip(pools, (case.cache.k_codes, case.cache.v_scales))]
        kept = torch.ones_like(changed[0])
        for s, (c, n) in enumerate(zip(case.cached, case.new)):
            for pos in range(c, c + n):
                if not lost(s, pos):
                    kept[case.table[s, pos // 16], pos % 16] = False
        assert not (changed[0] & kept).any() and not (changed[1] & kept).any()


def test_in_place_and_on_another_stream():
    case = Case(8, 2, 128, [30, 0], [3, 40], packed=True)
    case.out = case.q
    want = case.q.clone()
    efim.efim_kv_append(case.plain, case.batch, case.rope, want, case.k, case.v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    efim.efim_kv4_append(case.cache, case.batch, None, case.rope, case.q, case.k, case.v, case.q, case.status, stream=side)
    side.synchronize()
    assert torch.equal(case.q.view(torch.int16), want.view(torch.int16)) and case.status.item() == 0


@pytest.mark.parametrize("hkv,d", [(1, 64), (8, 128), (3, 128), (32, 64)])
@pytest.mark.parametrize("both", [True, False])
def test_unpack(hkv, d, both):
    """Every byte as code and as scale, pages twice and in any order; a page outside the pool leaves its place."""
    g = torch.Generator().manual_seed(d)
    codes, scales = ([torch.randint(256, (9, hkv, 16, d // n), generator=g, dtype=torch.uint8).cuda() for _ in range(2)] for n in (2, 16))
    cache = efim.Cache4(*codes, *scales, hkv, 0.5, 2.0 ** -30)
    pages = torch.tensor([3, 3, 8, -1, 0, 9, 5, -(1 << 31), (1 << 31) - 1], dtype=torch.int32, device="cuda")
    out = [torch.full((len(pages), hkv, 16, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    efim.efim_kv4_unpack(cache, pages, out[0] if both else None, out[1], status)
    assert status.item() == BAD_PAGE
    for x, scale in enumerate((0.5, 2.0 ** -30)):
        got = _f64(out[x])
        for i, page in enumerate(pages.tolist()):
            if 0 <= page < 9 and (both or x == 1):
                want = orc.held(codes[x][page].cpu().numpy(), scales[x][page].cpu().numpy(), scale)
                assert np.array_equal(got[i], want, equal_nan=True)
            else:
                assert (got[i] == 7).all()
