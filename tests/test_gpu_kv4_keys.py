"""Keys of the 4-bit append against their definition: norm and rotation in 64 bits, rounded to fp32 and that to bf16, then to blocks.  What is
held is whole numbers, which have to be the oracle's: a key in fp32 that lies next to a border may come out on the other side of it, and then a code,
or all sixteen of a block, are others."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from oracle import efim_kv4_oracle as orc
from oracle.efim_oracle import bf16_to_f64

pytestmark = pytest.mark.gpu


def _f64(t):
    return bf16_to_f64(t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16))


def _check(k, hq, first=0, table=None, interleaved=False, weight=None, offset=0.0, eps=1e-6, g=0.5):
    """Keys [tokens, heads, D] of one sequence at positions from `first` on, appended beside queries and values."""
    t, hkv, d = k.shape
    pages = -(-(first + t) // 16)
    cache = efim.Cache4.empty(pages, hkv, d, hq, g, 1.0)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    batch = efim.Batch([first], [t], order.view(1, -1).numpy())
    rope = efim.Rope.from_table(table, interleaved) if table is not None else None
    norm = efim.QkNorm(weight, weight, eps, offset) if weight is not None else None
    q = torch.ones(t, hq, d, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    efim.efim_kv4_append(cache, batch, norm, rope, q, k, k, q, status)
    torch.cuda.synchronize()
    assert status.item() == 0
    at, slot = order.long()[torch.arange(first, first + t) // 16], torch.arange(first, first + t) % 16
    got = [pool[at.cuda(), :, slot.cuda()].cpu().numpy() for pool in (cache.k_codes, cache.k_scales)]
    for lo in range(0, t, 1600):
        rows = slice(lo, min(t, lo + 1600))
        turn = table[first + lo:first + rows.stop].cpu().numpy()[:, None] if table is not None else None
        w = weight.double().cpu().numpy() + offset if weight is not None else None
        codes, scales = orc.quantize(orc.key(_f64(k[rows]), turn, interleaved, w, float(np.float32(eps))), g)
        assert np.array_equal(got[1][rows], scales), int((got[1][rows] != scales).sum())
        nan = np.repeat(scales == 127, 8, axis=-1)                          # (their codes say nothing)
        assert not ((got[0][rows] != codes) & ~nan).any(), int((got[0][rows] != codes).sum())


def _table(d, positions, size=1.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    return (size * torch.cat([angle.cos(), angle.sin()], 1)).float().cuda()


def _keys(t, hkv, d, seed, size=1.0):
    x = size * torch.randn(t, hkv, d, generator=torch.Generator().manual_seed(seed))
    return (x * (1 + 3 * (torch.arange(d) % 23 == 5))).bfloat16().cuda()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_many_keys(norm, interleaved):
    """Ten million values: a dozen normalised ones lie so near to a border that fp32 takes the other side."""
    weight = (1 + 0.2 * torch.randn(128, generator=torch.Generator().manual_seed(3))).bfloat16().cuda() if norm else None
    _check(_keys(9600, 8, 128, norm + 2 * interleaved), 8, 5120, _table(128, 14720), interleaved, weight)


@pytest.mark.parametrize("hq,hkv,d", [(3, 3, 64), (1, 1, 128), (9, 3, 128), (5, 5, 64)])
@pytest.mark.parametrize("rotated", [False, True])
def test_heads_that_share_a_warp_with_queries_and_values(hq, hkv, d, rotated):
    weight = (0.3 * torch.randn(d, generator=torch.Generator().manual_seed(hq))).cuda()
    for offset in (0.0, 1.0):
        _check(_keys(2000, hkv, d, hq), hq, 3, _table(d, 2003) if rotated else None, False, weight, offset)


@pytest.mark.parametrize("size", [1e-30, 1e-5, 1e18, 1e30])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes(size, interleaved):
    """Heads whose squares leave fp32, and heads beside which eps counts."""
    k = _keys(700, 4, 64, 4, size)
    weight = (1 + 0.2 * torch.randn(64, generator=torch.Generator().manual_seed(3))).bfloat16().cuda()
    _check(k, 4, 0, _table(64, 700), interleaved, weight)
    _check(k, 4, 0, _table(64, 700), interleaved, None, g=2.0 ** 60 if size > 1 else 2.0 ** -60 if size < 1e-20 else 2.0 ** -15)


def test_ends_of_the_range():
    """Sums beyond bf16 and beyond fp32 (a scaled table), zeros of both signs, infinities, NaN."""
    k = _keys(64, 2, 128, 5)
    for interleaved in (False, True):
        for size, scale in ((3e38, 1.0), (3e38, 4.0), (1e38, 3.0)):
            big = (k.sign().float() * size).bfloat16()
            _check(big, 2, 0, _table(128, 64, scale), interleaved, g=2.0 ** 60)
        special = k.clone()
        special[0], special[1, 0, ::3], special[2, 1, 7], special[3, 0, 70], special[4, 1, 40] = 0.0, -0.0, float("inf"), float("nan"), -float("inf")
        for weight in (None, torch.full((128,), 1.5, device="cuda")):
            _check(special, 2, 0, _table(128, 64), interleaved, weight)


@pytest.mark.parametrize("interleaved", [False, True])
def test_products_beyond_fp32_that_cancel(interleaved):
    """In one pair of a head: the result's sign is that of the sum, not of the product that left fp32."""
    k = _keys(64, 2, 128, 6)
    k[:, :, 3], k[:, :, 2 if interleaved else 67] = 1e38, 1.1e38
    for g in (2.0 ** 60, 0.5):
        _check(k, 2, 0, _table(128, 64, 8.0), interleaved, g=g)


@pytest.mark.parametrize("tokens,hq,hkv,d", [(3000, 40, 40, 128), (4000, 20, 20, 128), (700, 200, 100, 64)])
def test_many_heads(tokens, hq, hkv, d):
    """Several groups of keys a warp, beside warps that have none."""
    weight = (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(3))).cuda()
    _check(_keys(tokens, hkv, d, hkv), hq, 0, _table(d, tokens), False, weight)
