"""efim_kv4_append_prefill_attn: against the float64 definition, with the bounds of the single-token form where few rows go through its
kernel; where the pages are unpacked the results are those of efim_append_prefill_attn on the same values, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2505_21889_b200 as efim
from tests.test_gpu_kv4_attn import Case as Attn, HEADS, _f64
from oracle import efim_kv4_oracle as orc

pytestmark = pytest.mark.gpu


class Case(Attn):
    def run(self, stream=None):
        self.batch = efim.Batch([c - n for c, n in zip(self.ctx, self.new)], self.new, self.table.numpy())
        size = efim.efim_kv4_prefill_workspace_bytes(self.cache, self.batch)
        self.ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        efim.efim_kv4_append_prefill_attn(self.cache, self.batch, self.q, self.out, self.lse, workspace=self.ws, status=self.status, stream=stream)

    def bf16(self):
        """The same on a bf16 cache of the same values."""
        n, hkv = self.cache.k_codes.shape[:2]
        pools = [torch.empty(n, hkv, 16, self.shape[2], dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        efim.efim_kv4_unpack(self.cache, torch.arange(n, dtype=torch.int32, device="cuda"), *pools)
        cache = efim.Cache(*pools, self.shape[0])
        out, lse = torch.full_like(self.out, 5.0), torch.full_like(self.lse, 5.0)
        ws = torch.empty(efim.efim_prefill_workspace_bytes(cache, self.batch), dtype=torch.uint8, device="cuda")
        efim.efim_append_prefill_attn(cache, self.batch, self.q, out, lse, 0.0, ws)
        return out, lse


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("new", [(1, 1, 1), (1, 2, 1)])
def test_few_rows(hq, hkv, d, new):
    """Up to 16 rows a kv head go through the decode kernel here, more are the bf16 call's results."""
    case = Case(hq, hkv, d, [50, 800, 17], new, seed=hq)
    case.run()
    if max(new) * hq // hkv <= 16:
        case.check()
    else:
        out, lse = case.bf16()
        assert torch.equal(case.out.view(torch.int16), out.view(torch.int16)) and torch.equal(case.lse, lse)
    assert case.status.item() == 0


def test_few_rows_of_many_pages():
    """From 64 (page, kv head) pairs an SM on, up to 80 rows do."""
    case = Case(32, 8, 128, [8000, 16000, 500], [3, 20, 1], seed=1)
    case.run()
    case.check(only={0, 2})
    assert case.status.item() == 0


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (8, 8, 64), (24, 1, 64)])
@pytest.mark.parametrize("new", [(100, 1, 70), (0, 300, 0), (257, 256, 0), (65, 0, 1)])
def test_many_rows(hq, hkv, d, new):
    """The bf16 call's results; lengths without new tokens, contexts that are the new tokens alone."""
    ctx = [max(c, n) for c, n in zip((1300, 40, 90), new)]
    case = Case(hq, hkv, d, ctx, new, seed=sum(new))
    case.run()
    out, lse = case.bf16()
    torch.cuda.synchronize()
    assert case.status.item() == 0
    assert torch.equal(case.out.view(torch.int16), out.view(torch.int16)) and torch.equal(case.lse, lse)
    # and the definition's, on the last row of the first sequence that has one; bf16 weights there: 2^-8 of each
    s = next(i for i, n in enumerate(new) if n)
    row = sum(new[:s + 1]) - 1
    k_pool, v_pool = case.held()
    pages = case.table[s, :-(-ctx[s] // 16)].numpy()
    k, v = (x[pages, 0].reshape(-1, d)[:ctx[s]] for x in (k_pool, v_pool))
    want, _, size, _ = orc.attend(_f64(case.q[row, :1]), k, v, [ctx[s]], d ** -0.5)
    assert (np.abs(_f64(case.out[row, :1]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * size + 1e-3).all()


def test_bad_pages_and_another_stream():
    case = Case(32, 8, 128, [200, 300], [40, 40])
    case.table[0, 3] = -9
    case.run(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert case.status.item() == 1
    out, _ = case.bf16()
    assert torch.equal(case.out[40:].view(torch.int16), out[40:].view(torch.int16)) and torch.isfinite(case.out.float()).all()


def test_workspace_is_checked():
    for new in ([1, 2], [40, 50]):
        case = Case(32, 8, 128, [2000, 300], new)
        case.run()
        assert len(case.ws) > 1
        with pytest.raises(efim.EfimError) as e:
            efim.efim_kv4_append_prefill_attn(case.cache, case.batch, case.q, case.out, workspace=case.ws[:-1])
        assert e.value.code == 4
