"""Arguments that the calls of a drafted step refuse, on the host and before any launch (a launch without a GPU is answered with
EFIM_ERR_CUDA; the addresses are never used)."""
import ctypes

import pytest

import paper_2505_21889_b200 as efim
from paper_2505_21889_b200 import binding as B
from paper_2505_21889_b200 import build as efim_build

OK, INVALID_ARG, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    efim_build.build()
    return efim.load_library()


def _norm_call(lib, cache=None, batch=None, norm=None, rope=None, q=0x1000000, q_stride=1536, k=0x1000800, k_stride=1536,
               v=0x1000A00, v_stride=1536, out=0x4000000):
    """8/2 heads x 128 as views of one projection of 10 tokens: rows of 1,536 values."""
    cache = cache or B._CacheDesc(0x10000, 0x20000, 64, 16, 8, 2, 128)
    batch = batch or B._BatchDesc(2, 8, 10, 0x1000, 0x1000, 0x1000, 0x1000, None, None)
    norm = norm or B._QkNormDesc(0x5000, 0x6000, 0, 1e-6, 0.0)
    return lib.efim_qk_norm_append(ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(norm),
                                   ctypes.byref(rope) if rope else None, q, q_stride, k, k_stride, v, v_stride, out, None, None)


def test_norm_append(lib):
    assert lib.efim_qk_norm_append(None, None, None, None, None, 0, None, 0, None, 0, None, None, None) == INVALID_ARG
    assert _norm_call(lib, cache=B._CacheDesc(0x10000, 0x20000, 64, 16, 8, 2, 96)) == UNSUPPORTED
    for batch in (B._BatchDesc(0, 8, 0), B._BatchDesc(2, 8, 0, 0x1000, 0x1000, 0x1000, 0x1000)):
        assert _norm_call(lib, batch=batch) == OK                                 # nothing to do
    nan, inf = float("nan"), float("inf")
    for norm in (B._QkNormDesc(0, 0, 0, 0.0, 0), B._QkNormDesc(0, 0, 0, -1e-6, 0), B._QkNormDesc(0, 0, 0, nan, 0),
                 B._QkNormDesc(0, 0, 0, inf, 0), B._QkNormDesc(0, 0, 2, 1e-6, 0), B._QkNormDesc(0x5008, 0, 0, 1e-6, 0),
                 B._QkNormDesc(0, 0x5004, 1, 1e-6, 0)):
        assert _norm_call(lib, norm=norm) == INVALID_ARG
    for bad in (dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(q=0x1000008), dict(out=0x4000002), dict(k=0x1000802),
                dict(v=0x1000A08), dict(q_stride=1020), dict(q_stride=1540), dict(k_stride=248), dict(v_stride=-1536)):
        assert _norm_call(lib, **bad) == INVALID_ARG, bad
    assert _norm_call(lib, rope=B._RopeDesc(0x30000, 0, 0)) == INVALID_ARG
    assert _norm_call(lib, rope=B._RopeDesc(0x30008, 100, 0)) == INVALID_ARG
    # results on top of what is still to be read: another token's row of q, k or v (the last one ends 10 rows behind the first)
    for out in (0x1000000, 0x1000010, 0x1000000 - 16, 0x1000000 - 10 * 2048 + 16, 0x1000000 + 9 * 3072 + 3072 - 16):
        assert _norm_call(lib, out=out) == INVALID_ARG
    packed = dict(q_stride=1024, k=0x2000000, k_stride=256, v=0x3000000, v_stride=256)
    for out in (0x2000000, 0x3000000 + 10 * 512 - 16, 0x1000000 + 2048):
        assert _norm_call(lib, out=out, **packed) == INVALID_ARG


def _lookup(lib, batch=2, hist=0x1000, stride=100, max_len=100, length=0x2000, lo=1, hi=4, k=3, drafts=0x3000, n=0x4000):
    return lib.efim_draft_lookup(batch, hist, stride, max_len, length, lo, hi, k, drafts, n, None, None)


def test_lookup(lib):
    for bad in (dict(batch=-1), dict(hist=None), dict(hist=0x1002), dict(stride=99), dict(max_len=0), dict(length=None), dict(lo=0),
                dict(lo=5), dict(k=0), dict(drafts=None), dict(n=None)):
        assert _lookup(lib, **bad) == INVALID_ARG, bad
    assert _lookup(lib, hi=33) == UNSUPPORTED
    assert _lookup(lib, batch=0, hist=None) == OK


def _verify(lib, accepted=0x1000, nxt=0x2000, out=None, logs=None, out_stride=0, ws=0x100000, ws_bytes=None, **changed):
    fields = dict(batch=2, total_rows=6, vocab=1000, target_kind=0, d_row_indptr=0x3000, d_tokens=0x4000, d_target=0x5002,
                  target_stride=1001, d_draft_probs=0x6004, draft_stride=1000, d_uniform=0x7000, d_noise=0x8000, noise_stride=1000,
                  d_temperature=0x9000)
    desc = B._VerifyDesc(**{**fields, **changed})
    if ws_bytes is None:
        ws_bytes = lib.efim_verify_workspace_bytes(desc.batch, desc.total_rows, desc.vocab, desc.target_kind)
    return lib.efim_verify_drafts(ctypes.byref(desc), accepted, nxt, out, logs, out_stride, ws, ws_bytes, None, None)


def test_verify(lib):
    assert lib.efim_verify_drafts(None, 0x1000, 0x1000, None, None, 0, 0x1000, 1 << 20, None, None) == INVALID_ARG
    for bad in (dict(batch=-1), dict(total_rows=-1), dict(vocab=0), dict(target_kind=3), dict(target_kind=-1), dict(d_row_indptr=None),
                dict(d_tokens=None), dict(d_target=None), dict(target_stride=999), dict(d_target=0x5001), dict(target_kind=1),
                dict(draft_stride=999), dict(d_draft_probs=0x6002), dict(d_uniform=None), dict(noise_stride=999),
                dict(d_noise=0x8001), dict(accepted=None), dict(nxt=None), dict(out=0xA000), dict(logs=0xA000, out_stride=-1),
                dict(target_kind=2, d_target=0x5004), dict(target_kind=2, d_target=0x5004, d_temperature=None, d_noise=None)):
        assert _verify(lib, **bad) == INVALID_ARG, bad
    assert _verify(lib, batch=0, d_row_indptr=None) == OK
    huge = (1 << 30) + 1
    assert _verify(lib, vocab=huge, target_stride=huge, draft_stride=huge, noise_stride=huge) == UNSUPPORTED
    size = lib.efim_verify_workspace_bytes
    wide = dict(vocab=100000, target_stride=100000, draft_stride=100000, noise_stride=100000)
    need = size(2, 6, 100000, 0)
    assert need > 0 and _verify(lib, ws_bytes=need - 1, **wide) == _verify(lib, ws=None, **wide) == WORKSPACE
    assert _verify(lib, ws=0x100010, **wide) == INVALID_ARG
    for smaller in ((1, 6, 100000), (2, 1, 100000), (2, 6, 40000), (2, 0, 100000)):
        assert 0 < size(*smaller, 0) <= need
    assert size(0, 6, 100000, 0) == size(2, 6, 0, 0) == 0
    assert [size(2, 6, v, k) == 0 for v, k in ((32768, 0), (32769, 0), (16384, 1), (16385, 1), (16384, 2), (16385, 2))] == [True, False] * 3


def test_python_side(lib):
    """Types, shapes and strides that the binding can see (tensors of the host, never read)."""
    torch = pytest.importorskip("torch")
    half, whole = torch.bfloat16, torch.int32
    pools = torch.zeros(4, 1, 16, 64, dtype=half)
    cache = efim.Cache(pools, pools.clone(), 2)
    batch = efim.Batch([0], [4], torch.zeros(1, 4, dtype=whole), device="cpu")
    norm = efim.QkNorm(None, None)
    x = torch.zeros(4, 300, dtype=half)
    good = dict(q=x[:, :128], k=x[:, 128:192], v=x[:, 192:256], q_out=torch.zeros(4, 2, 64, dtype=half))

    def append(**changed):
        efim.efim_qk_norm_append(cache, batch, norm, None, **{**good, **changed}, stream=0)
    for error, changed in [(ValueError, dict(q=x[:, :256:2])), (ValueError, dict(q=x[:3, :128])), (ValueError, dict(k=x[:, 128:200])),
                           (ValueError, dict(v=x[:, :64].reshape(4, 8, 8).transpose(1, 2))), (ValueError, dict(q_out=x[:, :128])),
                           (ValueError, dict(k=x[0, :64])), (TypeError, dict(k=x[:, :64].float())),
                           (TypeError, dict(q_out=good["q_out"].half()))]:
        with pytest.raises(error):
            append(**changed)
    with pytest.raises(ValueError):                     # weights of heads of another size
        efim.efim_qk_norm_append(cache, batch, efim.QkNorm(None, torch.zeros(32)), None, **good, stream=0)
    for bad in (lambda: efim.QkNorm(torch.zeros(8), torch.zeros(8, dtype=half)), lambda: efim.QkNorm(torch.zeros(16)[::2], None),
                lambda: efim.QkNorm(torch.zeros(8, dtype=torch.float16), None),
                lambda: efim.Rope.from_table(torch.zeros(4, 8, dtype=torch.float64)), lambda: efim.Rope.from_table(torch.zeros(8, 8).t()[:, :4])):
        with pytest.raises(ValueError):
            bad()
    hist, drafts, n = torch.zeros(2, 50, dtype=whole), torch.zeros(2, 3, dtype=whole), torch.zeros(2, dtype=whole)
    for error, args in [(ValueError, (hist[:, ::2], n, 1, 2, drafts, n)), (ValueError, (hist, n, 1, 2, drafts[:, :2], n)),
                        (ValueError, (hist, n, 1, 2, drafts[:1], n)), (TypeError, (hist.long(), n, 1, 2, drafts, n)),
                        (TypeError, (hist, n.long(), 1, 2, drafts, n)), (ValueError, (hist, n[:1], 1, 2, drafts, n)),
                        (ValueError, (hist, hist[:, 0], 1, 2, drafts, n)), (ValueError, (hist, n, 1, 2, drafts, drafts[:, 1])), (TypeError, (hist, n, 1, 2.5, drafts, n))]:
        with pytest.raises(error):
            efim.efim_draft_lookup(*args, stream=0)
    logits, ws = torch.zeros(5, 100, dtype=half), None
    r = dict(row_indptr=torch.zeros(3, dtype=whole), tokens=torch.zeros(5, dtype=whole), target=logits, accepted=n, next_token=n.clone(),
             uniform=torch.zeros(5), noise=torch.zeros(2, 100), workspace=ws)
    wide = torch.zeros(2, 6)
    for error, changed in [(TypeError, dict(target=logits.half())), (TypeError, dict(target=logits, target_is_probs=True)),
                           (TypeError, dict(noise=torch.zeros(2, 100, dtype=half))), (ValueError, dict(noise=torch.zeros(3, 100))),
                           (ValueError, dict(noise=torch.zeros(2, 99))), (ValueError, dict(draft_probs=torch.zeros(4, 100))),
                           (ValueError, dict(target=torch.zeros(100, 5, dtype=half).t())), (TypeError, dict(tokens=torch.zeros(5, dtype=torch.int64))),
                           (ValueError, dict(out_tokens=torch.zeros(2, 6, dtype=whole), out_logprobs=wide[:, :5].contiguous())),
                           (ValueError, dict(out_logprobs=wide[:, :5])), (ValueError, dict(out_tokens=torch.zeros(1, 6, dtype=whole))),
                           (TypeError, dict(temperature=torch.zeros(2, dtype=torch.float64))),
                           (ValueError, dict(row_indptr=torch.zeros(2, dtype=whole))), (ValueError, dict(tokens=torch.zeros(4, dtype=whole))),
                           (ValueError, dict(uniform=torch.zeros(4))), (ValueError, dict(uniform=torch.zeros(5, 2)[:, 0])),
                           (ValueError, dict(temperature=torch.zeros(1))), (ValueError, dict(accepted=hist[:, 0])),
                           (ValueError, dict(next_token=n[:1]))]:
        with pytest.raises(error):
            efim.efim_verify_drafts(**{**r, **changed}, stream=0)
    big = dict(target=torch.zeros(5, 40000, dtype=half), noise=torch.zeros(2, 40000))
    assert efim.efim_verify_workspace_bytes(2, logits) == 0 < efim.efim_verify_workspace_bytes(2, big["target"])
    with pytest.raises(efim.EfimError) as e:
        efim.efim_verify_drafts(**{**r, **big, "workspace": torch.zeros(256, dtype=torch.uint8)}, stream=0)
    assert e.value.code == WORKSPACE
