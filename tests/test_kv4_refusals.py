"""Arguments that the calls of a step over a 4-bit cache refuse, on the host and before any launch (a launch without a GPU is answered
with EFIM_ERR_CUDA; the addresses are never used)."""
import ctypes

import pytest

import paper_2505_21889_b200 as efim
from paper_2505_21889_b200 import binding as B
from paper_2505_21889_b200 import build as efim_build

OK, INVALID_ARG, UNSUPPORTED, OUT_OF_RANGE, WORKSPACE = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    efim_build.build()
    return efim.load_library()


def _cache(**changed):
    fields = dict(d_k_codes=0x10000, d_v_codes=0x20000, d_k_scales=0x30000, d_v_scales=0x40000, num_pages=64, page_size=16, num_q_heads=8,
                  num_kv_heads=2, head_dim=128, k_scale=1.0, v_scale=0.5)
    return B._Cache4Desc(**{**fields, **changed})


BAD_CACHES = [(dict(d_k_codes=None), INVALID_ARG), (dict(d_v_codes=0x20040), INVALID_ARG), (dict(d_k_scales=None), INVALID_ARG),
              (dict(d_v_scales=0x40010), INVALID_ARG), (dict(num_pages=0), INVALID_ARG), (dict(num_q_heads=7), INVALID_ARG),
              (dict(num_kv_heads=0), INVALID_ARG), (dict(page_size=32), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
              (dict(head_dim=256), UNSUPPORTED), (dict(num_pages=(1 << 31) - 1), UNSUPPORTED),
              *((dict(k_scale=x), INVALID_ARG) for x in (0.0, -1.0, 3.0, float("nan"), float("inf"), 2.0 ** 61, 2.0 ** -61, 1e-40)),
              (dict(v_scale=1.5), INVALID_ARG)]


def _append(lib, cache=None, batch=None, norm=None, rope=None, q=0x1000000, q_stride=1536, k=0x1000800, k_stride=1536, v=0x1000A00,
            v_stride=1536, out=0x4000000):
    batch = batch or B._BatchDesc(2, 8, 10, 0x1000, 0x1000, 0x1000, 0x1000, None, None)
    ref = lambda x: ctypes.byref(x) if x is not None else None  # noqa: E731
    return lib.efim_kv4_append(ctypes.byref(cache or _cache()), ref(batch), ref(norm), ref(rope), q, q_stride, k, k_stride, v, v_stride, out, None, None)


def test_append(lib):
    for changed, status in BAD_CACHES:
        assert _append(lib, cache=_cache(**changed)) == status, changed
    assert lib.efim_kv4_append(None, None, None, None, None, 0, None, 0, None, 0, None, None, None) == INVALID_ARG
    assert lib.efim_kv4_append(ctypes.byref(_cache()), None, None, None, None, 0, None, 0, None, 0, None, None, None) == INVALID_ARG
    for batch in (B._BatchDesc(0, 8, 0), B._BatchDesc(2, 8, 0, 0x1000, 0x1000, 0x1000, 0x1000)):
        assert _append(lib, batch=batch) == OK
    for batch in (B._BatchDesc(-1, 8, 1), B._BatchDesc(2, 0, 1, 0x1000, 0x1000, 0x1000, 0x1000), B._BatchDesc(2, 8, -1), B._BatchDesc(2, 8, 4, 0x1000)):
        assert _append(lib, batch=batch) == INVALID_ARG
    for norm in (B._QkNormDesc(0, 0, 0, 0.0, 0), B._QkNormDesc(0, 0, 0, float("nan"), 0), B._QkNormDesc(0, 0, 2, 1e-6, 0), B._QkNormDesc(0x5008, 0, 0, 1e-6, 0)):
        assert _append(lib, norm=norm) == INVALID_ARG
    for bad in (dict(k=None), dict(v=None), dict(q=None), dict(out=None), dict(q=0x1000008), dict(out=0x4000002), dict(q_stride=1020),
                dict(q_stride=1540), dict(k_stride=248), dict(v_stride=-1536), dict(rope=B._RopeDesc(0x30000, 0, 0)),
                dict(rope=B._RopeDesc(0x30008, 100, 0)), dict(out=0x1000000), dict(out=0x1000010)):
        assert _append(lib, **bad) == INVALID_ARG, bad


def test_unpack(lib):
    def call(cache=None, pages=0x1000, n=5, k=0x100000, v=0x200000):
        return lib.efim_kv4_unpack(ctypes.byref(cache or _cache()), pages, n, k, v, None, None)
    for changed, status in BAD_CACHES:
        assert call(cache=_cache(**changed)) == status
    assert call(n=0) == OK
    for bad in (dict(n=-1), dict(pages=None), dict(k=None, v=None), dict(k=0x100008), dict(v=0x200001)):
        assert call(**bad) == INVALID_ARG, bad


def _decode(lib, cache=None, batch=3, ctx=0x1000, max_ctx=3000, table=0x2000, width=200, indptr=0x3000, rows=9, new=4, q=0x100000, out=0x200000,
            ws=0x800000, ws_bytes=None):
    cache = cache or _cache()
    if ws_bytes is None:
        ws_bytes = lib.efim_kv4_decode_workspace_bytes(ctypes.byref(cache), max(batch, 1), max(new, 1), max_ctx)
    return lib.efim_kv4_decode_attn(ctypes.byref(cache), batch, ctx, max_ctx, table, width, indptr, rows, new, q, out, None, 0.0, ws, ws_bytes, None, None)


def test_decode(lib):
    for changed, status in BAD_CACHES:
        assert _decode(lib, cache=_cache(**changed)) == status, changed
    for bad in (dict(batch=-1), dict(width=0), dict(rows=-1), dict(new=0), dict(indptr=None), dict(indptr=None, new=1), dict(ctx=None), dict(table=None),
                dict(q=None), dict(out=None), dict(q=0x100008), dict(out=0x200002), dict(ws=0x800010)):
        assert _decode(lib, **bad) == INVALID_ARG, bad
    assert _decode(lib, max_ctx=3201) == OUT_OF_RANGE
    assert _decode(lib, batch=0) == _decode(lib, rows=0) == OK
    size = lib.efim_kv4_decode_workspace_bytes
    need = size(ctypes.byref(_cache()), 3, 4, 3000)
    assert need > 0 and _decode(lib, ws_bytes=need - 1) == _decode(lib, ws=None) == WORKSPACE
    assert size(ctypes.byref(_cache()), 0, 4, 3000) == size(ctypes.byref(_cache()), 3, 0, 3000) == size(ctypes.byref(_cache(head_dim=32)), 3, 4, 3000) == 0
    assert size(ctypes.byref(_cache()), 3, 1, 200) == 0
    assert _decode(lib, new=1 << 30, ws_bytes=0) == UNSUPPORTED


def test_prefill(lib):
    import numpy as np
    cached, new = np.array([500, 0, 70], np.int32), np.array([200, 0, 90], np.int32)

    def call(cache=None, q=0x100000, out=0x200000, ws=0x8000000, ws_bytes=None, **changed):
        fields = dict(batch=3, max_pages_per_seq=64, total_new_tokens=290, d_cached_len=0x1000, d_new_len=0x1000, d_q_indptr=0x1000,
                      d_block_table=0x1000, h_cached_len=cached.ctypes.data, h_new_len=new.ctypes.data)
        c, b = ctypes.byref(cache or _cache()), ctypes.byref(B._BatchDesc(**{**fields, **changed}))
        n = lib.efim_kv4_prefill_workspace_bytes(c, b) if ws_bytes is None else ws_bytes
        return lib.efim_kv4_append_prefill_attn(c, b, q, out, None, 0.0, ws, n, None, None), n
    for changed, status in BAD_CACHES:
        assert call(cache=_cache(**changed)) == (status, 0), changed
    for bad in (dict(q=None), dict(out=0x200008), dict(ws=0x8000080)):
        assert call(**bad)[0] == INVALID_ARG, bad
    for bad in (dict(total_new_tokens=289), dict(h_new_len=None), dict(d_new_len=None)):
        assert call(**bad) == (INVALID_ARG, 0), bad
    assert call(max_pages_per_seq=40) == (OUT_OF_RANGE, 0)
    need = call()[1]
    assert need > 2 * 54 * 2 * 16 * 128 * 2 and call(ws_bytes=need - 1)[0] == call(ws=None)[0] == WORKSPACE
    assert call(batch=0)[0] == OK


def _tables(lib, batch=2, cached=0x1000, new=0x1100, table=0x2000, width=10, free=0x3000, capacity=50, count=0x4000, out=0x5000, count_out=0x4000,
            indptr=0x6000, rows=20, positions=0x7000, slots=0x8000, seqs=0x9000, ws=0xA000, ws_bytes=12):
    return lib.efim_step_tables(batch, cached, new, table, width, free, capacity, count, out, count_out, indptr, rows, positions, slots, seqs, ws,
                                ws_bytes, None, None)


def test_tables(lib):
    for bad in (dict(batch=-1), dict(width=0), dict(capacity=-1), dict(rows=-1), dict(cached=None), dict(new=None), dict(table=None), dict(free=None),
                dict(count=None), dict(out=None), dict(count_out=None), dict(indptr=None), dict(cached=0x1002), dict(slots=0x8004),
                dict(positions=0x7001), dict(ws=0xA002)):
        assert _tables(lib, **bad) == INVALID_ARG, bad
    assert _tables(lib, ws=None) == _tables(lib, ws_bytes=11) == WORKSPACE
    assert _tables(lib, batch=0) == OK and lib.efim_step_tables_workspace_bytes(0) == 0
    def release(batch=2, keep=0x1000, table=0x2000, width=10, free=0x3000, capacity=50, count=0x4000, ws=0xA000, ws_bytes=12):
        return lib.efim_release_pages(batch, keep, table, width, free, capacity, count, ws, ws_bytes, None, None)
    for bad in (dict(batch=-1), dict(width=0), dict(capacity=-1), dict(keep=None), dict(table=0x2001), dict(free=None), dict(count=None), dict(ws=0xA001)):
        assert release(**bad) == INVALID_ARG, bad
    assert release(ws=None) == release(ws_bytes=8) == WORKSPACE
    assert release(batch=0) == OK


def _adjust(lib, out=0x9000000, out_stride=1001, **changed):
    fields = dict(batch=2, total_rows=6, vocab=1000, logits_f32=0, d_row_indptr=0x1000, d_logits=0x2000, logits_stride=1001, d_tokens=0x3000,
                  d_history=0x4000, history_stride=100, max_len=100, bias_entries=3, d_len=0x5000, d_prompt_len=0x6000, d_repetition=0x7000,
                  d_presence=0x7100, d_frequency=0x7200, d_bias_indptr=0x7300, d_bias_tokens=0x7400, d_bias=0x7500, d_mask=0x7600, mask_stride=32)
    return lib.efim_adjust_logits(ctypes.byref(B._AdjustDesc(**{**fields, **changed})), out, out_stride, None, None)


def test_adjust(lib):
    assert lib.efim_adjust_logits(None, 0x1000, 10, None, None) == INVALID_ARG
    for bad in (dict(batch=-1), dict(total_rows=-1), dict(vocab=0), dict(logits_f32=2), dict(d_row_indptr=None), dict(d_logits=None), dict(out=None),
                dict(logits_stride=999), dict(out_stride=999), dict(d_logits=0x2001), dict(logits_f32=1, d_logits=0x2002), dict(d_len=None),
                dict(max_len=0), dict(history_stride=99), dict(d_history=None), dict(d_bias_indptr=None), dict(d_bias_tokens=None),
                dict(bias_entries=-1), dict(mask_stride=31), dict(d_mask=0x7602), dict(d_tokens=0x3001),
                dict(out=0x2002), dict(out=0x2000, out_stride=1002), dict(out=0x2000 + 5 * 2002 + 1998)):
        assert _adjust(lib, **bad) == INVALID_ARG, bad
    assert _adjust(lib, batch=0) == _adjust(lib, total_rows=0) == OK
    huge = (1 << 30) + 1
    assert _adjust(lib, vocab=huge, logits_stride=huge, out_stride=huge, mask_stride=huge) == UNSUPPORTED
    assert _adjust(lib, total_rows=huge) == UNSUPPORTED


def test_python_side(lib):
    """Types, shapes and strides that the binding can see (tensors of the host, never read)."""
    torch = pytest.importorskip("torch")
    half, whole, byte = torch.bfloat16, torch.int32, torch.uint8
    codes, scales = torch.zeros(4, 1, 16, 32, dtype=byte), torch.zeros(4, 1, 16, 4, dtype=byte)
    cache = efim.Cache4(codes, codes.clone(), scales, scales.clone(), 2)
    for bad in ((codes.int(), codes, scales, scales), (codes, codes[:3], scales, scales), (codes, codes, scales[..., :2], scales),
                (codes, codes, scales, torch.zeros(4, 1, 16, 8, dtype=byte)[..., ::2]), (codes[0], codes[0], scales[0], scales[0]),
                (codes, codes, scales.view(torch.float8_e4m3fn), scales)):
        with pytest.raises(ValueError):
            efim.Cache4(*bad, 2)
    batch = efim.Batch([0], [4], torch.zeros(1, 4, dtype=whole), device="cpu")
    x = torch.zeros(4, 300, dtype=half)
    good = dict(q=x[:, :128], k=x[:, 128:192], v=x[:, 192:256], q_out=torch.zeros(4, 2, 64, dtype=half))
    rope = efim.Rope.from_table(torch.zeros(64, 128))
    for error, norm, r, changed in [(ValueError, None, None, dict(q=x[:3, :128])), (ValueError, None, None, dict(k=x[:, 128:200])),
                                    (TypeError, None, None, dict(v=x[:, :64].float())), (ValueError, None, None, dict(q_out=x[:, :128])),
                                    (ValueError, None, rope, {}), (ValueError, efim.QkNorm(None, torch.zeros(32)), None, {})]:
        with pytest.raises(error):
            efim.efim_kv4_append(cache, batch, norm, r, **{**good, **changed}, stream=0)
    pages, page = torch.zeros(3, dtype=whole), torch.zeros(3, 1, 16, 64, dtype=half)
    for error, args in [(ValueError, (pages[:2], page, page)), (TypeError, (pages.long(), page, page)), (ValueError, (pages, page[:2], page)),
                        (TypeError, (pages, page.float(), None)), (ValueError, (pages, page[..., :32], None))]:
        with pytest.raises(error):
            efim.efim_kv4_unpack(cache, *args, stream=0)
    n, table, q = torch.zeros(2, dtype=whole), torch.zeros(2, 5, dtype=whole), torch.zeros(2, 2, 64, dtype=half)
    call = dict(cache=cache, batch=2, d_ctx_len=n, max_ctx_len=80, d_block_table=table, q=q, out=q.clone())
    for error, changed in [(ValueError, dict(d_ctx_len=n[:1])), (TypeError, dict(d_ctx_len=n.long())), (ValueError, dict(d_block_table=table[:1])),
                           (ValueError, dict(d_block_table=table[:, :4])), (ValueError, dict(q=q[:, :1])), (ValueError, dict(out=q[:1])),
                           (TypeError, dict(q=q.float())), (ValueError, dict(q_indptr=n)), (ValueError, dict(lse=torch.zeros(3))),
                           (TypeError, dict(status=n.long())), (OverflowError, dict(max_ctx_len=1 << 32)),
                           (ValueError, dict(q=torch.zeros(2, 4, 64, dtype=half)[:, ::2]))]:
        with pytest.raises(error):
            efim.efim_kv4_decode_attn(**{**call, **changed}, stream=0)
    with pytest.raises(efim.EfimError) as e:                                  # more rows than sequences, without their offsets
        efim.efim_kv4_decode_attn(**{**call, "q": torch.zeros(3, 2, 64, dtype=half), "out": torch.zeros(3, 2, 64, dtype=half)}, stream=0)
    assert e.value.code == INVALID_ARG
    with pytest.raises(ValueError):
        efim.efim_kv4_append_prefill_attn(cache, batch, good["q_out"][:3], good["q_out"][:3], stream=0)
    free, count, ws = torch.zeros(9, dtype=whole), torch.zeros(1, dtype=whole), torch.zeros(64, dtype=byte)
    call = dict(cached_len=n, new_len=n, block_table=table, free_pages=free, num_free=count, q_indptr=torch.zeros(3, dtype=whole), workspace=ws)
    for error, changed in [(ValueError, dict(cached_len=n[:1])), (ValueError, dict(q_indptr=n)), (TypeError, dict(slots=free)),
                           (ValueError, dict(positions=free, sequences=free[:8].clone())), (ValueError, dict(block_table_out=table[:, :4].contiguous())),
                           (ValueError, dict(block_table=table[:, ::2])), (ValueError, dict(free_pages=torch.zeros(9, 2, dtype=whole)[:, 0])),
                           (TypeError, dict(num_free=count.long())), (ValueError, dict(num_free_out=count[:0])), (TypeError, dict(new_len=n.float()))]:
        with pytest.raises(error):
            efim.efim_step_tables(**{**call, **changed}, stream=0)
    with pytest.raises(ValueError):
        efim.efim_release_pages(n[:1], table, free, count, workspace=ws, stream=0)
    with pytest.raises(efim.EfimError) as e:
        efim.efim_release_pages(n, table, free, count, workspace=ws[:8], stream=0)
    assert e.value.code == WORKSPACE
    logits, hist = torch.zeros(5, 100, dtype=half), torch.zeros(2, 50, dtype=whole)
    call = dict(row_indptr=torch.zeros(3, dtype=whole), logits=logits, history=hist, lengths=n, repetition=torch.ones(2))
    for error, changed in [(TypeError, dict(logits=logits.half())), (ValueError, dict(logits=logits[:, ::2])), (ValueError, dict(history=hist[:1])),
                           (TypeError, dict(history=hist.long())), (ValueError, dict(lengths=n[:1])), (ValueError, dict(repetition=torch.ones(1))),
                           (TypeError, dict(presence=n)), (ValueError, dict(tokens=torch.zeros(4, dtype=whole))), (ValueError, dict(out=logits[:4].clone())),
                           (TypeError, dict(out=logits.float())), (ValueError, dict(mask=torch.zeros(5, 3, dtype=whole))),
                           (ValueError, dict(mask=torch.zeros(4, 4, dtype=whole))), (ValueError, dict(bias=(torch.zeros(3, dtype=whole), n, torch.zeros(3)))),
                           (ValueError, dict(bias=(n, n, torch.zeros(2)))), (ValueError, dict(logits=torch.zeros(5, 2, 50, dtype=half)))]:
        with pytest.raises(error):
            efim.efim_adjust_logits(**{**call, **changed}, stream=0)
    with pytest.raises(efim.EfimError) as e:
        efim.efim_adjust_logits(**{**call, "history": None, "lengths": None}, stream=0)
    assert e.value.code == INVALID_ARG


def test_batches_of_lengths_on_the_device():
    torch = pytest.importorskip("torch")
    n, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 5, dtype=torch.int32)
    batch = efim.Batch.from_device(n, n, torch.zeros(3, dtype=torch.int32), table, 7)
    assert batch.desc.total_new_tokens == 7 and batch.desc.max_pages_per_seq == 5
    for bad in ((n.long(), n, torch.zeros(3, dtype=torch.int32), table), (n, n[:1], torch.zeros(3, dtype=torch.int32), table),
                (n, n, n, table), (n, n, torch.zeros(3, dtype=torch.int32), table[:, :3]), (n, n, torch.zeros(3, dtype=torch.int32), n)):
        with pytest.raises(ValueError):
            efim.Batch.from_device(*bad, 7)
    cache = efim.Cache(*(torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16) for _ in range(2)), 2)
    q, k = torch.zeros(7, 2, 64, dtype=torch.bfloat16), torch.zeros(7, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: efim.efim_kv_append(cache, batch, None, q, k, k, stream=0),
                 lambda: efim.efim_qk_norm_append(cache, batch, efim.QkNorm(None, None), None, q, k, k, q, stream=0)):
        with pytest.raises(ValueError, match="device"):
            call()
    assert efim.efim_prefill_workspace_bytes(cache, batch) == 0
    with pytest.raises(efim.EfimError):
        efim.efim_append_prefill_attn(cache, batch, q, q.clone(), workspace=torch.zeros(256, dtype=torch.uint8), stream=0)
