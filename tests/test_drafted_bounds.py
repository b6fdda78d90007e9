"""Sizes and arguments at the ends of what the calls of a drafted step take, on the host and before any launch (the addresses are
never used)."""
import ctypes

import pytest

import paper_2505_21889_b200 as efim
from paper_2505_21889_b200 import binding as B
from paper_2505_21889_b200 import build as efim_build

UNSUPPORTED = 2


@pytest.fixture(scope="module")
def lib():
    efim_build.build()
    return efim.load_library()


def _verify(lib, **changed):
    fields = dict(batch=2, total_rows=6, vocab=1000, target_kind=0, d_row_indptr=0x3000, d_tokens=0x4000, d_target=0x5002,
                  target_stride=1001, d_draft_probs=0x6004, draft_stride=1000, d_uniform=0x7000, d_noise=0x8000, noise_stride=1000,
                  d_temperature=0x9000)
    desc = B._VerifyDesc(**{**fields, **changed})
    size = lib.efim_verify_workspace_bytes(desc.batch, desc.total_rows, desc.vocab, desc.target_kind)
    return lib.efim_verify_drafts(ctypes.byref(desc), 0x1000, 0x2000, None, None, 0, 0x100000, size, None, None)


def test_rows_are_counted_in_32_bits(lib):
    assert _verify(lib, total_rows=(1 << 30) + 1) == _verify(lib, total_rows=(1 << 31) - 1) == UNSUPPORTED
    assert _verify(lib, total_rows=(1 << 31) - 1, batch=1000, vocab=8, target_stride=8) == UNSUPPORTED


def test_rotary_tables_of_another_width(lib):
    """A table's rows are head_dim apart: one of another width would be read at other rows, and past its end."""
    torch = pytest.importorskip("torch")
    half, whole = torch.bfloat16, torch.int32
    cache = efim.Cache(torch.zeros(4, 1, 16, 128, dtype=half), torch.zeros(4, 1, 16, 128, dtype=half), 2)
    batch = efim.Batch([0], [4], torch.zeros(1, 4, dtype=whole), device="cpu")
    q, k = torch.zeros(4, 2, 128, dtype=half), torch.zeros(4, 1, 128, dtype=half)
    one = torch.ones(1, dtype=whole)
    for rope in (efim.Rope.from_table(torch.zeros(64, 64)), efim.Rope.from_table(torch.zeros(64, 256)),
                 efim.Rope(10000.0, 64, 64, False, "cpu")):
        for call in (lambda: efim.efim_qk_norm_append(cache, batch, efim.QkNorm(None, None), rope, q, k, k, q.clone(), stream=0),
                     lambda: efim.efim_kv_append(cache, batch, rope, q, k, k, stream=0),
                     lambda: efim.efim_append_prefill_step(cache, batch, rope, q, k, k, q.clone(), stream=0),
                     lambda: efim.efim_decode_step(cache, 1, one, 4, batch.d_block_table, rope, q[:1], k[:1], k[:1], q[:1].clone(),
                                                   stream=0)):
            with pytest.raises(ValueError, match="rotary"):
                call()
    # a table that fits goes on to the launch, which needs a GPU, or to the next refusal
    fits = efim.Rope.from_table(torch.zeros(64, 128))
    with pytest.raises(efim.EfimError):
        efim.efim_append_prefill_step(cache, batch, fits, q, k, k, q.clone(), stream=0)


def test_norm_weights_of_no_values():
    """None stands for weights of one; a vector without values does not, and is not read past its end."""
    torch = pytest.importorskip("torch")
    for dtype in (torch.bfloat16, torch.float32):
        for empty in (torch.zeros(0, dtype=dtype), torch.zeros(128, dtype=dtype)[:0]):
            with pytest.raises(ValueError):
                efim.QkNorm(empty, empty)
            with pytest.raises(ValueError):
                efim.QkNorm(None, empty)


def test_rows_that_are_no_lines(lib):
    """[batch, k + 1, vocab] is not [rows, vocab]: folded into rows of (k + 1) vocab it would be judged by wrong rows.  Dimensions of
    size 1 between change nothing."""
    torch = pytest.importorskip("torch")
    whole = torch.int32
    n = torch.zeros(2, dtype=whole)
    tokens, indptr = torch.zeros(6, dtype=whole), torch.tensor([0, 3, 6], dtype=whole)
    block = torch.zeros(2, 3, 40000)                                      # of a size that needs a workspace
    rows, noise, small = block.view(6, 40000), torch.ones(2, 40000), torch.zeros(256, dtype=torch.uint8)

    def verify(**changed):
        efim.efim_verify_drafts(**{**dict(row_indptr=indptr, tokens=tokens, target=rows, accepted=n, next_token=n.clone(),
                                          uniform=torch.zeros(6), noise=noise, workspace=small), **changed}, stream=0)
    for changed in (dict(target=block, noise=None), dict(target=block, noise=torch.ones(2, 120000)), dict(noise=noise.view(2, 200, 200)),
                    dict(draft_probs=rows.view(6, 2, 20000))):
        with pytest.raises(ValueError):
            verify(**changed)
    with pytest.raises(ValueError):
        efim.efim_verify_workspace_bytes(2, block)
    assert efim.efim_verify_workspace_bytes(2, rows[:, None]) == efim.efim_verify_workspace_bytes(2, rows) > 0
    for fits in (dict(), dict(target=rows[:, None], draft_probs=rows[:, None], noise=noise[:, None])):
        with pytest.raises(efim.EfimError) as e:
            verify(**fits)
        assert e.value.code == 4                                          # the workspace is too small
    drafts = torch.zeros(2, 3, dtype=whole)
    with pytest.raises(ValueError):
        efim.efim_draft_lookup(torch.zeros(2, 5, 8, dtype=whole), n, 1, 2, drafts, n.clone(), stream=0)
    with pytest.raises(efim.EfimError) as e:                              # (no n-gram of 33)
        efim.efim_draft_lookup(torch.zeros(2, 1, 8, dtype=whole), n, 1, 33, drafts, n.clone(), stream=0)
    assert e.value.code == UNSUPPORTED


def test_numbers_that_do_not_fit(lib):
    """A number past 32 bits is an error, not its lowest bits."""
    torch = pytest.importorskip("torch")
    whole = torch.int32
    history, n, drafts = torch.zeros(2, 8, dtype=whole), torch.zeros(2, dtype=whole), torch.zeros(2, 3, dtype=whole)
    for lo, hi in (((1 << 32) + 1, 2), (1, (1 << 32) + 2), (1, 1 << 31), (-(1 << 31) - 1, 2), (1, 1 << 70)):
        with pytest.raises(OverflowError):
            efim.efim_draft_lookup(history, n, lo, hi, drafts, n.clone(), stream=0)
    with pytest.raises(OverflowError):
        efim.efim_verify_workspace_bytes((1 << 32) + 2, torch.zeros(6, 40000))
    cache = efim.Cache(torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16), 2)
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(OverflowError):
        efim.efim_decode_attn(cache, 1, n, (1 << 32) + 16, drafts, q, q.clone(), stream=0)
    with pytest.raises(efim.EfimError) as e:                              # (the largest that fits; no n-gram of it)
        efim.efim_draft_lookup(history, n, 1, (1 << 31) - 1, drafts, n.clone(), stream=0)
    assert e.value.code == UNSUPPORTED
