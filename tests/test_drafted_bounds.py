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
