"""The workspace of the attention over a 4-bit cache without a bound of the lengths."""
import ctypes

import pytest

import paper_2505_21889_b200 as efim
from paper_2505_21889_b200 import binding as B
from paper_2505_21889_b200 import build as efim_build

UNSUPPORTED, WORKSPACE = 2, 4


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (32, 8, 128), (64, 1, 64), (1, 1, 64)])
@pytest.mark.parametrize("batch,new", [(1, 1), (3, 4), (500, 9)])
def test_without_a_bound_it_is_enough_for_every_table(hq, hkv, d, batch, new):
    efim_build.build()
    lib = efim.load_library()
    cache = ctypes.byref(B._Cache4Desc(0x10000, 0x20000, 0x30000, 0x40000, 64, 16, hq, hkv, d, 1.0, 1.0))
    size = lib.efim_kv4_decode_workspace_bytes
    most = size(cache, batch, new, 0)
    assert most == size(cache, batch, new, -5) == size(cache, batch, new, (1 << 31) - 1) > 0
    assert most >= max(size(cache, batch, new, c) for c in (1, 100, 512, 513, 3000, 100000, 1 << 24))
    for width in (40, 3000):                                               # (with a byte too few nothing is launched)
        need = size(cache, batch, new, 16 * width)
        assert lib.efim_kv4_decode_attn(cache, batch, 0x1000, 0, 0x2000, width, 0x3000, batch, new, 0x100000, 0x200000, None, 0.0, 0x800000, need - 1,
                                        None, None) == WORKSPACE


def test_keys_count_in_32_bits():
    """Contexts whose last trip would end behind 2^31 are refused (nothing is launched: there is no workspace)."""
    efim_build.build()
    lib = efim.load_library()
    cache = ctypes.byref(B._Cache4Desc(0x10000, 0x20000, 0x30000, 0x40000, 64, 16, 8, 2, 128, 1.0, 1.0))

    def call(max_ctx, width=1 << 27):
        return lib.efim_kv4_decode_attn(cache, 1, 0x1000, max_ctx, 0x2000, width, 0x3000, 1, 1, 0x100000, 0x200000, None, 0.0, None, 0, None, None)
    assert call((1 << 31) - 1) == call((1 << 31) - 1023) == UNSUPPORTED
    assert call((1 << 31) - 1024) == call(0) == WORKSPACE
