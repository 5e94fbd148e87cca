"""The quantised cache's calls and the rotary's refuse sizes that their kernels' 32-bit
counts do not hold, and no smaller ones.  CPU only: what is not refused for its size is
refused for a pointer that is checked after it."""
import ctypes

import pytest

from paper_2607_17652_amd import binding as fb
from test_cache_abi import BIG, at, cache, lib, refused, shape  # noqa: F401  (lib: a fixture)


def packed(lib, B, W, bl):
    h = fb.fb_pack()
    assert lib.fb_pack_init(ctypes.byref(h), at(0), BIG, B, W, bl, fb.FB_RAGGED) == fb.FB_OK
    return h


# Runs of eight channels of a block's tokens: bl Hkv d/8.  A thread's last step goes past
# them by at most 65535 workgroups of 256, which has to end below 2^31.
STEP = 65535 * 256


@pytest.mark.parametrize("bl,Hkv,d", [(511, 1 << 20, 32), (2047, 1 << 17, 64), (32, (1 << 24) - 1, 32),
                                      (127, (1 << 22) + 1, 32)])
def test_write_refuses_blocks_whose_runs_pass_32_bits_in_a_step(lib, bl, Hkv, d):
    assert (1 << 31) - STEP < bl * Hkv * (d // 8) < 1 << 31
    for bits in (fb.FB_MX4, fb.FB_MX8):
        refused(lib, "UNSUPPORTED", lib.fb_mx_write_window_kv(
            at(1), at(2, 1), cache(format=bits), at(14), packed(lib, 1, 1, bl),
            shape(Hq=Hkv, Hkv=Hkv, head_dim=d), None))


@pytest.mark.parametrize("bl,Hkv,d", [(508, 1 << 20, 32), (127, 1 << 22, 32), (1, 1 << 20, 128)])
def test_write_takes_blocks_below(lib, bl, Hkv, d):
    assert bl * Hkv * (d // 8) <= (1 << 31) - STEP
    refused(lib, "INVAL", lib.fb_mx_write_window_kv(at(1), at(2, 1), cache(), at(14),
                                                    packed(lib, 1, 1, bl),
                                                    shape(Hq=Hkv, Hkv=Hkv, head_dim=d), None))


@pytest.mark.parametrize("W,bl,g", [(9, 119304647, 2), (1, 119304647, 18), (2, 151, 7110873)])
def test_attention_refuses_windows_whose_last_group_passes_31_bits(lib, W, bl, g):
    """Groups of 128 rows: the last one's end has to be below 2^31."""
    assert (1 << 31) - 128 < W * bl * g < 1 << 31
    h, s = packed(lib, 1, W, bl), shape(Hq=g, Hkv=1, head_dim=32)
    assert lib.fb_mx_attention_workspace_bytes(h, s) == 0
    refused(lib, "UNSUPPORTED", lib.fb_mx_attention(at(1), cache(), at(14), h, s, at(2), at(3), BIG,
                                                    None))


@pytest.mark.parametrize("W,bl,g", [(1, (1 << 24) - 1, 128), (64, 1 << 17, 255), (2, 1 << 23, 127)])
def test_attention_takes_windows_below(lib, W, bl, g):
    assert W * bl * g <= (1 << 31) - 128
    assert lib.fb_mx_attention_workspace_bytes(packed(lib, 1, W, bl),
                                               shape(Hq=g, Hkv=1, head_dim=32)) > 0
