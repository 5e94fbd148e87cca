"""Limits that kernels of the model's tail rely on, from the host's side.  CPU only."""
import ctypes

import pytest

from paper_2607_17652_amd import binding as fb

BASE = ctypes.c_void_p(0x100000)      # never dereferenced


@pytest.mark.parametrize("rows", [1, 7, 255, 256, 257, 1000, 1024, 2048, 20416, 100000])
def test_a_wave_walks_at_most_32_windows_of_a_row(rows):
    """The logit rules keep a wave's list ranges in 32 lanes: the update's split of a row
    has to be so fine that no wave walks more than 32 windows, float32 (pieces of 8192
    logits) and V = 2^19 among them."""
    h = fb.fb_pack()
    assert fb.lib().fb_pack_init(ctypes.byref(h), BASE, 1 << 40, 1, 1, rows, fb.FB_RAGGED) == fb.FB_OK
    for V in (1, 8192, 16384, 16385, 157184, 262144, 262145, 300007, (1 << 19) - 1, 1 << 19):
        nsplit, rest = divmod(fb.lib().fb_update_workspace_bytes(ctypes.byref(h), V) - 16, rows * 16)
        assert rest == 0 and nsplit >= 1
        assert -(-V // (nsplit * 8192)) <= 32
