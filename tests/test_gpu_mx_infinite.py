"""Attention over a quantised cache that others have filled with scales past those that
the write makes: values past bf16's largest are infinite, for the rows that see their key
and in their channel alone."""
import numpy as np
import pytest
import torch

from cache_harness import Batch, f64, seen
from oracle import cache as oc
from test_gpu_mx_attention import LONG, Attend

pytestmark = pytest.mark.gpu

PLUS, MINUS, LARGE = 5, 6, 9          # channels of the group of 32 that hold something


def group(bits, scale):
    """A group's codes: infinities of both signs (the least and the largest codes that are),
    the code below the least one, a large finite value, and zeros."""
    grid = oc.GRID[bits] * 2.0 ** (scale - 127)
    least = int(np.argmax(grid >= 2.0 ** 128))
    assert 0 < least and grid[least - 1] <= (2 - 2.0 ** -7) * 2.0 ** 127
    codes = np.zeros(32, dtype=np.uint8)
    codes[PLUS], codes[MINUS] = least, len(grid) - 1 + (8 if bits == 4 else 128)
    codes[LARGE] = 1 if bits == 4 else 8
    return codes, oc.values(codes[None], np.array([[scale]], dtype=np.uint8), bits)[0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits,scale", [(4, 253), (4, 254), (8, 247), (8, 250), (8, 254)])
@pytest.mark.parametrize("Hq,d,ps,reach", [(1, 64, 8, 0), (32, 64, 8, 0), (32, 128, 32, 0),
                                           (2, 32, 32, 0), (2, 128, 32, LONG), (32, 64, 32, LONG),
                                           (64, 32, 64, 0)])
@pytest.mark.parametrize("where", [2, 34, 37, 39])
def test_infinite_values_reach_the_rows_that_see_them(where, Hq, d, ps, reach, bits, scale, dtype):
    bt = Batch(w=[3], o=[32], bl=3, W_max=3).cuda()
    a = Attend(bt, Hq, 1, d, ps, bits, dtype, seed=2, size=0.25, reach=reach)
    a.run()
    before = f64(a.out)
    c, g = a.c, d // 32 - 1                       # the head's last group
    codes, values = group(bits, scale)
    page, at = int(c.table[0, where // ps]), where % ps
    c.dev[2][page, 0, at, g * 4 * bits:(g + 1) * 4 * bits] = \
        torch.from_numpy(oc.pack_codes(codes, bits)).cuda()
    c.dev[3][page, 0, at, g] = scale
    a.run()
    got = f64(a.out)
    k, v = (x[:, 0] for x in c.gather(0, 41))
    v[where, g * 32:] = np.where(np.isinf(values) | (np.abs(values) >= 2.0 ** 128), 0, values)
    n_seen, _ = seen(bt)
    q = f64(a.q)
    # weights and their sum 2^-8 each in bf16, the result 2^-8; float32: scores' sums
    near = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -14
    for i, r in enumerate(bt.live):
        if where >= n_seen[i]:
            assert np.array_equal(got[r], before[r]), (i, n_seen[i])
            continue
        hit = g * 32 + np.array([PLUS, MINUS])
        assert not np.isfinite(got[r][:, hit]).any()
        assert not (got[r][:, hit[0]] == -np.inf).any() and not (got[r][:, hit[1]] == np.inf).any()
        assert np.array_equal(got[r][:, :g * 32], before[r][:, :g * 32])
        n = n_seen[i]
        z = q[r] @ k[:n].T * a.scale
        p = np.exp(z - z.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        keep = np.setdiff1d(np.arange(g * 32, d), hit)
        tol = near * (p @ np.abs(v[:n, keep]))
        assert (np.abs(got[r][:, keep] - p @ v[:n, keep]) <= tol).all()


@pytest.mark.parametrize("bits,scale", [(4, 254), (8, 254)])
@pytest.mark.parametrize("Hq", [1, 32])
@pytest.mark.parametrize("where", [34, 39])
def test_infinite_keys_reach_the_rows_that_see_them(where, Hq, bits, scale):
    bt = Batch(w=[3], o=[32], bl=3, W_max=3).cuda()
    a = Attend(bt, Hq, 1, 64, 8, bits, "bf16", seed=3)
    a.run()
    before = f64(a.out)
    codes, _ = group(bits, scale)
    page, at = int(a.c.table[0, where // 8]), where % 8
    a.c.dev[0][page, 0, at, 4 * bits:] = torch.from_numpy(oc.pack_codes(codes, bits)).cuda()
    a.c.dev[1][page, 0, at, 1] = scale
    a.run()
    got = f64(a.out)
    n_seen, _ = seen(bt)
    for i, r in enumerate(bt.live):
        if where >= n_seen[i]:
            assert np.array_equal(got[r], before[r])
