"""Attention over the quantised cache where the line of work passes 32 bits: of one KV
head, and by what the page table reaches."""
import numpy as np
import pytest
import torch

from cache_harness import EPS, Batch, Cache, f64, status
from paper_2607_17652_amd import binding as fb
from tail_harness import HALF_STEP
from test_gpu_mx_attention import Attend

pytestmark = pytest.mark.gpu


def test_a_head_whose_line_passes_31_bits():
    """2^23 query heads on one KV head, one token after 2^20 - 1 keys that repeat a page's:
    65536 groups of 32768 tiles and their starts.  Every head's result is there, and those
    looked at are the page's attention."""
    bt = Batch(w=[1], o=[(1 << 20) - 1], bl=1, W_max=1).cuda()
    Hq, d, ps = 1 << 23, 32, 1024
    assert Hq // 128 * ((1 << 20) // 32) >= 1 << 31
    c = Cache(Batch(w=[1], o=[ps - 1], bl=1, W_max=1), Hq, 1, d, ps, 4, "bf16", seed=1)
    c.table = np.full((1, 1 << 10), c.table[0, 0], dtype=np.int32)
    c.cuda()
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(1, Hq, d, generator=g, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7)
    ws = torch.empty(fb.fb_mx_attention_workspace_bytes(bt.pack, c.shape), dtype=torch.uint8,
                     device="cuda")
    fb.fb_mx_attention(q, c.mx, c.tab, bt.pack, c.shape, out, ws)
    assert status(bt.pack) == (0, -1)
    assert not (out == 7).all(-1).any()
    heads = np.unique(np.append(np.random.default_rng(3).integers(0, Hq, 60), [0, 127, 128, Hq - 1]))
    at = torch.from_numpy(heads).cuda()
    q, got = f64(q[0, at]), f64(out[0, at])
    k, v = (x[:, 0] for x in c.gather(0, ps))
    z = q @ k.T / np.sqrt(d)
    p = np.exp(z - z.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    want = p @ v
    # as Attend.check: scores and weights, sums of 2^20 float32 terms, the result's rounding
    top = (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) / np.sqrt(d)
    apart = np.stack([p[i] @ np.abs(v - want[i]) for i in range(len(heads))])
    tol = ((d + 12) * EPS * top + 2.0 ** -21 + 2.0 ** -8) * apart * (1 + 2.0 ** -6) + \
        ((1 << 20) + 64) * EPS * (p @ np.abs(v)) + HALF_STEP["bf16"] * np.abs(want) * (1 + 2.0 ** -6)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("w,bl,W_max,g", [([1] * 20, 1, 1, 4), ([2, 1, 2], 32, 2, 16)])
def test_tables_that_reach_2_to_the_31_keys(w, bl, W_max, g, bits, dtype):
    """Short contexts in one page of 2^20 keys, under a table of 2047 pages: the line of a
    full pack has more than 2^31 places."""
    B, Hkv, d, ps = len(w), 2, 32, 1 << 20
    groups = -(-W_max * bl * g // (32 if W_max * bl * g <= 32 else 128))
    assert B * Hkv * groups * (2047 * ps // 32) >= 1 << 31
    bt = Batch(w=w, o=[(i * 397) % 1900 for i in range(1, B + 1)], bl=bl, W_max=W_max).cuda()
    c = Cache(Batch(w=[1], o=[0], bl=1, W_max=1), g * Hkv, Hkv, d, ps, bits, dtype, seed=bits)
    table = np.full((B, 2047), -1, dtype=np.int32)
    table[:, 0] = c.table[0, 0]
    c.table = table
    a = Attend(bt, g * Hkv, Hkv, d, ps, bits, dtype, seed=4, cache=c.cuda())
    a.run()
    assert status(bt.pack) == (0, -1)
    rng = np.random.default_rng(5)
    a.check(rows=np.unique(np.append(rng.integers(0, len(bt.live), 24), [0, len(bt.live) - 1])))
    again = torch.full_like(a.out, 7)
    a.ws.fill_(0xff)
    a.run(again)
    assert torch.equal(again, a.out)
