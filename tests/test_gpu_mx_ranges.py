"""The quantised cache's attention over the formats' whole range of codes and scales, and
the write's bytes wherever tokens stand."""
import numpy as np
import pytest
import torch

from cache_harness import Batch, Cache, status
from paper_2607_17652_amd import binding as fb
from test_gpu_mx_attention import LONG, Attend

pytestmark = pytest.mark.gpu


def ranged(bt, Hq, d, ps, bits, dtype, k_scales, v_scales, reach):
    """Every code but E4M3's NaN, scales of the given ranges."""
    rng = np.random.default_rng(d + bits)
    c = Cache(bt, Hq, 2, d, ps, bits, dtype, seed=ps, reach=reach)
    for i, (lo, hi) in ((0, k_scales), (2, v_scales)):
        codes = rng.integers(0, 256, size=c.host[i].shape, dtype=np.uint8)
        if bits == 8:
            codes = np.where(codes & 127 == 127, codes - 1, codes).astype(np.uint8)
        c.host[i] = codes
        c.host[i + 1] = rng.integers(lo, hi + 1, size=c.host[i + 1].shape, dtype=np.uint8)
    return c.cuda()


# Keys at both ends of the scales that the write makes, queries of 2^-+100 and a score scale
# that brings their products back to a few units; values of 2^90 and 2^-60 (a row's sums of
# weights up to 2^8 times them stay in float32's range).
KEYS = {4: {"high": ((249, 252), 2.0 ** -100, 2.0 ** -27), "low": ((2, 5), 2.0 ** 100, 2.0 ** 21)},
        8: {"high": ((243, 246), 2.0 ** -100, 2.0 ** -29), "low": ((10, 13), 2.0 ** 100, 2.0 ** 6)}}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("keys", ["high", "low"])
@pytest.mark.parametrize("v_scales", [(214, 217), (64, 67)])
@pytest.mark.parametrize("Hq,d,ps,reach", [(4, 128, 32, 0), (4, 64, 8, LONG), (24, 128, 32, LONG),
                                           (24, 64, 64, 0), (24, 32, 4, 0), (4, 32, 32, 0)])
def test_codes_and_scales_of_the_whole_range(Hq, d, ps, reach, v_scales, keys, bits, dtype):
    bt = Batch(w=[2, 1, 3], o=[170, 31, 400], bl=5, W_max=3).cuda()
    k_scales, size, scale = KEYS[bits][keys]
    a = Attend(bt, Hq, 2, d, ps, bits, dtype, seed=d, scale=scale, size=size,
               cache=ranged(bt, Hq, d, ps, bits, dtype, k_scales, v_scales, reach))
    a.run()
    assert status(bt.pack) == (0, -1)
    a.check(rows=range(0, len(bt.live), 3))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("bl,Hq", [(32, 8), (64, 16), (128, 2)])
def test_units_whose_waves_all_have_rows(bl, Hq, d, bits):
    """bl times a KV head's query heads a multiple of 128, pages that hold a tile."""
    bt = Batch(w=[2, 1], o=[300, 77], bl=bl, W_max=2).cuda()
    for reach in (0, LONG):
        a = Attend(bt, Hq, 2, d, 32, bits, "bf16", seed=bl, reach=reach)
        a.run()
        rng = np.random.default_rng(d)
        a.check(rows=np.unique(np.append(rng.integers(0, len(bt.live), 30), [0, len(bt.live) - 1])))


@pytest.mark.parametrize("batch", [dict(w=[1, 1], o=[70000, 20000], bl=1, W_max=1),
                                   dict(w=[1, 2], o=[20000, 11], bl=16, W_max=2, layout="padded"),
                                   dict(w=[2, 1, 3] * 30, o=list(range(7, 4507, 50)), bl=32, W_max=3)])
@pytest.mark.parametrize("d,ps,bits", [(64, 16, 4), (128, 32, 8), (32, 64, 4)])
def test_shares_that_cut_units_anywhere_in_float32(batch, d, ps, bits):
    bt = Batch(**batch).cuda()
    a = Attend(bt, 8, 2, d, ps, bits, "f32", seed=3, reach=LONG)
    a.run()
    rng = np.random.default_rng(1)
    a.check(rows=np.unique(rng.integers(0, len(bt.live), 24)))
    again = torch.full_like(a.out, 7)
    a.ws.fill_(0xff)
    a.run(again)
    assert torch.equal(again, a.out)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_tokens_same_codes_and_scales_wherever_they_stand(dtype, bits):
    """Keys and values of other blocks, layouts, pages and neighbours: bytes, not values."""
    g = torch.Generator().manual_seed(1)
    new = [torch.randn(8, 2, 64, generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
           for _ in "kv"]
    new[0][3, 0, 5], new[0][3, 0, 6], new[1][7, 1, :32] = 0.0, -0.0, -0.0
    got = []
    for w, bl, layout, ps in (([4], 2, "ragged", 4), ([1, 2], 8, "padded", 16), ([1], 8, "ragged", 1)):
        bt = Batch(w=w, o=[9] * len(w), bl=bl, W_max=4, layout=layout).cuda()
        c = Cache(bt, 2, 2, 64, ps, bits, dtype, seed=bl).cuda()
        kv = []
        for x in new:
            t = torch.randn(bt.row_cap, 2, 64, generator=g).to(x.dtype)
            t[:8] = x
            kv.append(t.cuda())
        fb.fb_mx_write_window_kv(*kv, c.mx, c.tab, bt.pack, c.shape)
        pos = np.arange(9, 17)
        got.append([h[c.table[0, pos // ps], :, pos % ps] for h in c.read_back()])
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert np.array_equal(x, y)
