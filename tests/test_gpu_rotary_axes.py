"""Rotary positions along several axes against the definition in float64."""
import numpy as np
import pytest
import torch

from cache_harness import EPS, TORCH, Batch, f64
from oracle import cache as oc
from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES, HALF_STEP

pytestmark = pytest.mark.gpu


def inputs(bt, Hq, Hkv, d, dtype, axes, seed=0, far=False):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(bt.row_cap, h, d, generator=g).to(TORCH[dtype]) for h in (Hq, Hkv))
    top = 2 ** 31 - 1 if far else 40000
    p = rng.integers(-top, top, size=(axes, bt.row_cap))
    p[:, ::3] = 0
    if far:
        p[:, 1::5] = -2 ** 31
    return q, k, torch.from_numpy(p.astype(np.int32))


def check(bt, x, out, pos, freq, axis, pairing, dtype):
    """Live rows within the roundings; the others as they were (7)."""
    n = len(freq)
    xr = f64(x)[bt.live]
    want = oc.rotary_axes(xr, pos.numpy()[:, bt.live], freq, axis, pairing)
    got = f64(out)
    # a pair's magnitudes times: the angle rounded to float32 (at most pi 2^-24), sine and
    # cosine (2 units of 2^-24 each), two products and a sum
    mag = np.zeros_like(xr)
    for j in range(n):
        a, b = (j, n + j) if pairing == "halves" else (2 * j, 2 * j + 1)
        mag[..., a] = mag[..., b] = np.abs(xr[..., a]) + np.abs(xr[..., b])
    tol = mag * 12 * EPS + np.abs(want) * HALF_STEP[dtype] * (1 + 2 ** -6)
    tol[mag == 0] = 0.0
    same = np.arange(xr.shape[-1]) >= 2 * n
    assert np.array_equal(got[bt.live][..., same], xr[..., same])
    err = np.abs(got[bt.live] - want)
    assert (err <= tol).all(), (err - tol).max()
    dead = np.setdiff1d(np.arange(bt.row_cap), bt.live)
    assert (got[dead] == 7).all()


# (head_dim, sections, pairing): whole heads, parts of heads, one pair, odd counts
FORMS = [(128, (16, 24, 24), "halves"), (128, (11, 9), "halves"), (128, (64,), "neighbours"),
         (64, (7, 6, 5, 3), "neighbours"), (64, (32,), "halves"), (32, (1,), "halves"),
         (32, (3, 4), "neighbours"), (32, (8, 8), "halves"), (128, (13, 50), "neighbours")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,sections,pairing", FORMS)
@pytest.mark.parametrize("batch", BATCHES)
def test_rows_of_every_batch(batch, d, sections, pairing, dtype):
    bt = Batch(**BATCHES[batch]).cuda()
    Hq, Hkv = 6, 2
    freq, axis = fb.rotary_sections(d, sections)
    q, k, pos = inputs(bt, Hq, Hkv, d, dtype, len(sections), seed=d)
    dq, dk, dp = q.cuda(), k.cuda(), pos.cuda()
    qo, ko = torch.full_like(dq, 7), torch.full_like(dk, 7)
    sh = fb.make_shape(Hq, Hkv, d, dtype, 8, 1, 1)
    fb.fb_rotary_axes(dq, qo, dk, ko, dp, bt.pack, sh, fb.make_rotary(freq, axis, pairing))
    check(bt, q, qo, pos, freq, axis, pairing, dtype)
    check(bt, k, ko, pos, freq, axis, pairing, dtype)
    # in place, and each alone
    ip, only = dq.clone(), torch.full_like(dk, 7)
    fb.fb_rotary_axes(ip, ip, None, None, dp, bt.pack, sh, fb.make_rotary(freq, axis, pairing))
    fb.fb_rotary_axes(None, None, dk, only, dp, bt.pack, sh, fb.make_rotary(freq, axis, pairing))
    live = torch.from_numpy(bt.live).cuda()
    dead = torch.from_numpy(np.setdiff1d(np.arange(bt.row_cap), bt.live)).cuda()
    assert torch.equal(ip[live], qo[live]) and torch.equal(ip[dead], dq[dead])
    assert torch.equal(only, ko)


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_axes_in_any_order_and_far_positions(pairing):
    """Interleaved axes with frequencies of their own, positions over all of int32."""
    bt = Batch(**BATCHES["ragged"]).cuda()
    d, n = 64, 24
    axis = [j % 3 for j in range(n)]
    freq = [100.0 ** (-(j // 3) / 8) for j in range(n)]
    q, k, pos = inputs(bt, 4, 4, d, "f32", 3, seed=3, far=True)
    dq, dk = q.cuda(), k.cuda()
    qo, ko = torch.full_like(dq, 7), torch.full_like(dk, 7)
    sh = fb.make_shape(4, 4, d, "f32", 8, 1, 1)
    fb.fb_rotary_axes(dq, qo, dk, ko, pos.cuda(), bt.pack, sh, fb.make_rotary(freq, axis, pairing))
    # angles up to 2^31 in float64: 2^-22 of an angle's own rounding on both sides
    for x, out in ((q, qo), (k, ko)):
        want = oc.rotary_axes(f64(x)[bt.live], pos.numpy()[:, bt.live], freq, axis, pairing)
        mag = np.abs(f64(x)[bt.live]).max() * 2
        assert np.abs(f64(out)[bt.live] - want).max() <= mag * (2.0 ** -21 + 12 * EPS)


def test_one_axis_is_the_window_prologue_s_rotation():
    """The pack's own positions over all pairs: within a rounding of fb_window_prologue."""
    bt = Batch(w=[2, 1, 3], o=[64, 8, 1000], bl=8, W_max=3).cuda()
    Hq, Hkv, d, ps = 8, 2, 128, 16
    sh = fb.make_shape(Hq, Hkv, d, "bf16", ps, 80, 240)
    tab = torch.arange(240, dtype=torch.int32, device="cuda").view(3, 80)
    q, k, _ = inputs(bt, Hq, Hkv, d, "bf16", 1)
    dq, dk = q.cuda(), k.cuda()
    v = torch.zeros_like(dk)
    kc = torch.zeros(240, Hkv, ps, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(240, Hkv, d, ps, dtype=torch.bfloat16, device="cuda")
    q1, q2, k2 = torch.zeros_like(dq), torch.zeros_like(dq), torch.zeros_like(dk)
    fb.fb_window_prologue(dq, q1, dk, v, kc, vc, tab, bt.pack, sh)
    pos = bt.pack.view()["row_pos"].clone()
    freq, axis = fb.rotary_sections(d, (d // 2,))
    fb.fb_rotary_axes(dq, q2, dk, k2, pos, bt.pack, sh, fb.make_rotary(freq, axis))
    live = torch.from_numpy(bt.live).cuda()
    a, b = q1[live].float(), q2[live].float()
    assert (a - b).abs().max() <= 2 ** -7 * a.abs().max()
    assert (a != b).float().mean() < 1e-3
    p = pos[live].long()
    req = torch.from_numpy(bt.row_req[bt.live]).cuda()
    in_cache = kc[tab[req, p // ps].long(), :, p % ps].float()
    assert (in_cache - k2[live].float()).abs().max() <= 2 ** -7 * in_cache.abs().max()


def test_many_rows():
    """More rows than the grid's workgroups take at once, one row a workgroup's last."""
    bt = Batch(w=[3] * 40, o=[0] * 40, bl=37, W_max=3).cuda()
    freq, axis = fb.rotary_sections(32, (5, 4))
    q, k, pos = inputs(bt, 2, 1, 32, "bf16", 2, seed=9)
    dq, dk = q.cuda(), k.cuda()
    qo, ko = torch.full_like(dq, 7), torch.full_like(dk, 7)
    fb.fb_rotary_axes(dq, qo, dk, ko, pos.cuda(), bt.pack, fb.make_shape(2, 1, 32, "bf16", 8, 1, 1),
                      fb.make_rotary(freq, axis))
    check(bt, q, qo, pos, freq, axis, "halves", "bf16")
    check(bt, k, ko, pos, freq, axis, "halves", "bf16")


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_elements_that_stay_past_31_bits(pairing):
    """One pair of heads of 128, and so many heads that four rows' other elements are more
    than 2^31: all of them are there, and the pairs turned."""
    H, d, rows = 4_300_000, 128, 4
    if pairing == "neighbours":            # a run of four pairs takes six of them along
        H = 4_500_000
    assert rows * H * (d - (8 if pairing == "neighbours" else 2)) > 1 << 31
    bt = Batch(w=[1], o=[5], bl=rows, W_max=1).cuda()
    q = torch.empty(rows, H, d, dtype=torch.int16, device="cuda").random_(0x3000, 0x4100) \
        .view(torch.bfloat16)              # 2^-31 .. 8, and their negatives
    q[..., ::3] *= -1
    out = torch.zeros_like(q)
    pos = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda")
    fb.fb_rotary_axes(q, out, None, None, pos, bt.pack, fb.make_shape(H, 1, d, "bf16", 8, 1, 1),
                      fb.make_rotary([0.5], [0], pairing))
    for r in range(rows):
        assert torch.equal(out[r, :, 2:].view(torch.int16), q[r, :, 2:].view(torch.int16))
        for i in range(0, H, 1 << 20):
            a, b = (q[r, i:i + (1 << 20), j].double() for j in (0, 1))
            c, s = np.cos(0.5 * r), np.sin(0.5 * r)
            mag = (a.abs() + b.abs()) * 12 * EPS
            for got, want in ((out[r, i:i + (1 << 20), 0], a * c - b * s),
                              (out[r, i:i + (1 << 20), 1], b * c + a * s)):
                tol = mag + want.abs() * HALF_STEP["bf16"] * (1 + 2 ** -6)
                assert ((got.double() - want).abs() <= tol).all()


def test_a_last_workgroup_of_fewer_rows():
    """4551 rows, three of them a workgroup's last."""
    bt = Batch(w=[3] * 41, o=[0] * 41, bl=37, W_max=3).cuda()
    assert bt.row_cap % 4 == 3
    for d, sections, pairing in ((32, (5, 4), "halves"), (64, (20,), "neighbours")):
        freq, axis = fb.rotary_sections(d, sections)
        q, k, pos = inputs(bt, 2, 1, d, "bf16", len(sections), seed=9)
        dq, dk = q.cuda(), k.cuda()
        qo, ko = torch.full_like(dq, 7), torch.full_like(dk, 7)
        fb.fb_rotary_axes(dq, qo, dk, ko, pos.cuda(), bt.pack, fb.make_shape(2, 1, d, "bf16", 8, 1, 1),
                          fb.make_rotary(freq, axis, pairing))
        check(bt, q, qo, pos, freq, axis, pairing, "bf16")
        check(bt, k, ko, pos, freq, axis, pairing, "bf16")


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_angles_up_to_2_to_the_53(pairing):
    """Frequencies up to 2^22 at positions over all of int32.  The count of turns may be off
    by one, so that the angle that is left, up to 3 pi, is off by 2^-21 as a float32: 8 units
    of 2^-24; sine and cosine 2 each, two products and a sum."""
    bt = Batch(**BATCHES["ragged"]).cuda()
    d, n = 64, 24
    axis, freq = [j % 3 for j in range(n)], [1.0000001 * 2.0 ** (j - 2) for j in range(n)]
    q, k, pos = inputs(bt, 4, 4, d, "f32", 3, seed=4, far=True)
    dq, dk = q.cuda(), k.cuda()
    qo, ko = torch.full_like(dq, 7), torch.full_like(dk, 7)
    fb.fb_rotary_axes(dq, qo, dk, ko, pos.cuda(), bt.pack, fb.make_shape(4, 4, d, "f32", 8, 1, 1),
                      fb.make_rotary(freq, axis, pairing))
    for x, out in ((q, qo), (k, ko)):
        want = oc.rotary_axes(f64(x)[bt.live], pos.numpy()[:, bt.live], freq, axis, pairing)
        mag = np.abs(f64(x)[bt.live]).max() * 2
        assert np.abs(f64(out)[bt.live] - want).max() <= mag * 20 * EPS
