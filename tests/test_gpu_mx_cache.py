"""The quantised cache's write and read: codes and scales bit for bit against the
definition in float64, values exactly what the codes stand for."""
import numpy as np
import pytest
import torch

from cache_harness import TORCH, Batch, Cache, f64, status
from oracle import cache as oc
from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES

pytestmark = pytest.mark.gpu


def rows(bt, Hkv, d, dtype, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(bt.row_cap, Hkv, d, generator=g)
    if kind == "wide":           # groups of every size, some elements far below their group
        x = x * torch.exp2(torch.randint(-120, 120, (bt.row_cap, Hkv, d // 32, 1), generator=g).float()
                           ).expand(-1, -1, -1, 32).reshape(x.shape)
        x[..., ::7] *= 2.0 ** -6
        x[..., ::32] = 0
    elif kind == "grid":         # codes, the middles between them, and their neighbours
        grid = torch.tensor(np.concatenate([oc.E2M1, (oc.E2M1[1:] + oc.E2M1[:-1]) / 2, oc.E4M3,
                                            (oc.E4M3[1:] + oc.E4M3[:-1]) / 2]), dtype=torch.float32)
        x = grid[torch.randint(0, len(grid), x.shape, generator=g)] * torch.sign(x)
        near = torch.randint(0, 3, x.shape, generator=g)
        up = torch.nextafter(x, torch.full_like(x, torch.inf))
        x = torch.where(near == 0, x, torch.where(near == 1, up, torch.nextafter(x, torch.zeros_like(x))))
        x[..., :32] /= 64        # groups of the small grid alone
    return x.to(TORCH[dtype])


def expected(c, bt, k, v):
    """The cache after the window's write, on the host."""
    host = [h.copy() for h in c.host]
    pos = bt.packed["row_pos"]
    for i, x in ((0, k), (2, v)):
        codes, scales = oc.quantise(f64(x), c.bits)
        data = oc.pack_codes(codes, c.bits)
        for r in bt.live:
            p = pos[r]
            page = c.table[bt.row_req[r], p // c.ps]
            host[i][page, :, p % c.ps] = data[r]
            host[i + 1][page, :, p % c.ps] = scales[r]
    return host


def same_codes(got, want, scales, bits):
    """Equal codes wherever the group's scale is not NaN."""
    g, w = oc.unpack_codes(got, bits), oc.unpack_codes(want, bits)
    ok = np.repeat(scales != 255, 32, -1)
    return np.array_equal(g[ok], w[ok])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,d,ps", [("bf16", 128, 32), ("bf16", 64, 8), ("bf16", 32, 16),
                                        ("f32", 128, 4), ("f32", 64, 1), ("f32", 32, 64)])
@pytest.mark.parametrize("batch", BATCHES)
def test_write_then_read(batch, dtype, d, ps, bits):
    bt = Batch(**BATCHES[batch]).cuda()
    Hkv = 3
    c = Cache(bt, 6, Hkv, d, ps, bits, dtype, seed=d + ps).cuda()
    k, v = (rows(bt, Hkv, d, dtype, seed=s) for s in (1, 2))
    fb.fb_mx_write_window_kv(k.cuda(), v.cuda(), c.mx, c.tab, bt.pack, c.shape)
    want = expected(c, bt, k, v)
    got = c.read_back()
    for i in range(4):
        assert np.array_equal(got[i], want[i]), i
    # read back: each request's prefix and window, from positions anywhere
    w = np.where(bt.state["active"] > 0, bt.state["R"] - bt.state["L"], 0)
    T = int((bt.o + w * bt.bl).max()) + 3
    rng = np.random.default_rng(5)
    first = rng.integers(0, bt.o + 1)
    n = bt.o + w * bt.bl - first
    n[0] = min(n[0], 1)
    spans = torch.from_numpy(np.stack([first, n], 1).astype(np.int32)).cuda()
    out = [torch.full((bt.B, T, Hkv, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in "kv"]
    fb.fb_mx_read_kv(c.mx, c.tab, spans, *out, bt.pack, c.shape)
    one = torch.full_like(out[1], 7.0)
    fb.fb_mx_read_kv(c.mx, c.tab, spans, None, one, bt.pack, c.shape)
    assert torch.equal(one, out[1])
    assert status(bt.pack) == (0, -1)
    for b in range(bt.B):
        kv = c.gather(b, first[b] + n[b], want)
        for o, x in zip(out, kv):
            assert np.array_equal(f64(o[b, :n[b]]), x[first[b]:])
            assert (o[b, n[b]:] == 7).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["wide", "grid"])
def test_codes_of_every_size(kind, dtype, bits):
    bt = Batch(w=[3, 2], o=[5, 70], bl=16, W_max=3).cuda()
    c = Cache(bt, 4, 4, 128, 16, bits, dtype).cuda()
    k, v = (rows(bt, 4, 128, dtype, seed=s, kind=kind) for s in (3, 4))
    fb.fb_mx_write_window_kv(k.cuda(), v.cuda(), c.mx, c.tab, bt.pack, c.shape)
    for g, w in zip(c.read_back(), expected(c, bt, k, v)):
        assert np.array_equal(g, w)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ends_of_the_range_and_what_is_not_finite(dtype, bits):
    """The least and largest numbers, zeros of both signs, NaN and infinities: a group
    that is not finite reads as NaN, its neighbours as they are."""
    bt = Batch(w=[1], o=[3], bl=8, W_max=1).cuda()
    c = Cache(bt, 2, 2, 128, 8, bits, dtype).cuda()
    k = rows(bt, 2, 128, dtype, seed=6)
    big, tiny = torch.finfo(k.dtype).max, torch.finfo(k.dtype).smallest_normal
    k[0, 0, :32] = 0.0
    k[0, 0, 32:64] = -0.0
    k[0, 0, 64:96] = big
    k[0, 0, 96:] = -big
    k[0, 1, :32] = tiny
    k[0, 1, 32:64] = tiny / 64
    k[0, 1, 64:96] = tiny / 64 * torch.arange(32)
    k[1, 0, 40] = float("nan")
    k[1, 1, 127] = float("inf")
    k[2, 0, 0] = -float("inf")
    k[3, 0, :64] = float("nan")
    v = k.flip(0).contiguous()
    fb.fb_mx_write_window_kv(k.cuda(), v.cuda(), c.mx, c.tab, bt.pack, c.shape)
    want, got = expected(c, bt, k, v), c.read_back()
    for i in (0, 2):
        assert np.array_equal(got[i + 1], want[i + 1])
        assert same_codes(got[i], want[i], want[i + 1], bits)
    out = torch.zeros(1, 16, 2, 128, dtype=k.dtype, device="cuda")
    spans = torch.tensor([[3, 8]], dtype=torch.int32, device="cuda")
    fb.fb_mx_read_kv(c.mx, c.tab, spans, out, None, bt.pack, c.shape)
    back = f64(out[0, :8])
    bad = ~np.isfinite(f64(k)).reshape(8, 2, 4, 32).all(-1)
    assert np.array_equal(np.isnan(back).reshape(8, 2, 4, 32).all(-1), bad)
    ok = ~np.repeat(bad, 32, -1).reshape(back.shape)
    assert np.array_equal(back[ok], c.gather(0, 11, want)[0][3:][ok])
    assert np.isfinite(back[ok]).all()


def test_same_tokens_same_bytes_wherever_they_stand():
    """Windows of other blocks, layouts and neighbours: the codes go by the group alone."""
    got = []
    for w, bl, layout in (([4], 2, "ragged"), ([1, 2], 8, "padded"), ([1], 8, "ragged")):
        bt = Batch(w=w, o=[9] * len(w), bl=bl, W_max=4, layout=layout).cuda()
        c = Cache(bt, 1, 1, 64, 4, 4, "bf16").cuda()
        k = torch.zeros(bt.row_cap, 1, 64, dtype=torch.bfloat16)
        k[:8] = torch.randn(8, 1, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
        fb.fb_mx_write_window_kv(k.cuda(), k.cuda(), c.mx, c.tab, bt.pack, c.shape)
        spans = torch.tensor([[9, 8]] * bt.B, dtype=torch.int32, device="cuda")
        out = torch.zeros(bt.B, 8, 1, 64, dtype=torch.bfloat16, device="cuda")
        fb.fb_mx_read_kv(c.mx, c.tab, spans, None, out, bt.pack, c.shape)
        got.append(out[0])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_bad_pages_and_spans_are_recorded_and_skipped():
    bt = Batch(w=[1, 2, 1], o=[6, 10, 3], bl=4, W_max=2).cuda()
    c = Cache(bt, 2, 2, 64, 4, 4, "bf16", seed=2)
    c.table[1, 3] = c.pages            # positions 12 .. 15 of request 1
    c.table[2, 1] = -5                 # 4 .. 7 of request 2
    c.cuda()
    k = rows(bt, 2, 64, "bf16", seed=8)
    fb.fb_mx_write_window_kv(k.cuda(), k.cuda(), c.mx, c.tab, bt.pack, c.shape)
    assert status(bt.pack) == (fb.FB_DERR_PAGE, 1)
    got = c.read_back()
    want = [h.copy() for h in c.host]
    for i in (0, 2):
        codes, scales = oc.quantise(f64(k), 4)
        data = oc.pack_codes(codes, 4)
        for r in bt.live:
            b, p = bt.row_req[r], bt.packed["row_pos"][r]
            page = c.table[b, p // 4]
            if 0 <= page < c.pages:
                want[i][page, :, p % 4], want[i + 1][page, :, p % 4] = data[r], scales[r]
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    # spans: one ill-formed each way, beside good ones
    M = c.table.shape[1] * 4
    for bad in ([-1, 3], [0, -1], [0, 17], [M - 2, 3], [2 ** 31 - 1, 5]):
        bt.repack()
        spans = torch.tensor([[2, 5], bad, [0, 3]], dtype=torch.int32, device="cuda")
        out = torch.full((3, 16, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        fb.fb_mx_read_kv(c.mx, c.tab, spans, out, None, bt.pack, c.shape)
        assert status(bt.pack) == (fb.FB_DERR_SPAN, 1), bad
        assert (out[1] == 7).all() and (out[0, 5:] == 7).all() and (out[2, 3:] == 7).all()
        assert np.array_equal(f64(out[0, :5]), c.gather(0, 7, got)[0][2:])
    # a bad page inside a span leaves its positions
    bt.repack()
    spans = torch.tensor([[0, 0], [9, 9], [0, 0]], dtype=torch.int32, device="cuda")
    out = torch.full((3, 16, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    fb.fb_mx_read_kv(c.mx, c.tab, spans, out, None, bt.pack, c.shape)
    assert status(bt.pack) == (fb.FB_DERR_PAGE, 1)
    assert (out[1, 3:7] == 7).all() and (out[0] == 7).all() and not (out[1, :3] == 7).all()
    # a window past the table's last column
    short = fb.make_shape(2, 2, 64, "bf16", 4, 3, c.pages)
    tab = c.tab[:, :3].contiguous()
    bt.repack()
    fb.fb_mx_write_window_kv(k.cuda(), k.cuda(), c.mx, tab, bt.pack, short)
    assert status(bt.pack) == (fb.FB_DERR_PAGE, 1)


def test_offsets_past_32_bits():
    """A cache of 4.3 GB of codes: the last page's slots, written and read."""
    bt = Batch(w=[2], o=[30], bl=16, W_max=2).cuda()
    Hkv, d, ps = 8, 128, 128
    pages = (1 << 32) // (Hkv * ps * 64) + 64
    dev = []
    for n in (64, 4):
        dev.append(torch.zeros(pages, Hkv, ps, n, dtype=torch.uint8, device="cuda"))
    mx = fb.make_mx_cache(fb.FB_MX4, dev[0], dev[1], dev[0], dev[1])    # values over keys
    sh = fb.make_shape(Hkv, Hkv, d, "bf16", ps, 1, pages)
    tab = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    k = rows(bt, Hkv, d, "bf16", seed=4)
    fb.fb_mx_write_window_kv(k.cuda(), k.cuda(), mx, tab, bt.pack, sh)
    codes, scales = oc.quantise(f64(k), 4)
    got = dev[0][pages - 1].cpu().numpy()[:, 30:62]
    assert np.array_equal(got, oc.pack_codes(codes, 4).swapaxes(0, 1))
    assert np.array_equal(dev[1][pages - 1].cpu().numpy()[:, 30:62], scales.swapaxes(0, 1))
    assert int(dev[0][: pages - 1].max()) == 0
    out = torch.zeros(1, 32, Hkv, d, dtype=torch.bfloat16, device="cuda")
    spans = torch.tensor([[30, 32]], dtype=torch.int32, device="cuda")
    fb.fb_mx_read_kv(mx, tab, spans, out, None, bt.pack, sh)
    assert np.array_equal(f64(out[0]), oc.values(codes, scales, 4))
