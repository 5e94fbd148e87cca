"""Attention over the quantised cache against softmax attention in float64 on the values
that the codes stand for."""
import numpy as np
import pytest
import torch

from cache_harness import EPS, TORCH, Batch, Cache, f64, seen, status
from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES, HALF_STEP

pytestmark = pytest.mark.gpu


class Attend:
    def __init__(self, bt, Hq, Hkv, d, ps, bits, dtype, seed=0, scale=0.0, size=1.0, cache=None,
                 reach=0):
        self.bt = bt
        self.c = c = cache or Cache(bt, Hq, Hkv, d, ps, bits, dtype, seed=seed, reach=reach)
        if cache is None:
            c.cuda()
        c.shape.sm_scale = scale
        self.scale = scale if scale > 0 else 1 / np.sqrt(d)
        g = torch.Generator().manual_seed(seed + 1)
        self.q = (size * torch.randn(bt.row_cap, Hq, d, generator=g)).to(TORCH[dtype])
        self.dq = self.q.cuda()
        self.out = torch.full_like(self.dq, 7)
        self.ws = torch.empty(fb.fb_mx_attention_workspace_bytes(bt.pack, c.shape),
                              dtype=torch.uint8, device="cuda")

    def run(self, out=None, stream=None):
        fb.fb_mx_attention(self.dq, self.c.mx, self.c.tab, self.bt.pack, self.c.shape,
                           self.out if out is None else out, self.ws, stream)

    def check(self, out=None, rows=None, host=None):
        """Of the rows given (all), and that dead rows are as they were."""
        bt, c = self.bt, self.c
        got = f64(self.out if out is None else out)
        n_seen, req = seen(bt)
        q, g = f64(self.q), c.Hq // c.Hkv
        held = {b: c.gather(b, int(n_seen[req == b].max()), host) for b in np.unique(req)}
        for i in range(len(bt.live)) if rows is None else rows:
            n, r = n_seen[i], bt.live[i]
            k, v = (x[:n] for x in held[req[i]])
            qr = q[r].reshape(c.Hkv, g, c.d)
            z = np.einsum("jhd,hgd->hgj", k, qr) * self.scale
            p = np.exp(z - z.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            want = np.einsum("hgj,jhd->hgd", p, v)
            # the score's float32 sum (d/16 steps of 16 products), scale and exponent; bf16
            # weights are rounded, and off from the others' share only as far as values differ
            top = self.scale * np.einsum("jhd,hgd->hgj", np.abs(k), np.abs(qr)).max(-1)
            weight = (c.d + 12) * EPS * top[..., None] + 2.0 ** -21
            if c.dtype == "bf16":
                weight = weight + 2.0 ** -8
            apart = np.stack([np.einsum("gj,gjd->gd", p[h], np.abs(v[None, :, h] - want[h][:, None]))
                              for h in range(c.Hkv)])
            size = np.einsum("hgj,jhd->hgd", p, np.abs(v))
            tol = weight * apart * (1 + 2.0 ** -6) + (n + 64) * EPS * size + \
                HALF_STEP[c.dtype] * np.abs(want) * (1 + 2.0 ** -6) + 1e-30
            err = np.abs(got[r].reshape(want.shape) - want)
            assert (err <= tol).all(), (i, int(n), (err / tol).max())
        dead = np.setdiff1d(np.arange(bt.row_cap), bt.live)
        assert (got[dead] == 7).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,ps", [(128, 32), (64, 8), (32, 4), (128, 1), (64, 128)])
@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (3, 1), (16, 1)])
def test_batches(batch, Hq, Hkv, d, ps, dtype, bits):
    bt = Batch(**BATCHES[batch]).cuda()
    a = Attend(bt, Hq, Hkv, d, ps, bits, dtype, seed=d + ps)
    a.run()
    a.check()
    assert status(bt.pack) == (0, -1)


LONG = 5000      # a page table of so many keys: contexts are divided, however short they are


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,ps", [(128, 32), (64, 8), (32, 64)])
@pytest.mark.parametrize("Hq", [2, 24])
def test_short_contexts_under_long_tables(Hq, d, ps, dtype, bits):
    bt = Batch(w=[2, 1, 3], o=[700, 31, 1100], bl=5, W_max=3).cuda()
    a = Attend(bt, Hq, 2, d, ps, bits, dtype, seed=d, reach=LONG)
    a.run()
    a.check()
    again = torch.full_like(a.out, 7)
    a.ws.fill_(0xff)
    a.run(again)
    assert torch.equal(again, a.out)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 63, 64, 95, 127, 128, 129, 255, 257, 1000, 4093])
def test_one_token_after_prefixes_of_every_length(n, dtype, bits):
    bt = Batch(w=[1], o=[n], bl=1, W_max=1).cuda()
    for reach in (0, LONG):
        a = Attend(bt, 8, 2, 64, 16, bits, dtype, seed=n, reach=reach)
        a.run()
        a.check()


@pytest.mark.parametrize("dtype,d,ps,bits", [("bf16", 64, 16, 4), ("f32", 64, 16, 4), ("bf16", 128, 32, 8),
                                             ("f32", 128, 64, 8)])
@pytest.mark.parametrize("w,bl,g", [(1, 32, 1), (1, 33, 1), (4, 8, 1), (1, 1, 32), (1, 1, 33), (4, 32, 4),
                                    (3, 43, 1), (2, 64, 1), (2, 65, 1), (5, 13, 3), (6, 1, 5)])
def test_groups_of_rows(w, bl, g, dtype, d, ps, bits):
    """Rows on both sides of a wave's 32 and a workgroup's 128, blocks that end inside
    groups, and windows whose blocks see different tiles."""
    bt = Batch(w=[w, max(1, w - 1)], o=[45, 300], bl=bl, W_max=w).cuda()
    a = Attend(bt, 2 * g, 2, d, ps, bits, dtype, seed=bl)
    a.run()
    rng = np.random.default_rng(w)
    a.check(rows=np.unique(np.append(rng.integers(0, len(bt.live), 40), [0, len(bt.live) - 1])))


@pytest.mark.parametrize("batch", [dict(w=[1] * 70, o=list(range(0, 2100, 30)), bl=1, W_max=1),
                                   dict(w=[2, 1, 3] * 30, o=list(range(7, 4507, 50)), bl=32, W_max=3),
                                   dict(w=[1] * 300, o=[(i * 37) % 90 for i in range(300)], bl=1, W_max=1,
                                        inactive=tuple(range(5, 300, 7))),
                                   dict(w=[1] * 300, o=[(i * 53) % 400 for i in range(300)], bl=1, W_max=1,
                                        inactive=tuple(i for i in range(300) if i not in (3, 4, 150, 299))),
                                   dict(w=[2] * 200, o=[(i * 53) % 400 for i in range(200)], bl=20, W_max=2,
                                        layout="padded", inactive=tuple(i for i in range(200) if i % 66)),
                                   dict(w=[1, 2], o=[20000, 11], bl=16, W_max=2, layout="padded"),
                                   dict(w=[1], o=[70000], bl=1, W_max=1)])
@pytest.mark.parametrize("d,ps,bits", [(64, 16, 4), (128, 32, 8), (32, 64, 4)])
def test_shares_that_cut_units_anywhere(batch, d, ps, bits):
    """Few and many units, long beside short ones, more requests than threads."""
    bt = Batch(**batch).cuda()
    a = Attend(bt, 8, 2, d, ps, bits, "bf16", seed=3, reach=LONG)
    a.run()
    rng = np.random.default_rng(1)
    a.check(rows=np.unique(rng.integers(0, len(bt.live), 24)))
    again = torch.full_like(a.out, 7)
    a.ws.fill_(0xff)
    a.run(again)
    assert torch.equal(again, a.out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,size", [(1.0, 4.0), (0.01, 1.0), (30.0, 1.0)])
def test_sharp_and_flat_softmaxes(scale, size, dtype):
    """Weights that all go to a key or two, late ones among them, and even weights."""
    bt = Batch(w=[2, 1], o=[400, 31], bl=16, W_max=2).cuda()
    a = Attend(bt, 4, 2, 128, 16, 8, dtype, scale=scale, size=size)
    a.run()
    a.check(rows=range(0, len(bt.live), 5))


def test_rising_scores():
    """Every tile's scores pass the ones before, so the running maximum moves each time."""
    bt = Batch(w=[1], o=[640], bl=1, W_max=1).cuda()
    c = Cache(bt, 4, 1, 64, 32, 4, "f32")
    c.host[0][:] = 0x22                       # every element 1
    for i, page in enumerate(c.table[0, :21]):
        c.host[1][page] = 100 + i             # 2^-27 .. 2^-7
    a = Attend(bt, 4, 1, 64, 32, 4, "f32", scale=2.0 ** 8, cache=c.cuda())
    a.q.fill_(1.0)
    a.dq.fill_(1.0)
    a.run()
    a.check()


def test_out_may_be_q_and_streams_of_its_own():
    bt = Batch(w=[2, 1, 3], o=[170, 0, 900], bl=5, W_max=3).cuda()
    for Hq in (2, 16):                        # both forms
        a = Attend(bt, Hq, 2, 64, 16, 8, "bf16", seed=Hq)
        a.run()
        torch.cuda.synchronize()
        st, q = torch.cuda.Stream(), a.dq.clone()
        with torch.cuda.stream(st):
            fb.fb_mx_attention(q, a.c.mx, a.c.tab, bt.pack, a.c.shape, q, a.ws)
        st.synchronize()
        live = torch.from_numpy(bt.live).cuda()
        assert torch.equal(q[live], a.out[live])
        other = torch.full_like(a.out, 7)
        st.wait_stream(torch.cuda.current_stream())
        a.run(other, st)
        st.synchronize()
        assert torch.equal(other, a.out)


@pytest.mark.parametrize("Hq", [2, 32])
def test_what_lies_past_the_keys_is_not_read_for_a_result(Hq):
    """NaN scales and any codes in the slots past a request's window, and in pages that
    are not its own."""
    bt = Batch(w=[2, 1], o=[37, 5], bl=3, W_max=2).cuda()
    a = Attend(bt, Hq, 1, 64, 16, 8, "bf16", seed=1)
    a.run()
    want = a.out.clone()
    mine = np.zeros((a.c.pages, 16), dtype=bool)
    n_seen, req = seen(bt)
    for b in range(2):
        for p in range(int(n_seen[req == b].max())):
            mine[a.c.table[b, p // 16], p % 16] = True
    hole = torch.from_numpy(~mine).cuda()
    for t, x in zip(a.c.dev, (0x7f, 255, 0xff, 255)):
        t[hole[:, None, :].expand(t.shape[:3])] = x
    a.run()
    assert torch.equal(a.out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [1, 32])
@pytest.mark.parametrize("which", [1, 3])
@pytest.mark.parametrize("where", [2, 34, 37, 39])
def test_nan_scales_spoil_the_rows_that_see_them(where, which, Hq, dtype):
    """A NaN key spoils a row, a NaN value 32 channels of it; rows of earlier blocks do
    not see the window's later keys."""
    bt = Batch(w=[3], o=[32], bl=3, W_max=3).cuda()
    a = Attend(bt, Hq, 1, 64, 8, 4, dtype, seed=2)
    a.run()
    want = f64(a.out)
    a.c.dev[which][int(a.c.table[0, where // 8]), 0, where % 8, 1] = 255
    a.run()
    got = f64(a.out)
    n_seen, _ = seen(bt)
    for i, r in enumerate(bt.live):
        sees = where < n_seen[i]
        spoilt = np.zeros_like(want[r], dtype=bool)
        spoilt[:, 0 if which == 1 else 32:] = sees
        assert np.array_equal(np.isnan(got[r]), spoilt), (i, n_seen[i])
        assert np.array_equal(got[r][~spoilt], want[r][~spoilt])


@pytest.mark.parametrize("Hq", [2, 32])
def test_rows_that_are_not_finite_stay_apart(Hq):
    bt = Batch(w=[2], o=[70], bl=4, W_max=2).cuda()
    a = Attend(bt, Hq, 2, 64, 16, 4, "f32", seed=5)
    a.run()
    want = f64(a.out)
    a.dq[1, 0, 3], a.dq[2, 1, 5] = float("nan"), float("inf")
    a.run()
    got = f64(a.out)
    assert np.isnan(got[1, 0]).all() and np.isnan(got[2, 1]).any()
    keep = np.ones(want.shape[:2], dtype=bool)
    keep[1, 0] = keep[2, 1] = False
    assert np.array_equal(got[keep], want[keep])


@pytest.mark.parametrize("Hq", [2, 32])
def test_bad_pages_are_recorded(Hq):
    bt = Batch(w=[1, 2], o=[40, 20], bl=4, W_max=2).cuda()
    c = Cache(bt, Hq, 1, 64, 8, 4, "bf16", seed=4)
    a = Attend(bt, Hq, 1, 64, 8, 4, "bf16", cache=c.cuda())
    a.run()
    want = a.out.clone()
    c.tab[1, 1] = c.pages
    a.run()
    assert status(bt.pack) == (fb.FB_DERR_PAGE, 1)
    assert torch.equal(a.out[:4], want[:4])
    # a window that the page table does not reach: skipped
    bt.repack()
    c.tab[1, 1] = int(c.table[1, 1])
    short = fb.make_shape(Hq, 1, 64, "bf16", 8, 3, c.pages)
    a.out.fill_(7)
    fb.fb_mx_attention(a.dq, c.mx, c.tab[:, :3].contiguous(), bt.pack, short, a.out, a.ws)
    assert status(bt.pack) == (fb.FB_DERR_PAGE, 0) and (a.out == 7).all()


def test_offsets_past_32_bits():
    """Pages whose codes lie past 4 GiB."""
    bt = Batch(w=[1], o=[300], bl=4, W_max=1).cuda()
    Hkv, d, ps = 4, 128, 128
    pages = (1 << 32) // (Hkv * ps * 64) + 8
    ids = [pages - 1, pages - 5, pages - 3]
    codes = torch.zeros(pages, Hkv, ps, 64, dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, Hkv, ps, 4), 255, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(0)
    small = [rng.integers(0, 256, size=(3, Hkv, ps, 64), dtype=np.uint8),
             rng.integers(124, 127, size=(3, Hkv, ps, 4)).astype(np.uint8)]
    codes[ids], scales[ids] = torch.from_numpy(small[0]).cuda(), torch.from_numpy(small[1]).cuda()
    for Hq in (4, 64):
        c = Cache(bt, Hq, Hkv, d, ps, 4, "bf16")
        c.host, c.table, c.pages = small * 2, np.array([[0, 1, 2]]), pages
        c.mx = fb.make_mx_cache(4, codes, scales, codes, scales)
        c.tab = torch.tensor([ids], dtype=torch.int32, device="cuda")
        c.shape = fb.make_shape(Hq, Hkv, d, "bf16", ps, 3, pages)
        a = Attend(bt, Hq, Hkv, d, ps, 4, "bf16", cache=c)
        a.run()
        a.check()


def test_captured_graphs_that_share_a_workspace():
    """Two graphs on one workspace, replayed in turn with eager calls between."""
    runs, graphs, want = [], [], []
    for w, bl, Hq in (([2, 1], 16, 16), ([1, 1], 1, 4)):
        bt = Batch(w=w, o=[500, 77], bl=bl, W_max=2).cuda()
        runs.append(Attend(bt, Hq, 2, 128, 32, 4, "bf16", seed=bl))
    ws = max((a.ws for a in runs), key=lambda t: t.numel())
    for a in runs:
        a.ws = ws
        a.run()
        torch.cuda.synchronize()
        want.append(a.out.clone())
        st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=st):
            a.run()
        graphs.append(g)
    for turn in range(3):
        for a, g, x in zip(runs, graphs, want):
            a.out.fill_(7)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out, x)
            a.out.fill_(7)
            a.run()
            torch.cuda.synchronize()
            assert torch.equal(a.out, x)
