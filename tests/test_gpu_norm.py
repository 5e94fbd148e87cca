"""fb_residual_norm against the float64 definition.

Tolerance: the sums of D squares and the few products around them round at
most 80 times in sequence, each by 2^-24 relative to positive partial sums (the
sums) or to the terms |h| + |a g u| (the residual), whose size the norm of h'
passes on; then half a step of the output's type."""
import numpy as np
import pytest
import torch

from oracle import tail
from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES, HALF_STEP, TORCH, Batch, f64

pytestmark = pytest.mark.gpu
A, EPS = 0.7, 1e-6


def inputs(bt, D, dtype, gate, seed=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def make(*shape):      # `shift` elements past the allocation's alignment
        n = int(np.prod(shape))
        return torch.randn(n + shift, generator=g, device="cuda").to(TORCH[dtype])[shift:].view(shape)
    cap = bt.row_cap
    shape = {"none": None, "all": (D,), "request": (bt.B, D), "row": (cap, D)}[gate]
    return dict(y=make(cap, D), h=3 * make(cap, D), gate=None if shape is None else make(*shape),
                w_post=make(D), w_pre=make(D))


def check(bt, D, dtype, gate, t, h_out, n_out):
    live = bt.live
    req = bt.row_req[live]
    v = {k: None if x is None else f64(x) for k, x in t.items()}
    rows = {k: None if v[k] is None else v[k][live] for k in ("y", "h")}
    g = v["gate"]
    g = None if g is None else {"all": lambda: g, "request": lambda: g[req],
                                "row": lambda: g[live]}[gate]()
    # the library holds eps and the residual scale as float32
    a, eps = float(np.float32(A)), float(np.float32(EPS))
    h, n = tail.residual_norm(rows["y"], rows["h"], g, v["w_post"], v["w_pre"], eps, a)
    size = np.abs(rows["h"]) + np.abs(h - rows["h"])
    r = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    w = 1 if v["w_pre"] is None else np.abs(v["w_pre"])
    u = 80 * 2.0 ** -24
    half = HALF_STEP[dtype]
    if h_out is not None:
        assert np.all(np.abs(f64(h_out)[live] - h) <= u * size + half * np.abs(h))
    if n_out is not None:
        assert np.all(np.abs(f64(n_out)[live] - n) <= 2 * u * size * r * w + half * np.abs(n))
    dead = np.setdiff1d(np.arange(bt.row_cap), live)
    for out in (h_out, n_out):
        if out is not None:
            assert np.all(f64(out)[dead] == 5)


def outputs(t):
    return torch.full_like(t["h"], 5.0), torch.full_like(t["h"], 5.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 7, 64, 65, 509, 512, 1000, 2048, 2056, 4096, 5001, 8192, 16384])
@pytest.mark.parametrize("batch,gate", [("ragged", "request"), ("padded", "row")])
def test_widths(batch, gate, D, dtype):
    bt = Batch(**BATCHES[batch]).cuda()
    t = inputs(bt, D, dtype, gate, seed=D)
    h_out, n_out = outputs(t)
    fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack, fb.make_norm_shape(D, dtype, gate, EPS, A))
    check(bt, D, dtype, gate, t, h_out, n_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,shift", [(256, 0), (777, 0), (1024, 1)])
@pytest.mark.parametrize("absent", [(), ("w_post",), ("w_pre",), ("w_post", "w_pre"), ("n_out", "w_pre"),
                                    ("y", "gate", "w_post", "h_out")])
@pytest.mark.parametrize("gate", ["none", "all", "request", "row"])
@pytest.mark.parametrize("batch", ["token", "ragged", "nothing"])
def test_forms(batch, gate, absent, D, shift, dtype):
    """Every gate and every array that may be absent, from one row on; pointers
    that are not 16-byte aligned."""
    if "gate" in absent:
        gate = "none"
    bt = Batch(**BATCHES[batch]).cuda()
    t = inputs(bt, D, dtype, gate, seed=3, shift=shift)
    h_out, n_out = outputs(t)
    for k in absent:
        if k in t:
            t[k] = None
    h_out = None if "h_out" in absent else h_out
    n_out = None if "n_out" in absent else n_out
    fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack, fb.make_norm_shape(D, dtype, gate, EPS, A))
    check(bt, D, dtype, gate, t, h_out, n_out)


@pytest.mark.parametrize("D", [100, 1024, 6000])
def test_in_place(D):
    """h_out over h and n_out over y give the same bits."""
    bt = Batch(**BATCHES["ragged"]).cuda()
    t = inputs(bt, D, "bf16", "all", seed=1)
    sh = fb.make_norm_shape(D, "bf16", "all", EPS, A)
    h_out, n_out = outputs(t)
    fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack, sh)
    live = torch.from_numpy(bt.live).cuda()
    fb.fb_residual_norm(*t.values(), t["h"], t["y"], bt.pack, sh)
    assert torch.equal(t["h"][live], h_out[live]) and torch.equal(t["y"][live], n_out[live])


def test_rows_that_are_zero_huge_or_not_finite_stay_their_own():
    bt = Batch(**BATCHES["ragged"]).cuda()
    D = 1024
    t = inputs(bt, D, "f32", "none", seed=2)
    t["y"][0] = t["h"][0] = 0
    t["y"][1] = t["h"][1] = 1e18        # squares reach 1e36, their sum 1e39 would not fit a float
    t["h"][2, 5] = float("nan")
    t["y"][3, 7] = float("inf")
    h_out, n_out = outputs(t)
    fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack, fb.make_norm_shape(D, "f32", "none", EPS, A))
    assert torch.all(h_out[0] == 0) and torch.all(n_out[0] == 0)
    assert torch.isnan(n_out[2]).all() and torch.isnan(h_out[2]).sum() == 1
    assert torch.isnan(n_out[3]).any()
    for k in t:
        if t[k] is not None and t[k].dim() == 2:
            t[k][1:4] = 0
    rest = torch.cat([h_out[4:], n_out[4:]])
    assert torch.isfinite(rest).all()


def test_large_pack():
    """More rows than workgroups at once, wide enough for the pipelined form."""
    bt = Batch(w=[4, 2, 3, 4] * 16, o=[64] * 64, bl=32, W_max=4).cuda()
    for D in (1024, 4096):
        t = inputs(bt, D, "bf16", "request", seed=D)
        h_out, n_out = outputs(t)
        fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack,
                            fb.make_norm_shape(D, "bf16", "request", EPS, A))
        check(bt, D, "bf16", "request", t, h_out, n_out)


def test_offsets_past_32_bits():
    """140800 rows of 16384: rows around element 2^31 and the last ones."""
    D = 16384
    bt = Batch(w=[4] * 1100, o=[32] * 1100, bl=32, W_max=4).cuda()
    g = torch.Generator(device="cuda").manual_seed(0)
    y, h = (torch.randn(bt.row_cap, D, generator=g, device="cuda", dtype=torch.bfloat16)
            for _ in range(2))
    w = torch.randn(D, generator=g, device="cuda").to(torch.bfloat16)
    rows = np.r_[0, 2 ** 31 // D - 2:2 ** 31 // D + 2, bt.row_cap - 2:bt.row_cap]
    assert np.isin(rows, bt.live).all()
    h0 = f64(h[rows])
    fb.fb_residual_norm(y, h, None, None, w, h, y, bt.pack,
                        fb.make_norm_shape(D, "bf16", "none", EPS, 0.0))
    assert np.array_equal(f64(h[rows]), h0)     # a = 0
    n = h0 / np.sqrt((h0 * h0).mean(1, keepdims=True) + float(np.float32(EPS))) * f64(w)
    tol = (160 * 2.0 ** -24 + HALF_STEP["bf16"]) * np.abs(n)
    assert np.all(np.abs(f64(y[rows]) - n) <= tol)
