"""The plain reduction on logits masked with very low finite values, the type's lowest
among them: threads, waves and shares that hold nothing else, and rows of nothing else.
Confidences as in tests/harness.py, relative to the float64 definition."""
import numpy as np
import pytest
import torch

from harness import CONF_ATOL, CONF_RTOL
from oracle import update as oupdate
from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES, TORCH, Batch

pytestmark = pytest.mark.gpu
LOW = {"lowest": None, "-1e30": -1e30, "-3e9": -3e9, "-2^30": -2.0 ** 30, "-1e9": -1e9, "-1e4": -1e4}


def update(bt, z, V):
    ws = torch.full((fb.fb_update_workspace_bytes(bt.pack, V),), 0xa5, dtype=torch.uint8, device="cuda")
    conf = torch.full((bt.row_cap,), 5.0, device="cuda")
    argmax = torch.full((bt.row_cap,), -7, dtype=torch.int32, device="cuda")
    pe = torch.zeros(bt.B, bt.n_max, dtype=torch.uint8, device="cuda")
    prm = fb.make_params(0.9, 0.8, 0.5, V - 1, -1, 2, bt.W_max)
    fb.fb_vocab_reduce(z, bt.pack, ws)
    fb.fb_denoise_apply(V, bt.tok, conf, argmax, bt.st, pe, torch.zeros_like(pe), bt.pack, prm, None, ws)
    return conf.cpu().numpy(), argmax.cpu().numpy()


def check(bt, z, V):
    conf, argmax = update(bt, z, V)
    live = bt.live
    with np.errstate(over="ignore"):
        xhat, p = oupdate.vocab_reduce(z[live].double().cpu().numpy())
    assert np.array_equal(argmax[live], xhat)
    assert np.all(np.abs(conf[live] - p) <= CONF_RTOL * p + CONF_ATOL), (conf[live], p)


@pytest.mark.parametrize("low", LOW)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [7, 1000, 5003, 40000, 157184])
def test_masked_rows(V, dtype, low):
    """A few allowed tokens, scattered or together; a twentieth; all but a few; one."""
    bt = Batch(**BATCHES["ragged"], V=V).cuda()
    rng = np.random.default_rng(V)
    value = torch.finfo(TORCH[dtype]).min if LOW[low] is None else LOW[low]
    z = (torch.randn(bt.row_cap, V, generator=torch.Generator("cuda").manual_seed(V), device="cuda") * 4).to(TORCH[dtype])
    for i, row in enumerate(bt.live):
        keep = rng.random(V) < (0.05, 0.5, 0.99, 0)[i % 4]
        if i % 5 == 0:
            at = rng.integers(0, V)
            keep[:] = False
            keep[at:at + max(1, V // 50)] = True
        keep[rng.integers(0, V)] = True
        z[int(row), torch.from_numpy(~keep).cuda()] = value
    check(bt, z, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 1000, 5003, 40000])
def test_rows_of_nothing_else(V, dtype):
    """Every entry at one low value; two low values; low values among -inf; one maximum
    among low values."""
    bt = Batch(**BATCHES["padded"], V=V).cuda()
    rng = np.random.default_rng(V)
    lowest = torch.finfo(TORCH[dtype]).min
    z = torch.randn(bt.row_cap, V, device="cuda").to(TORCH[dtype])
    values = [v for v in (lowest, -1e30, -3e9, -2.0 ** 31, -2.0 ** 30, -1e9)]
    for i, row in enumerate(bt.live):
        a, b = values[i % 6], values[(i // 6) % 6]
        z[int(row)] = a
        if i % 3 == 1:
            z[int(row), torch.from_numpy(rng.random(V) < 0.3).cuda()] = b
        if i % 3 == 2:
            z[int(row), torch.from_numpy(rng.random(V) < 0.7).cuda()] = -float("inf")
            z[int(row), int(rng.integers(0, V))] = a
    check(bt, z, V)


def test_many_rows_one_share_each():
    """Rows of two shares, one masked throughout."""
    V = 30000
    bt = Batch(w=[4] * 20, o=[64] * 20, bl=32, W_max=4, V=V).cuda()
    z = torch.randn(bt.row_cap, V, device="cuda").bfloat16() * 3
    z[:, 100:] = torch.finfo(torch.bfloat16).min
    z[::2, 20000:20100] = 1.0
    check(bt, z, V)
