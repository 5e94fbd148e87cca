"""fb_residual_norm on rows whose squares, or whose sum of squares, lie past the
float range while the row and its norm do not.  Tolerances as in test_gpu_norm.py:
the powers of two that bring such a row into range round nothing."""
import numpy as np
import pytest
import torch

from paper_2607_17652_amd import binding as fb
from tail_harness import BATCHES, Batch
from test_gpu_norm import A, EPS, check, inputs, outputs

pytestmark = pytest.mark.gpu
# the sizes of a row's entries: sums of squares that fit, that do not, squares that do not
SIZES = [1e-12, 1.0, 1e15, 3e16, 1e18, 1e19, 4e19, 1e24, 1e30, 1e36]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("w_post", [True, False])
@pytest.mark.parametrize("D", [37, 1024, 5001, 16384])
@pytest.mark.parametrize("batch,gate", [("ragged", "request"), ("many", "row")])
def test_rows_of_any_size(batch, gate, D, w_post, dtype):
    """The block's output and the residual stream, each large by itself and both."""
    bt = Batch(w=[3, 1, 2] * 10 + [3], o=[14] * 31, bl=7, W_max=3) if batch == "many" else \
        Batch(**BATCHES[batch])
    bt.cuda()
    t = inputs(bt, D, dtype, gate, seed=D)
    rng = np.random.default_rng(D)
    for k in ("y", "h"):
        size = torch.from_numpy(rng.choice(SIZES, (bt.row_cap, 1))).cuda()
        t[k] = (t[k].double() * size).to(t[k].dtype)
    if not w_post:
        t["w_post"] = None
    h_out, n_out = outputs(t)
    fb.fb_residual_norm(*t.values(), h_out, n_out, bt.pack, fb.make_norm_shape(D, dtype, gate, EPS, A))
    check(bt, D, dtype, gate, t, h_out, n_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 64, 1024, 16384])
def test_plain_norm_of_the_largest_rows(D, dtype):
    """Entries up to the type's largest value, all of them, one among small ones, and
    rows of 1e18, whose squares fit a float and whose sum does not."""
    bt = Batch(**BATCHES["ragged"]).cuda()
    t = inputs(bt, D, dtype, "none", seed=D)
    big = torch.finfo(t["h"].dtype).max
    t["h"][0] = big
    t["h"][1] = torch.sign(t["h"][1]) * big
    t["h"][2] = 1e18
    t["h"][3] = -1e18
    t["h"][4] = 1e14
    t["h"][4, D // 2] = 1e25
    for k in ("y", "w_post", "w_pre"):
        t[k] = None
    n_out = torch.full_like(t["h"], 5.0)
    fb.fb_residual_norm(None, t["h"], None, None, None, None, n_out, bt.pack,
                        fb.make_norm_shape(D, dtype, "none", EPS, A))
    check(bt, D, dtype, "none", t, None, n_out)


@pytest.mark.parametrize("cap", ["few", "many"])
def test_infinities_and_nan_stay_what_they_are(cap):
    bt = Batch(w=[1], o=[0], bl=8 if cap == "few" else 600, W_max=1).cuda()
    D = 1024
    t = inputs(bt, D, "f32", "none", seed=2)
    t["h"][1, 5] = float("inf")
    t["h"][2, 7] = float("nan")
    t["h"][3] = 1e30
    t["h"][3, 9] = float("inf")
    n_out = torch.full_like(t["h"], 5.0)
    fb.fb_residual_norm(None, t["h"], None, None, None, None, n_out, bt.pack,
                        fb.make_norm_shape(D, "f32", "none", EPS, A))
    for row, at in ((1, 5), (3, 9)):
        assert torch.isnan(n_out[row, at]) and torch.isnan(n_out[row]).sum() == 1
        assert torch.all(n_out[row, :at] == 0) and torch.all(n_out[row, at + 1:] == 0)
    assert torch.isnan(n_out[2]).all()
    assert torch.isfinite(n_out[0]).all() and torch.isfinite(n_out[4:]).all()
