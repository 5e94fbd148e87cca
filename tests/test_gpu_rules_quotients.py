"""The repetition penalty's quotient is float32's for every logit: subnormal ones,
subnormal quotients, and quotients at the ends of the range.  Bit for bit."""
import numpy as np
import pytest
import torch

from test_gpu_rules import Rules, Run
from tail_harness import TORCH, Batch

pytestmark = pytest.mark.gpu
R = [2.0 ** -40, 1.3e-12, 3e-5, 0.1, 0.7, np.nextafter(np.float32(1), np.float32(0)), 1.0,
     np.nextafter(np.float32(1), np.float32(2)), 1.1, 1.2, 1.5, 1.9999999, 3.0, 7.7e4, 7.7e11, 2.0 ** 40]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lo,hi", [(-149, -126), (-126, -100), (-100, -70), (-81, -79), (-20, 20), (80, 127)])
def test_every_size(lo, hi, dtype):
    V, B = 4096, len(R)
    tokens = np.tile(np.arange(V + 40), (B, 1)) % V            # every token is seen, none generated
    bt = Batch(w=[1] * B, o=[V] * B, bl=2, W_max=1, tokens=tokens, V=V, prompt=[V] * B).cuda()
    rules = Rules(bt, V, n_bias=None, n_masks=0)
    rules.params[:] = 0
    rules.params[:, 0] = R
    rng = np.random.default_rng(hi + 200)
    z = np.ldexp(rng.uniform(1, 2, (bt.row_cap, V)), rng.integers(lo, hi, (bt.row_cap, V)))
    z[:, 0], z[:, 1] = np.ldexp(1.0, lo), np.ldexp(1.0, hi)
    z *= rng.choice([-1, 1], z.shape, p=[0.2, 0.8])
    z = torch.from_numpy(z).to(torch.float32).to(TORCH[dtype]).cuda()
    run = Run(bt, V, dtype, rules, z).go()
    zf = z.float().cpu().numpy()
    r = np.asarray(R, dtype=np.float32)[bt.row_req][:, None]
    with np.errstate(all="ignore"):
        want = np.where(zf > 0, zf / r, zf * r)
    assert want.dtype == np.float32
    want = torch.from_numpy(want).to(TORCH[dtype]).float()
    assert torch.equal(run.out.float().cpu(), want)
