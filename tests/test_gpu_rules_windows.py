"""Logit rules where a wave has much to do: windows full of touched tokens, walks
over many windows.  Exactness as in test_gpu_rules.py."""
import numpy as np
import pytest
import torch

from test_gpu_rules import Rules, Run, check, logits
from tail_harness import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_masks", [0, 3])
@pytest.mark.parametrize("V", [2048, 9003])
def test_every_token_is_touched(V, n_masks, dtype):
    """The whole window is exchanged between the lanes: each adjusts tokens that others
    loaded and fold.  One request touches every token, one every third, one a single
    token of each 512."""
    rng = np.random.default_rng(V)
    o = [2 * V, V, V]
    tokens = np.empty((3, 2 * V + 20), dtype=np.int64)
    tokens[0] = np.concatenate([rng.permutation(V), rng.integers(0, V, V + 20)])
    tokens[1] = rng.integers(0, V // 3, 2 * V + 20) * 3
    tokens[2] = rng.integers(0, V // 512, 2 * V + 20) * 512 + 77
    bt = Batch(w=[2, 1, 2], o=o, bl=4, W_max=2, tokens=tokens, V=V, prompt=[V // 2, 10, 0]).cuda()
    rules = Rules(bt, V, seed=V, n_bias=40, n_masks=n_masks)
    z = logits(bt, V, dtype, seed=1)
    check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [157184, 300007, 1 << 19])
def test_walks_over_many_windows(V, dtype):
    """1024 rows, so a row's share is cut in two and a wave walks up to 32 windows (all
    of them at 2^19 float32 logits): lists that begin late, masks that empty windows,
    equal maxima in several windows, touched and not."""
    rng = np.random.default_rng(V)
    B, bl = 128, 8
    live = (0, 63, 127)
    o = np.full(B, 3000)
    tokens = np.zeros((B, 3000 + 3 * bl), dtype=np.int64)
    tokens[0] = rng.integers(0, V, tokens.shape[1])
    tokens[63] = V - 1 - rng.integers(0, 5000, tokens.shape[1])     # the last windows alone
    tokens[127] = rng.integers(0, 40, tokens.shape[1]) * (V // 40)
    bt = Batch(w=[1] * B, o=o, bl=bl, W_max=1, tokens=tokens, V=V, prompt=np.full(B, 1500),
               inactive=[b for b in range(B) if b not in live])
    assert bt.row_cap == 1024
    bt.cuda()
    rules = Rules(bt, V, seed=V, n_bias=60, n_masks=4, keep=(0.9, 0.5, 0.02, 0.9))
    window = 2048
    for m, part in ((1, 0.5), (2, 0.3), (3, 0.98)):      # windows that the mask empties
        for w in np.flatnonzero(rng.random(-(-V // window)) < part):
            rules.allowed[m, w * window:(w + 1) * window] = False
    rules.masks = np.packbits(np.pad(rules.allowed, ((0, 0), (0, -V % 32))), axis=1,
                              bitorder="little").view(np.int32)
    rules.params[127] = [1, 0, 0, 0]                     # touched and left as they are
    z = logits(bt, V, dtype, seed=2)
    for i, row in enumerate(bt.live):
        rules.row_mask[row] = (-1, 0, 1, 2, 3, -1, 1, 3)[i % 8]
        # ties: of tokens in many windows, some of them touched
        at = rng.choice(V, 24, replace=False)
        at[:4] = rng.integers(0, 40, 4) * (V // 40)
        z[int(row), at] = 60.0
    check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())
