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
