"""Batches for the tests of the model's tail: request states with given windows
and prefixes, their pack, and the live rows by the oracle's pack."""
import numpy as np
import torch

from oracle import pack as opack
from paper_2607_17652_amd import binding as fb


class Batch:
    """Requests with windows w, prefixes o, prompts of `prompt` tokens."""

    def __init__(self, w, o, bl, W_max, layout="ragged", prompt=None, tokens=None, V=1000,
                 seed=0, inactive=()):
        rng = np.random.default_rng(seed)
        w, o = np.asarray(w), np.asarray(o)
        B = len(w)
        L = o // bl // 2
        self.state = dict(gen_start=o - L * bl, prompt_len=o - L * bl if prompt is None
                          else np.asarray(prompt), n_blocks=L + W_max + 1, L=L, R=L + w,
                          active=np.ones(B, dtype=int), eos_hit=np.zeros(B, dtype=int))
        self.state["active"][list(inactive)] = 0
        self.B, self.bl, self.W_max, self.layout, self.o, self.V = B, bl, W_max, layout, o, V
        self.T_max = int(o.max()) + (W_max + 2) * bl
        self.n_max = int(self.state["n_blocks"].max())
        self.tokens = rng.integers(0, V, size=(B, self.T_max)) if tokens is None else tokens
        rec = np.zeros((B, 8), dtype=np.int32)
        for i, k in enumerate(("gen_start", "prompt_len", "n_blocks", "L", "R", "active")):
            rec[:, i] = self.state[k]
        self.st_host = rec
        self.packed = opack.pack_wavefronts(self.state, W_max, bl, layout)
        self.row_cap = B * W_max * bl
        self.row_req = np.full(self.row_cap, -1)
        self.row_req[:len(self.packed["row_req"])] = self.packed["row_req"]
        self.live = np.flatnonzero(self.row_req >= 0)

    def cuda(self):
        self.st = torch.from_numpy(self.st_host).cuda()
        self.tok = torch.from_numpy(self.tokens.astype(np.int32)).cuda()
        buf = torch.zeros(fb.fb_pack_bytes(self.B, self.W_max, self.bl), dtype=torch.uint8,
                          device="cuda")
        self.pack = fb.fb_pack_init(buf, self.B, self.W_max, self.bl, self.layout)
        self.repack()
        return self

    def repack(self, stream=None):
        fb.fb_pack_wavefronts(self.st, self.tok, self.n_max, self.T_max, self.pack, stream)


BATCHES = {
    # one row of one request
    "token": dict(w=[1], o=[0], bl=1, W_max=1),
    "ragged": dict(w=[2, 1, 3, 1], o=[17, 0, 40, 9], bl=5, W_max=3),
    # an inactive request, and dead rows inside the layout
    "padded": dict(w=[1, 3, 2], o=[12, 7, 33], bl=8, W_max=3, layout="padded", inactive=(1,)),
    "window96": dict(w=[3], o=[64], bl=32, W_max=3),
    "nothing": dict(w=[2, 1], o=[8, 8], bl=4, W_max=2, inactive=(0, 1)),
}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # torch.finfo(t).eps / 2


def f64(t):
    return t.double().cpu().numpy()
