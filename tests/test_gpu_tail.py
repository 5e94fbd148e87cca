"""The model's tail run together, as a step uses it: residual and norm, the
4-bit LM head, the logit rules beside it on another stream, the reduction and
the update; eager, on a side stream, and captured in a graph."""
import numpy as np
import pytest
import torch

from paper_2607_17652_amd import binding as fb
from tail_harness import Batch, f64
from test_gpu_mx4 import check as check_linear
from test_gpu_norm import check as check_norm, inputs as norm_inputs
from test_gpu_rules import Rules, Run, check as check_rules

pytestmark = pytest.mark.gpu


class Tail:
    def __init__(self, layout, seed, D=320, V=5000):
        self.bt = bt = Batch(w=[2, 1, 3, 2], o=[40, 0, 700, 16], bl=8, W_max=3, V=V, layout=layout,
                             seed=seed).cuda()
        self.D, self.V = D, V
        rng = np.random.default_rng(seed)
        self.t = norm_inputs(bt, D, "bf16", "request", seed=seed)
        self.shape = fb.make_norm_shape(D, "bf16", "request", 1e-6, 0.7)
        self.h_out, self.n_out = (torch.full_like(self.t["h"], 5.0) for _ in range(2))
        self.codes = rng.integers(0, 256, size=(V, D // 2), dtype=np.uint8)
        self.scales = rng.integers(122, 125, size=(V, D // 32), dtype=np.uint8)
        self.dc, self.ds = torch.from_numpy(self.codes).cuda(), torch.from_numpy(self.scales).cuda()
        self.z = torch.full((bt.row_cap, V), 5.0, device="cuda")
        self.rules = Rules(bt, V, seed=seed)
        self.run = Run(bt, V, "f32", self.rules, self.z)
        self.side = torch.cuda.Stream()
        self.prm = fb.make_params(0.4, 0.3, 0.5, V - 1, -1, 2, 3)
        self.st0, self.tok0 = bt.st.clone(), bt.tok.clone()
        self.pe = torch.zeros(bt.B, bt.n_max, dtype=torch.uint8, device="cuda")
        self.fin = torch.zeros_like(self.pe)
        self.torch_done = torch.cuda.Event()

    def step(self, update=True):
        bt, r = self.bt, self.run
        main = torch.cuda.current_stream()
        bt.st.copy_(self.st0)
        bt.tok.copy_(self.tok0)
        self.pe.zero_()
        self.fin.zero_()
        bt.repack()
        self.side.wait_stream(main)
        fb.fb_rules_build(r.r, bt.st, bt.tok, self.V, bt.pack, r.ws, self.side)
        fb.fb_residual_norm(*self.t.values(), self.h_out, self.n_out, bt.pack, self.shape)
        fb.fb_mx4_linear(self.n_out, self.dc, self.ds, bt.pack, self.z)
        main.wait_stream(self.side)
        fb.fb_vocab_reduce_rules(self.z, bt.pack, r.r, r.ws, r.upd, r.conf, r.argmax)
        fb.fb_logits_rules(self.z, r.out, bt.pack, r.r, r.ws)
        if update:
            fb.fb_denoise_apply(self.V, bt.tok, r.conf, r.argmax, bt.st, self.pe, self.fin, bt.pack,
                                self.prm, None, r.upd)

    def outputs(self):
        bt, r = self.bt, self.run
        return [x.clone() for x in (self.h_out, self.n_out, self.z, r.conf, r.argmax, r.out, bt.tok,
                                    bt.st, self.pe, self.fin)]


@pytest.mark.parametrize("layout", ["ragged", "padded"])
def test_each_part_on_the_one_before(layout):
    s = Tail(layout, seed=1)
    s.step(update=False)
    torch.cuda.synchronize()
    check_norm(s.bt, s.D, "bf16", "request", s.t, s.h_out, s.n_out)
    check_linear(s.bt, s.codes, s.scales, s.n_out.cpu(), s.z, "f32")
    check_rules(s.bt, s.V, "f32", s.rules, s.z, s.run)


def test_graph_replays_equal_eager_steps():
    """Two tails captured on their own streams, replayed in turn with eager
    steps and synchronisations between them."""
    tails = [Tail("ragged", seed=2), Tail("padded", seed=3)]
    want, graphs = [], []
    for s in tails:
        s.step()
        torch.cuda.synchronize()
        want.append(s.outputs())
    for s in tails:
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(st):
            s.step()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=st):
                s.step()
        graphs.append(g)
    for turn in range(3):
        for s, g, w in zip(tails, graphs, want):
            s.z.fill_(float("nan") if turn % 2 else 0.0)
            s.h_out.fill_(5.0)
            s.n_out.fill_(5.0)
            live = torch.from_numpy(s.bt.live).cuda()
            g.replay()
            torch.cuda.synchronize()
            got = s.outputs()
            for k, (a, b) in enumerate(zip(got, w)):
                if k < 6:
                    a, b = a[live], b[live]
                assert torch.equal(a, b), (turn, k)
            s.step()
            torch.cuda.synchronize()
            for k, (a, b) in enumerate(zip(s.outputs(), w)):
                if k < 6:
                    a, b = a[live], b[live]
                assert torch.equal(a, b), (turn, k)


def test_on_a_stream_of_its_own():
    s = Tail("ragged", seed=4)
    s.step()
    torch.cuda.synchronize()
    want = s.outputs()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        s.step()
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.outputs(), want))
    assert np.all(np.isfinite(f64(s.run.conf)))
