"""The quantised cache's operators run together, as a layer uses them: queries and fresh
keys turned by their positions, keys and values into the cache, the attention over it, a
prefix read back; eager, on a side stream, and captured in graphs."""
import numpy as np
import pytest
import torch

from cache_harness import Batch, Cache, f64
from oracle import cache as oc
from paper_2607_17652_amd import binding as fb
from test_gpu_mx_attention import Attend
from test_gpu_mx_cache import expected, rows
from test_gpu_rotary_axes import check as check_rotary

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, seed, bits, dtype, layout="ragged", bl=4, Hq=8, d=64, window=True):
        w = [2, 1, 3, 2] if window else [1] * 4
        self.bt = bt = Batch(w=w, o=[37, 0, 300, 1500], bl=bl, W_max=3 if window else 1, layout=layout,
                             seed=seed).cuda()
        self.dtype, self.Hq, self.Hkv, self.d = dtype, Hq, 2, d
        self.freq, self.axis = fb.rotary_sections(d, (d // 8, d // 8, d // 4))
        self.rot = fb.make_rotary(self.freq, self.axis)
        self.c = c = Cache(bt, Hq, 2, d, 16, bits, dtype, seed=seed).cuda()
        self.start = [t.clone() for t in c.dev]
        rng = np.random.default_rng(seed)
        self.pos = torch.from_numpy(rng.integers(0, 5000, size=(3, bt.row_cap)).astype(np.int32))
        self.q = rows(bt, Hq, d, dtype, seed=seed)
        self.k, self.v = rows(bt, 2, d, dtype, seed=seed + 1), rows(bt, 2, d, dtype, seed=seed + 2)
        self.dpos, self.dq, self.dk, self.dv = (t.cuda() for t in (self.pos, self.q, self.k, self.v))
        self.a = Attend(bt, Hq, 2, d, 16, bits, dtype, cache=c)
        self.q_out, self.k_out = torch.zeros_like(self.dq), torch.zeros_like(self.dk)
        live = bt.state["active"] > 0
        n = np.where(live, np.minimum(bt.o + 2, 40), 0)
        self.spans = torch.from_numpy(np.stack([bt.o + 2 - n, n], 1).astype(np.int32)).cuda()
        self.back = [torch.zeros(bt.B, 40, 2, d, dtype=self.q.dtype, device="cuda") for _ in "kv"]
        self.n = n

    def step(self):
        c, bt = self.c, self.bt
        for t, s in zip(c.dev, self.start):
            t.copy_(s)
        bt.repack()
        fb.fb_rotary_axes(self.dq, self.q_out, self.dk, self.k_out, self.dpos, bt.pack, c.shape, self.rot)
        fb.fb_mx_write_window_kv(self.k_out, self.dv, c.mx, c.tab, bt.pack, c.shape)
        fb.fb_mx_attention(self.q_out, c.mx, c.tab, bt.pack, c.shape, self.a.out, self.a.ws)
        fb.fb_mx_read_kv(c.mx, c.tab, self.spans, *self.back, bt.pack, c.shape)

    def outputs(self):
        live = torch.from_numpy(self.bt.live).cuda()
        return [self.q_out[live], self.k_out[live], self.a.out[live]] + [
            t.clone() for t in self.c.dev + self.back]

    def spoil(self, x):
        for t in (self.q_out, self.k_out, self.a.out):
            t.fill_(x)


@pytest.mark.parametrize("bits,dtype,layout,bl,Hq,d,window", [
    (4, "bf16", "ragged", 4, 8, 64, True), (8, "bf16", "padded", 33, 8, 128, True),
    (4, "f32", "padded", 5, 2, 32, True), (8, "f32", "ragged", 1, 8, 64, False),
    (4, "bf16", "ragged", 1, 16, 128, False)])
def test_each_part_on_the_one_before(bits, dtype, layout, bl, Hq, d, window):
    s = Layer(1, bits, dtype, layout, bl, Hq, d, window)
    s.spoil(7.0)
    s.step()
    torch.cuda.synchronize()
    bt, c = s.bt, s.c
    check_rotary(bt, s.q, s.q_out, s.pos, s.freq, s.axis, "halves", dtype)
    check_rotary(bt, s.k, s.k_out, s.pos, s.freq, s.axis, "halves", dtype)
    want = expected(c, bt, s.k_out.cpu(), s.v)
    assert all(np.array_equal(g, w) for g, w in zip(c.read_back(), want))
    s.a.q = s.q_out.cpu()
    s.a.check(rows=range(0, len(bt.live), 3), host=want)
    for b in range(bt.B):
        kv = c.gather(b, bt.o[b] + 2, want)
        for o, x in zip(s.back, kv):
            assert np.array_equal(f64(o[b, :s.n[b]]), x[bt.o[b] + 2 - s.n[b]:])


def test_graph_replays_equal_eager_steps():
    """Two layers captured on their own streams, replayed in turn with eager steps and
    synchronisations between them."""
    layers = [Layer(2, 4, "bf16"), Layer(3, 8, "f32", "padded", bl=1, Hq=4, window=False)]
    want, graphs = [], []
    for s in layers:
        s.step()
        torch.cuda.synchronize()
        want.append(s.outputs())
    for s in layers:
        st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            s.step()
            torch.cuda.synchronize()
            with torch.cuda.graph(g, stream=st):
                s.step()
        graphs.append(g)
    for turn in range(3):
        for s, g, w in zip(layers, graphs, want):
            s.spoil(float("nan") if turn % 2 else 0.0)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(s.outputs(), w)), turn
            s.step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(s.outputs(), w)), turn


def test_two_layers_on_streams_of_their_own_at_once():
    layers = [Layer(4, 4, "bf16"), Layer(5, 8, "bf16", bl=1, Hq=4, window=False)]
    want = []
    for s in layers:
        s.step()
        torch.cuda.synchronize()
        want.append(s.outputs())
        s.spoil(0.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(4):
        for s, st in zip(layers, streams):
            with torch.cuda.stream(st):
                s.step()
    torch.cuda.synchronize()
    for s, w in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip(s.outputs(), w))


def test_quantised_attention_beside_the_bf16_one():
    """The same keys and values, representable in 4 bits, in both caches: the two
    attentions agree within their roundings."""
    bt = Batch(w=[2, 3], o=[64, 320], bl=32, W_max=3).cuda()
    Hq, Hkv, d, ps = 8, 2, 128, 32
    g = torch.Generator().manual_seed(0)
    codes = torch.from_numpy(oc.E2M1)[torch.randint(0, 8, (bt.row_cap, Hkv, d), generator=g)]
    x = (codes * torch.sign(torch.randn(codes.shape, generator=g))).bfloat16().cuda()
    c = Cache(bt, Hq, Hkv, d, ps, 4, "bf16").cuda()
    kc = torch.zeros(c.pages, Hkv, ps, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros(c.pages, Hkv, d, ps, dtype=torch.bfloat16, device="cuda")
    for t in c.dev:
        t.zero_()                             # code 0, which reads as zeros
    q = torch.randn(bt.row_cap, Hq, d, generator=g).bfloat16().cuda()
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    fb.fb_write_window_kv(x, x, kc, vc, c.tab, bt.pack, c.shape)
    ws = torch.empty(fb.fb_attention_workspace_bytes(bt.pack, c.shape), dtype=torch.uint8, device="cuda")
    fb.fb_wavefront_attention(q, kc, vc, c.tab, bt.pack, c.shape, a, ws)
    fb.fb_mx_write_window_kv(x, x, c.mx, c.tab, bt.pack, c.shape)
    ws = torch.empty(fb.fb_mx_attention_workspace_bytes(bt.pack, c.shape), dtype=torch.uint8, device="cuda")
    fb.fb_mx_attention(q, c.mx, c.tab, bt.pack, c.shape, b, ws)
    # each within a rounding of its weights (2^-8 of values up to 6) and of its output
    live = torch.from_numpy(bt.live).cuda()
    assert (a[live].float() - b[live].float()).abs().max() <= 2 * 6 * (2.0 ** -8 + 2.0 ** -8)
