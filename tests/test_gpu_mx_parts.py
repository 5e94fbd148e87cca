"""float32 attention over the quantised cache holds all 24 bits of queries and softmax
weights, which go through the matrix cores in three bf16 parts: inputs whose results are
the lowest parts' alone, with a tolerance that two parts miss (shown on the CPU)."""
import numpy as np
import pytest
import torch

from cache_harness import Batch, Cache, f64, seen, status
from oracle import cache as oc
from test_gpu_mx_attention import LONG, Attend

# Relative to the result, in units of 2^-24.  The weight: log2 e and the exponent rounded
# (both under 5.8 in size) 7, exp2 2.  The denominator: ones, whose sums are exact but
# where the exponent grows (at most 17 times), and eight weights: 26; four waves joined 4.
# Divided units: two pieces' log-sum-exps (up to 16) 33, their exponentials 4, up to 20
# pieces in a row and eight lanes 28.  Quotients and products 12.
TOL = 128 * 2.0 ** -24
FORMS = {
    "few": dict(w=[1, 1, 1], o=[200, 33, 1000], bl=1, W_max=1, Hq=8, Hkv=2, d=64, ps=16),
    "few of 128": dict(w=[2, 1], o=[90, 500], bl=3, W_max=2, Hq=8, Hkv=2, d=128, ps=32),
    "few of 32": dict(w=[1, 1], o=[64, 700], bl=4, W_max=1, Hq=8, Hkv=1, d=32, ps=8),
    "few, divided": dict(w=[1, 1, 1], o=[1200, 333, 900], bl=1, W_max=1, Hq=16, Hkv=2, d=64, ps=16,
                         reach=LONG),
    "few, long": dict(w=[1], o=[70000], bl=1, W_max=1, Hq=16, Hkv=2, d=128, ps=64),
    "wide": dict(w=[2, 1, 3], o=[300, 90, 700], bl=5, W_max=3, Hq=24, Hkv=2, d=128, ps=32),
    "wide, all rows": dict(w=[2, 1], o=[300, 90], bl=16, W_max=2, Hq=16, Hkv=2, d=64, ps=32),
    "wide, small pages": dict(w=[2, 1, 3], o=[300, 90, 700], bl=5, W_max=3, Hq=24, Hkv=2, d=64, ps=8),
    "wide, divided": dict(w=[2, 1], o=[1100, 400], bl=16, W_max=2, Hq=16, Hkv=2, d=32, ps=64, reach=LONG),
    "wide, long": dict(w=[2], o=[20000], bl=16, W_max=2, Hq=16, Hkv=2, d=64, ps=32),
    "wide of 128, long": dict(w=[1], o=[40000], bl=33, W_max=1, Hq=4, Hkv=2, d=128, ps=16),
}


class Case:
    """Zero keys but for at most eight of a request, which score -u and have the value 1
    in a channel each: that channel becomes e^-u / (n - m + m e^-u), m of n keys marked.

    weights  u is a query element, anything up to 4
    queries  u is 2^17 times the difference of two query elements that differ in their
             last eight bits only
    """

    def __init__(self, kind, w, o, bl, W_max, Hq, Hkv, d, ps, bits, reach=0):
        rng = np.random.default_rng(7)
        self.bt = bt = Batch(w=w, o=o, bl=bl, W_max=W_max)
        self.c = c = Cache(bt, Hq, Hkv, d, ps, bits, "f32", reach=reach)
        for i, x in enumerate((0, 127, 0, 127)):
            c.host[i][:] = x
        one, sign = (2, 8) if bits == 4 else (0x38, 0x80)
        self.channels = []
        for b in range(bt.B):
            first = int(bt.o[b]) + bl                 # keys that every row of the request sees
            m = min(8, first // 2)
            self.channels.append(rng.choice(d, m, replace=False))
            for p, ch in zip(rng.choice(first, m, replace=False), self.channels[-1]):
                k, v = np.zeros((2, d), dtype=np.uint8)
                k[0], k[1] = one | sign, one if kind == "queries" else 0
                v[ch] = one
                page = c.table[b, p // ps]
                c.host[0][page, :, p % ps] = oc.pack_codes(k, bits)
                c.host[2][page, :, p % ps] = oc.pack_codes(v, bits)
        self.kind, rows = kind, (bt.row_cap, Hq)
        self.q = np.zeros(rows + (d,), dtype=np.float32)
        if kind == "weights":
            self.scale = 1.0
            self.q[..., 0] = rng.uniform(0.05, 4, size=rows)
        else:
            self.scale = 2.0 ** 17
            base = 1 + rng.integers(0, 1 << 15, size=rows) * 2.0 ** -15
            self.q[..., 0] = base + rng.integers(1, 256, size=rows) * 2.0 ** -23
            self.q[..., 1] = base
        self.n_seen, self.req = seen(bt)

    def weight(self, q):
        """e^-u of the live rows' heads from q."""
        x = q.astype(np.float64)[self.bt.live]
        return np.exp(-self.scale * (x[..., 0] - x[..., 1]))

    def result(self, weight, part):
        """The live rows' result where `part` of the weight reaches the products."""
        out = np.zeros((len(self.bt.live),) + self.q.shape[1:])
        for i, b in enumerate(self.req):
            m = len(self.channels[b])
            den = self.n_seen[i] - m + m * weight[i]
            out[i][:, self.channels[b]] = (part[i] / den)[:, None]
        return out

    def check(self, got):
        w = self.weight(self.q)
        want = self.result(w, w)
        assert (got[want == 0] == 0).all()
        err = np.abs(got - want)
        assert (err <= TOL * want).all(), (err / np.where(want == 0, 1, want)).max() / TOL


def cut(x, bits):
    """float32 x with the last `bits` of its 24 bits dropped."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32)
    return (u & np.uint32(0xffffffff << bits & 0xffffffff)).view(np.float32)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind", ["weights", "queries"])
def test_two_parts_would_be_seen(kind, form):
    """In float64 with all bits the check passes; with 16 bits of the weights, or of the
    queries, it does not."""
    a = Case(kind, bits=4, **FORMS[form])
    w = a.weight(a.q)
    a.check(a.result(w, w))
    a.check(a.result(w, w.astype(np.float32)))
    with pytest.raises(AssertionError):
        a.check(a.result(w, cut(w, 8)))
    if kind == "queries":
        w = a.weight(cut(a.q, 8))
        with pytest.raises(AssertionError):
            a.check(a.result(w, w))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind", ["weights", "queries"])
def test_float32_holds_24_bits(kind, form, bits):
    f = FORMS[form]
    x = Case(kind, bits=bits, **f)
    x.bt.cuda()
    a = Attend(x.bt, f["Hq"], f["Hkv"], f["d"], f["ps"], bits, "f32", scale=x.scale, cache=x.c.cuda())
    a.dq.copy_(torch.from_numpy(x.q))
    a.run()
    assert status(x.bt.pack) == (0, -1)
    x.check(f64(a.out)[x.bt.live])
