"""Logit rules against their definition (every operation rounded to float32).

The written float32 logits and the argmax are exact.  bf16 logits are the same
values rounded once (half a step).  Confidences: as for the plain reduction
(tests/harness.py), relative to float64."""
import numpy as np
import pytest
import torch

from harness import CONF_ATOL, CONF_RTOL
from oracle import tail
from oracle import update as oupdate
from paper_2607_17652_amd import binding as fb
from paper_2607_17652_amd import synth
from tail_harness import BATCHES, TORCH, Batch, f64

pytestmark = pytest.mark.gpu


class Rules:
    def __init__(self, bt, V, seed=0, params=True, n_bias=12, n_masks=3, keep=(0.02, 0.5, 0.95)):
        rng = np.random.default_rng(seed)
        B = bt.B
        self.params = np.stack([rng.uniform(0.6, 1.9, B), rng.uniform(-0.5, 1, B),
                                rng.uniform(-0.2, 0.5, B), np.zeros(B)], 1).astype(np.float32) \
            if params else None
        self.start = self.ids = self.val = None
        if n_bias is not None:
            n = rng.integers(0, n_bias + 1, B)
            self.start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
            self.ids = np.concatenate([np.sort(rng.integers(0, V, k)) for k in n]
                                      + [np.zeros(0, dtype=int)]).astype(np.int32)
            self.val = rng.standard_normal(len(self.ids)).astype(np.float32) * 3
            self.val[rng.random(len(self.val)) < 0.2] = -np.inf
        self.masks = self.row_mask = None
        if n_masks:
            words = -(-V // 32)
            bits = rng.random((n_masks, words * 32)) < np.asarray(keep)[:, None]
            self.allowed = bits[:, :V]
            self.masks = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
            self.row_mask = rng.integers(-1, n_masks, bt.row_cap).astype(np.int32)

    def cuda(self):
        d = [None if a is None else torch.from_numpy(a).cuda() for a in
             (self.params, self.start, self.ids, self.val, self.masks, self.row_mask)]
        return fb.make_rules(*d)

    def rows(self, bt, V, z):
        """z' of the live rows (float64 of the float32 definition)."""
        out = np.empty((len(bt.live), V))
        known = {}
        for i, row in enumerate(bt.live):
            b = bt.row_req[row]
            if b not in known:
                seen, count = tail.history(bt.tokens[b], bt.state["prompt_len"][b], bt.o[b], V)
                if self.params is None:
                    seen[:], count[:] = False, 0
                bias, biased = np.zeros(V, dtype=np.float32), np.zeros(V, dtype=bool)
                if self.start is not None:
                    for j in range(self.start[b], self.start[b + 1]):
                        v = self.ids[j]
                        bias[v] = bias[v] + self.val[j] if biased[v] else self.val[j]
                        biased[v] = True
                known[b] = seen, count, bias, biased
            p = (1, 0, 0) if self.params is None else self.params[b, :3]
            m = None if self.masks is None or self.row_mask[row] < 0 \
                else self.allowed[self.row_mask[row]]
            out[i] = tail.rule_logits(z[i], *known[b], p, m)
        return out


def logits(bt, V, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(bt.row_cap, V, generator=g, device="cuda") * 4
    return z.to(TORCH[dtype])


class Run:
    def __init__(self, bt, V, dtype, rules, z, out=None):
        self.r = rules.cuda()
        self.ws = torch.full((fb.fb_rules_workspace_bytes(bt.pack, V),), 0xa5, dtype=torch.uint8,
                             device="cuda")       # nothing in it is taken as it was
        self.upd = torch.full((fb.fb_update_workspace_bytes(bt.pack, V),), 0xa5,
                              dtype=torch.uint8, device="cuda")
        self.conf = torch.full((bt.row_cap,), 5.0, device="cuda")
        self.argmax = torch.full((bt.row_cap,), -7, dtype=torch.int32, device="cuda")
        self.out = torch.full_like(z, 5.0) if out is None else out
        self.bt, self.z, self.V = bt, z, V

    def go(self, stream=None):
        bt = self.bt
        fb.fb_rules_build(self.r, bt.st, bt.tok, self.V, bt.pack, self.ws, stream)
        fb.fb_vocab_reduce_rules(self.z, bt.pack, self.r, self.ws, self.upd, self.conf, self.argmax,
                                 stream)
        fb.fb_logits_rules(self.z, self.out, bt.pack, self.r, self.ws, stream)
        return self


def check(bt, V, dtype, rules, z, run, rows=slice(None)):
    live = bt.live[rows]
    zl = z.float().cpu().numpy()[bt.live]
    want = rules.rows(bt, V, zl)[rows]
    got = run.out.float().cpu()[live]
    w = torch.from_numpy(want)
    assert torch.equal(got, w.to(TORCH[dtype]).float())    # rounded once, to nearest even
    xhat, p = tail.predict(want)
    conf, argmax = f64(run.conf)[live], run.argmax.cpu().numpy()[live]
    assert np.array_equal(argmax, xhat)
    assert np.all(np.abs(conf - p) <= CONF_RTOL * p + CONF_ATOL)
    assert np.all(conf[xhat < 0] == 0)
    dead = np.setdiff1d(np.arange(bt.row_cap), bt.live)
    assert torch.all(run.conf[dead] == 5) and torch.all(run.argmax[dead] == -7)
    assert torch.all(run.out[dead] == 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 3, 7, 8, 31, 33, 100, 1000, 5003, 20000])
@pytest.mark.parametrize("batch", ["token", "ragged", "padded"])
def test_vocabularies(batch, V, dtype):
    bt = Batch(**BATCHES[batch], V=V).cuda()
    rules = Rules(bt, V, seed=V)
    z = logits(bt, V, dtype, V)
    check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [999, 1024])
@pytest.mark.parametrize("kw", [dict(params=False), dict(n_bias=None), dict(n_masks=0),
                                dict(params=False, n_bias=None), dict(params=False, n_masks=0),
                                dict(n_bias=None, n_masks=0), dict(n_bias=0),
                                dict(params=False, n_bias=None, n_masks=0), dict(n_bias=2500)])
def test_rules_that_are_absent(kw, V, dtype):
    bt = Batch(**BATCHES["ragged"], V=V).cuda()
    rules = Rules(bt, V, seed=1, **kw)
    z = logits(bt, V, dtype)
    check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())


def test_prefixes():
    """Lengths of zero, one and thousands, prompts longer than the prefix, one
    token over and over, ids outside the vocabulary."""
    V, rng = 3000, np.random.default_rng(0)
    o = [0, 1, 4096, 7000, 64, 5000]
    tokens = rng.integers(-5, V + 5, size=(6, 7000 + 20))
    tokens[3, :] = 17
    tokens[5, ::2] = V - 1
    bt = Batch(w=[1, 2, 2, 1, 1, 2], o=o, bl=4, W_max=2, tokens=tokens, V=V,
               prompt=[0, 5, 100, 0, 64, 2500]).cuda()
    rules = Rules(bt, V, seed=3)
    z = logits(bt, V, "f32")
    check(bt, V, "f32", rules, z, Run(bt, V, "f32", rules, z).go())


def test_empty_rows_and_spoiled_masked_places():
    """Masks that leave nothing or one token; masked entries hold NaN and
    infinities; allowed ones -inf and the type's lowest value."""
    V = 4099
    for dtype, lowest in (("bf16", None), ("f32", None), ("f32", -1e9), ("bf16", -2.0 ** 26)):
        bt = Batch(**BATCHES["ragged"], V=V).cuda()
        rules = Rules(bt, V, seed=2, n_masks=4, keep=(0.0, 0.3, 0.3, 0.0))
        rules.allowed[3, 4098] = True
        rules.masks = np.packbits(np.pad(rules.allowed, ((0, 0), (0, -V % 32))), axis=1,
                                  bitorder="little").view(np.int32)
        z = logits(bt, V, dtype)
        low = torch.finfo(TORCH[dtype]).min if lowest is None else lowest
        z[:, ::5] = -float("inf")
        z[:, 1::5] = low
        z[bt.live[-4:], 10:] = low              # nothing but such values past the tenth
        z[bt.live[-4:], :10] = -float("inf")
        rules.row_mask[bt.live[-4:]] = [-1, 1, 2, -1]
        for row in bt.live:
            m = rules.row_mask[row]
            if m >= 0:
                off = torch.from_numpy(np.flatnonzero(~rules.allowed[m])).cuda()
                z[row, off[::3]] = float("nan")
                z[row, off[1::3]] = float("inf")
        rules.val[np.isneginf(rules.val)] = -1.0   # lowest - something stays finite or -inf
        check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())


def test_ties_take_the_lowest_id():
    V = 40000
    bt = Batch(**BATCHES["token"], V=V).cuda()
    for at in ([39999, 7], [16384, 16383, 30000], [5, 6, 7]):
        rules = Rules(bt, V, params=False, n_bias=None, n_masks=1, keep=(1.0,))
        rules.row_mask[:] = 0
        z = torch.zeros(bt.row_cap, V, dtype=torch.bfloat16, device="cuda")
        z[:, at] = 3.0
        z[:, min(at) - 1] = 3.0
        rules.allowed[0, min(at) - 1] = False
        rules.masks = np.packbits(rules.allowed, axis=1, bitorder="little").view(np.int32)
        run = Run(bt, V, "bf16", rules, z).go()
        assert run.argmax[bt.live[0]].item() == min(at)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_of_touched_and_untouched_tokens(dtype):
    """Equal z' of tokens that go through the rules and tokens that do not, in
    every order: the lowest id wins."""
    V, rng = 60000, np.random.default_rng(5)
    for trial in range(12):
        at = np.sort(rng.choice(V, 6, replace=False)) if trial % 2 else \
            rng.integers(0, V - 64) + np.sort(rng.choice(64, 6, replace=False))
        tokens = np.concatenate([rng.permutation(at)[:3], rng.integers(0, V, 37)])[None]
        bt = Batch(w=[1], o=[40], bl=1, W_max=1, tokens=np.pad(tokens, ((0, 0), (0, 20))), V=V).cuda()
        rules = Rules(bt, V, seed=trial, n_bias=None, n_masks=0)
        rules.params[:] = [1, 0, 0, 0]          # touched and left as they are
        z = torch.randn(bt.row_cap, V, device="cuda").to(TORCH[dtype])
        z[:, at] = 9.0
        run = Run(bt, V, dtype, rules, z).go()
        assert run.argmax.item() == at[0]


def test_in_place():
    V = 5003
    bt = Batch(**BATCHES["padded"], V=V).cuda()
    rules = Rules(bt, V, seed=8)
    z = logits(bt, V, "bf16")
    a = Run(bt, V, "bf16", rules, z).go()
    same = z.clone()
    fb.fb_logits_rules(same, same, bt.pack, a.r, a.ws)
    dead = np.setdiff1d(np.arange(bt.row_cap), bt.live)
    assert torch.equal(same[bt.live], a.out[bt.live]) and torch.equal(same[dead], z[dead])


@pytest.mark.parametrize("spoil", ["repetition", "nan", "unsorted", "id", "inf", "start", "mask",
                                   "low_mask"])
def test_bad_rules_are_recorded_and_allow_nothing(spoil):
    V = 1000
    bt = Batch(**BATCHES["ragged"], V=V).cuda()
    rules = Rules(bt, V, seed=6)
    rules.start = np.array([0, 3, 6, 9, 12], dtype=np.int32)
    rules.ids = np.array([1, 5, 9] * 4, dtype=np.int32)
    rules.val = np.ones(12, dtype=np.float32)
    b = 2
    bad = np.isin(bt.row_req[bt.live], [b])
    if spoil == "repetition":
        rules.params[b, 0] = 0
    elif spoil == "nan":
        rules.params[b, 2] = np.nan
    elif spoil == "unsorted":
        rules.ids[7] = 0
    elif spoil == "id":
        rules.ids[8] = V
    elif spoil == "inf":
        rules.val[6] = np.inf
    elif spoil == "start":
        rules.start[3:] = 13                    # past n_bias, for the last request too
        bad = np.isin(bt.row_req[bt.live], [2, 3])
    else:
        row = bt.live[bad][1]
        rules.row_mask[row] = 3 if spoil == "mask" else -2
        bad = bt.live == row
    z = logits(bt, V, "f32")
    run = Run(bt, V, "f32", rules, z).go()
    s = fb.fb_pack_read_status(bt.pack)
    assert (s["code"], s["request"]) == (fb.FB_DERR_RULE, b)
    assert torch.all(run.argmax[bt.live[bad]] == -1) and torch.all(run.conf[bt.live[bad]] == 0)
    assert torch.all(run.out[bt.live[bad]] == -float("inf"))
    assert torch.all(run.argmax[bt.live[~bad]] >= 0)
    bt.repack()
    assert fb.fb_pack_read_status(bt.pack)["code"] == fb.FB_DERR_NONE


def test_largest_vocabulary():
    """V = 2^19, the most the call takes."""
    V = 1 << 19
    bt = Batch(**BATCHES["token"], V=V).cuda()
    rules = Rules(bt, V, seed=1, n_masks=2, keep=(0.5, 0.9))
    rules.row_mask[:] = 1
    z = logits(bt, V, "bf16")
    check(bt, V, "bf16", rules, z, Run(bt, V, "bf16", rules, z).go())


def test_more_touched_tokens_than_fit_the_lds():
    """Many requests (one build workgroup each) over the largest vocabulary, one
    of them with a prefix of many different tokens."""
    V, B, rng = 1 << 19, 130, np.random.default_rng(7)
    o = np.full(B, 20)
    o[5] = 16000
    tokens = rng.integers(0, V, size=(B, 16004))
    bt = Batch(w=[1] * B, o=o, bl=1, W_max=1, tokens=tokens, V=V, prompt=[9000 if b == 5 else 7 for b in range(B)],
               inactive=[b for b in range(B) if b not in (0, 5, 129)]).cuda()
    rules = Rules(bt, V, seed=1, n_bias=40, n_masks=1, keep=(0.9,))
    z = logits(bt, V, "bf16")
    check(bt, V, "bf16", rules, z, Run(bt, V, "bf16", rules, z).go())


def test_full_vocabulary_long_prefix():
    """V = 157184, prefixes of thousands: several partitions a row."""
    V = 157184
    bt = Batch(w=[2, 1], o=[9000, 300], bl=4, W_max=2, V=V, prompt=[100, 300]).cuda()
    for dtype in ("bf16", "f32"):
        rules = Rules(bt, V, seed=5, n_bias=300)
        z = logits(bt, V, dtype)
        check(bt, V, dtype, rules, z, Run(bt, V, dtype, rules, z).go())


@pytest.mark.parametrize("force", [False, True])
def test_update_under_rules_is_the_update_on_adjusted_logits(force):
    """fb_rules_build + fb_vocab_reduce_rules + fb_denoise_apply against the
    oracle's update on z'; a block whose rows have nothing left is not decoded,
    not even by forced progress."""
    V, mask_id = 2000, 1999
    bt = Batch(w=[2, 1, 2], o=[24, 8, 32], bl=4, W_max=2, V=V - 1, seed=3)
    rng = np.random.default_rng(1)
    for b in range(bt.B):
        lo = bt.o[b]
        hit = rng.random(bt.bl * 2) < 0.6
        bt.tokens[b, lo:lo + bt.bl * 2][hit] = mask_id
    bt.tokens[1, 8:12] = mask_id
    bt.V = V
    bt.cuda()
    rules = Rules(bt, V, seed=4, keep=(0.0, 0.5, 0.95))
    rules.row_mask[bt.live[bt.row_req[bt.live] == 1]] = 0       # request 1: nothing left
    z = logits(bt, V, "f32") * 2
    run = Run(bt, V, "f32", rules, z).go()
    prm = dict(tau_mask=0.5, tau_edit=0.4, theta=0.5, mask_id=mask_id, eos_id=-1, S_pe=2, W=2,
               edit_masked=False, force_progress=force, sync_window=False)
    pe = torch.zeros(bt.B, bt.n_max, dtype=torch.uint8, device="cuda")
    fin = torch.zeros_like(pe)
    conf, argmax = torch.zeros(bt.row_cap, device="cuda"), \
        torch.zeros(bt.row_cap, dtype=torch.int32, device="cuda")
    fb.fb_denoise_apply(V, bt.tok, conf, argmax, bt.st, pe, fin, bt.pack, fb.make_params(**prm),
                        None, run.upd)
    assert torch.equal(conf[bt.live], run.conf[bt.live])
    assert torch.equal(argmax[bt.live], run.argmax[bt.live])
    xhat, p = tail.predict(rules.rows(bt, V, z.float().cpu().numpy()[bt.live]))
    assert np.all((np.abs(p - 0.5) > 1e-4) & (np.abs(p - 0.4) > 1e-4))     # decisions are clear
    full_x, full_p = np.zeros(bt.row_cap, dtype=np.int64), np.zeros(bt.row_cap)
    # the oracle never writes a prediction equal to mask_id: so a row with none predicts it
    full_x[bt.live], full_p[bt.live] = np.where(xhat < 0, mask_id, xhat), p
    zeros = np.zeros((bt.B, bt.n_max), dtype=np.int64)
    o = oupdate.denoise_update(full_x, full_p, bt.tokens, bt.state, zeros, zeros, bt.packed, prm)
    assert np.array_equal(bt.tok.cpu().numpy(), o["tokens"])
    assert np.array_equal(pe.cpu().numpy(), o["pe"]) and np.array_equal(fin.cpu().numpy(), o["fin"])
    st = synth.state_from_records(bt.st.cpu().numpy())
    for k in ("L", "R", "active"):
        assert np.array_equal(st[k], o["state"][k])
    assert np.all(bt.tok.cpu().numpy()[1, 8:12] == mask_id)


@pytest.mark.parametrize("r", [2.0 ** -41, 2.0 ** 41, np.inf])
def test_repetition_out_of_range(r):
    bt = Batch(**BATCHES["ragged"], V=300).cuda()
    rules = Rules(bt, 300, seed=3, n_bias=None, n_masks=0)
    rules.params[1, 0] = r
    run = Run(bt, 300, "f32", rules, logits(bt, 300, "f32")).go()
    s = fb.fb_pack_read_status(bt.pack)
    assert (s["code"], s["request"]) == (fb.FB_DERR_RULE, 1)
    assert torch.all(run.argmax[bt.live[bt.row_req[bt.live] == 1]] == -1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [2.0 ** -40, 1.3e-12, 7.7e11, 2.0 ** 40])
def test_written_logits_of_any_size(r, dtype):
    """Quotients and products past the type's range are its infinities."""
    V = 500
    bt = Batch(**BATCHES["ragged"], V=V).cuda()
    rules = Rules(bt, V, seed=3)
    rules.params[:, 0] = r
    rng = np.random.default_rng(0)
    size = 2.0 ** rng.integers(-20, 127, size=(bt.row_cap, V))
    z = torch.from_numpy(rng.uniform(1, 2, size.shape) * size * rng.choice([-1, 1], size.shape)) \
        .to(TORCH[dtype]).cuda()
    run = Run(bt, V, dtype, rules, z).go()
    want = rules.rows(bt, V, z.float().cpu().numpy()[bt.live])
    assert torch.equal(run.out.float().cpu()[bt.live], torch.from_numpy(want).to(TORCH[dtype]).float())
