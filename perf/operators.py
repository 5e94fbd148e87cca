"""The cases that the operators of the model's tail are measured by: what stands
between a block's output and the denoise update, on the packed live rows.

    norm    fb_residual_norm: the norms after and before a block, its gate and
            its scaled residual
    linear  fb_mx4_linear: a product with 4-bit weights (E2M1 codes, one E8M0
            scale per 32 of K)
    reduce  fb_rules_build + fb_vocab_reduce_rules: penalties, biases and
            grammar masks, and each row's prediction from what they leave
    logits  fb_rules_build + fb_logits_rules: the same, as whole logits

``own`` false: the operators in elementary torch operations; true: the
library's calls.  ``exact`` gives the outputs in float64.
"""
import math

import numpy as np
import torch

own = False

_BASE = dict(bl=32, W=4, w_lo=1, w_hi=4, layout="ragged", lo=128, hi=8192)


def _case(kind, B, **kw):
    return dict(_BASE, kind=kind, B=B, **kw)


def listed():
    return [
        # One token of one request through a norm: latency alone.
        dict(_case("norm", 1, bl=1, W=1, w_hi=1, D=2048, dtype="bf16", gate="none",
                   post=False), name="norm_token"),
        # A serving batch's live rows, gated per request (conditioned blocks).
        dict(_case("norm", 256, D=4096, dtype="bf16", gate="request", post=True),
             name="norm_serve256"),
        # Full precision, an odd width, blocks of 96 in the padded layout, a gate per row.
        dict(_case("norm", 24, bl=96, W=3, w_hi=3, layout="padded", D=2011, dtype="f32",
                   gate="row", post=True), name="norm_odd24"),
        # One token through a projection: one pass over the weights.
        dict(_case("linear", 1, bl=1, W=1, w_hi=1, N=4096, K=4096, out="bf16"),
             name="linear_token"),
        # One request's window through the LM head, logits in bf16.
        dict(_case("linear", 1, W=3, w_lo=3, w_hi=3, N=157184, K=2048, out="bf16"),
             name="linear_head_single"),
        # Odd: a few padded rows, outputs that are no multiple of a tile, K that is no
        # multiple of 128, float32 out.
        dict(_case("linear", 5, bl=5, W=2, w_hi=2, layout="padded", N=5003, K=2080,
                   out="f32"), name="linear_odd"),
        # The live rows of a long-context batch through a wide projection: many rows.
        dict(_case("linear", 8, w_lo=4, N=16384, K=4096, out="bf16"), name="linear_long8"),
        # One token's logits, written whole: penalties of one short chat.
        dict(_case("logits", 1, bl=1, W=1, w_hi=1, lo=1024, hi=1024, V=157184, dtype="bf16",
                   masks=1, bias=16), name="logits_token"),
        # A few requests' window, rules and no update: whole logits for a sampler.
        dict(_case("logits", 8, w_lo=4, lo=16384, hi=32768, V=157184, dtype="bf16", masks=4,
                   bias=64), name="logits_long8"),
        # Odd vocabulary (rows that start anywhere), float32, padded layout.
        dict(_case("reduce", 7, bl=8, W=3, w_hi=3, layout="padded", lo=5, hi=700, V=5003,
                   dtype="f32", masks=3, bias=300), name="reduce_odd"),
        # A few long-context requests, predictions only.
        dict(_case("reduce", 8, w_lo=4, lo=16384, hi=32768, V=157184, dtype="bf16", masks=4,
                   bias=64), name="reduce_long8"),
        # The serving batch.
        dict(_case("reduce", 256, V=157184, dtype="bf16", masks=16, bias=64),
             name="reduce_serve256"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["norm", "linear", "linear", "logits", "reduce", "reduce"])
    bl = rng.choice([1, 4, 8, 16, 32, 32, 64, 96, 128])
    W = rng.randint(1, 5)
    most = {"norm": 20000, "linear": 1024, "logits": 1024, "reduce": 8192}[kind]
    B = max(1, min(256, _log_int(rng, 1, most) // (W * bl)))
    hi = _log_int(rng, 1, 32768)
    c = _case(kind, B, bl=bl, W=W, w_lo=rng.randint(1, W), w_hi=W, lo=rng.randint(1, hi), hi=hi,
              layout=rng.choice(["ragged", "ragged", "padded"]))
    if kind == "norm":
        D = _log_int(rng, 64, 16384)
        if rng.random() < 0.5:
            D = max(64, D // 64 * 64)
        while B * W * bl * D > 20416 * 4096:
            D = D // 2 + 1
        return dict(c, D=D, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    gate=rng.choice(["none", "all", "request", "row"]), post=rng.random() < 0.7)
    if kind == "linear":
        K = 32 * _log_int(rng, 4, 512)
        N = _log_int(rng, 16, 157184)
        while N * K > 157184 * 2048 or B * W * bl * N * K > 1024 * 16384 * 4096:
            N = N // 2 + 1
        return dict(c, N=N, K=K, out=rng.choice(["bf16", "bf16", "f32"]))
    return dict(c, V=_log_int(rng, 1000, 157184), dtype=rng.choice(["bf16", "bf16", "f32"]),
                masks=rng.choice([0, 1, 4, 16]), bias=rng.choice([0, 16, 300]))


# ----------------------------------------------------------------- inputs ---
_T = {"bf16": torch.bfloat16, "f32": torch.float32}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _batch(c, seed):
    """Request states, tokens, and the packed rows that are live, with their requests."""
    rng = np.random.default_rng([seed, 1])
    B, bl, W = c["B"], c["bl"], c["W"]
    w = rng.integers(c["w_lo"], c["w_hi"] + 1, size=B)
    w[0] = c["w_hi"]
    o = np.exp(rng.uniform(math.log(c["lo"]), math.log(c["hi"] + 0.999), size=B)).astype(np.int64)
    o = np.clip(o, c["lo"], c["hi"])
    L = rng.integers(0, o // bl + 1)            # committed blocks; the rest of the prefix is prompt
    st = np.zeros((B, 8), dtype=np.int32)
    st[:, 0] = st[:, 1] = o - L * bl            # gen_start, prompt_len
    st[:, 2] = L + W + 1                        # n_blocks
    st[:, 3], st[:, 4], st[:, 5] = L, L + w, 1  # L, R, active
    T_max = c["hi"] + (W + 2) * bl
    first = np.concatenate([[0], np.cumsum(w)[:-1]]) * bl if c["layout"] == "ragged" \
        else np.arange(B) * W * bl
    rows = np.concatenate([first[b] + np.arange(w[b] * bl) for b in range(B)])
    return dict(st=torch.from_numpy(st).cuda(), o=torch.from_numpy(o).cuda(), T_max=T_max,
                n_max=int(st[:, 2].max()), rows=torch.from_numpy(rows).cuda(),
                req=torch.from_numpy(np.repeat(np.arange(B), w * bl)).cuda(), cap=B * W * bl)


def _pack(c, s):
    """The packed batch's handle, as a decoding program keeps it for the step."""
    from paper_2607_17652_amd import binding as fb
    buf = torch.zeros(fb.fb_pack_bytes(c["B"], c["W"], c["bl"]), dtype=torch.uint8, device="cuda")
    pack = fb.fb_pack_init(buf, c["B"], c["W"], c["bl"], c["layout"])
    fb.fb_pack_wavefronts(s["st"], s.get("tokens"), s["n_max"], s["T_max"], pack)
    return pack


def prepare(case, seed):
    c = case
    s = dict(_batch(c, seed), case=c)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")
    B, cap = c["B"], s["cap"]
    if c["kind"] == "norm":
        D, t = c["D"], _T[c["dtype"]]
        # a residual stream with a few large channels, a block's output, gates around 0.5
        s["h"] = (randn(cap, D) * (1 + 9 * (rand(D) > 0.99))).to(t)
        s["y"] = randn(cap, D).to(t)
        shape = {"none": None, "all": (D,), "request": (B, D), "row": (cap, D)}[c["gate"]]
        s["gate"] = None if shape is None else (0.5 + 0.3 * randn(*shape)).to(t)
        s["w_post"] = (0.3 + 0.1 * randn(D)).to(t) if c["post"] else None
        s["w_pre"] = (1 + 0.2 * randn(D)).to(t)
        s["h_out"], s["n_out"] = torch.zeros_like(s["h"]), torch.zeros_like(s["h"])
    elif c["kind"] == "linear":
        N, K = c["N"], c["K"]
        # normal weights rounded to E2M1 by a power of two per 32
        a = randn(N, K // 32, 32) / math.sqrt(K)
        e = torch.floor(torch.log2(a.abs().amax(-1))) - 2
        a = a * torch.exp2(-e)[..., None]
        edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
        q = (torch.bucketize(a.abs(), edges, out_int32=True) + 8 * (a < 0)).to(torch.uint8)
        q = q.view(N, K // 2, 2)
        s["codes"] = q[..., 0] | (q[..., 1] << 4)          # element 2i in the low half of byte i
        s["scales"] = (e + 127).to(torch.uint8)
        s["x"] = randn(cap, K).to(torch.bfloat16)
        s["y"] = torch.zeros(cap, N, dtype=_T[c["out"]], device="cuda")
    else:
        V, t = c["V"], _T[c["dtype"]]
        # skewed token frequencies, logits of several widths, a peak on two rows of five
        s["tokens"] = (rand(B, s["T_max"]) ** 3 * V).to(torch.int32).clamp_(max=V - 1)
        z = randn(cap, V, dtype=t)
        z *= (1 + 7 * rand(cap, 1)).to(t)
        at = (rand(cap) * V).long().clamp_(max=V - 1)
        peak = torch.where(rand(cap) < 0.4, z.amax(1) + 4, z[torch.arange(cap, device="cuda"), at])
        z[torch.arange(cap, device="cuda"), at] = peak.to(t)
        s["logits"] = z
        s["params"] = torch.stack([1 + 0.5 * rand(B), 0.8 * rand(B), 0.4 * rand(B),
                                   torch.zeros(B, device="cuda")], 1)   # repetition, presence, frequency
        n = c["bias"]
        # ascending, one in every V / n of the vocabulary
        ids = ((torch.arange(n, device="cuda") + rand(B, n)) * (V / n)).to(torch.int32).clamp_(
            max=V - 1) if n else None
        s["bias_id"] = ids.reshape(-1).contiguous() if n else None
        val = (3 * randn(B, n)) if n else None
        if n:
            val[:, ::8] = -math.inf                        # banned outright
        s["bias_val"] = val.reshape(-1).contiguous() if n else None
        s["bias_start"] = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n if n else None
        m = c["masks"]
        if m:
            # a grammar's states: from a hundredth of the vocabulary to nearly all of it
            keep = torch.logspace(-2, -0.02, m, device="cuda")[:, None]
            words = -(-V // 32)
            bits = (rand(m, words * 32) < keep).view(m, words, 32).long()
            if m > 2:
                bits[0] = 0                                # a state that allows nothing
            packed = (bits << torch.arange(32, device="cuda")).sum(-1)
            s["masks"] = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
            s["row_mask"] = torch.where(rand(cap) < 0.5, (rand(cap) * m).long().clamp_(max=m - 1),
                                        -1).to(torch.int32)
        else:
            s["masks"] = s["row_mask"] = None
        if c["kind"] == "logits":
            s["out"] = torch.zeros_like(z)
        s["conf"] = torch.zeros(cap, device="cuda")
        s["argmax"] = torch.zeros(cap, dtype=torch.int32, device="cuda")
    if own:
        from paper_2607_17652_amd import binding as fb
        s["fb"], s["pack"] = fb, _pack(c, s)
        if c["kind"] == "norm":
            s["shape"] = fb.make_norm_shape(c["D"], c["dtype"], c["gate"], eps=1e-6, res_scale=0.7)
        elif c["kind"] != "linear":
            s["rules"] = fb.make_rules(s["params"], s["bias_start"], s["bias_id"], s["bias_val"],
                                       s["masks"], s["row_mask"])
            s["rules_ws"] = torch.empty(fb.fb_rules_workspace_bytes(s["pack"], c["V"]),
                                        dtype=torch.uint8, device="cuda")
            s["upd_ws"] = torch.empty(fb.fb_update_workspace_bytes(s["pack"], c["V"]),
                                      dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------- runs ---
def run(s):
    c = s["case"]
    if own:
        fb = s["fb"]
        if c["kind"] == "norm":
            fb.fb_residual_norm(s["y"], s["h"], s["gate"], s["w_post"], s["w_pre"], s["h_out"],
                                s["n_out"], s["pack"], s["shape"])
            return s["h_out"], s["n_out"]
        if c["kind"] == "linear":
            fb.fb_mx4_linear(s["x"], s["codes"], s["scales"], s["pack"], s["y"])
            return s["y"]
        fb.fb_rules_build(s["rules"], s["st"], s["tokens"], c["V"], s["pack"], s["rules_ws"])
        if c["kind"] == "logits":
            fb.fb_logits_rules(s["logits"], s["out"], s["pack"], s["rules"], s["rules_ws"])
            return s["out"]
        fb.fb_vocab_reduce_rules(s["logits"], s["pack"], s["rules"], s["rules_ws"], s["upd_ws"],
                                 s["conf"], s["argmax"])
        return s["conf"], s["argmax"]
    rows = s["rows"]
    if c["kind"] == "norm":
        u = s["y"][rows].float()
        if s["w_post"] is not None:
            u = u * torch.rsqrt(u.square().mean(1, keepdim=True) + 1e-6) * s["w_post"].float()
        if s["gate"] is not None:
            gate = s["gate"].float()
            u = u * (gate if c["gate"] == "all" else gate[s["req"]] if c["gate"] == "request"
                     else gate[rows])
        h = s["h"][rows].float() + 0.7 * u
        n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * s["w_pre"].float()
        s["h_out"][rows] = h.to(s["h_out"].dtype)
        s["n_out"][rows] = n.to(s["n_out"].dtype)
        return s["h_out"], s["n_out"]
    if c["kind"] == "linear":
        table = torch.tensor(_E2M1, device="cuda")
        q = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(c["N"], c["K"] // 32, 32)
        w = table[q.int()] * torch.exp2(s["scales"].float() - 127)[..., None]
        y = s["x"][rows].float() @ w.view(c["N"], c["K"]).T
        s["y"][rows] = y.to(s["y"].dtype)
        return s["y"]
    z = _adjusted(s)
    if c["kind"] == "logits":
        s["out"][rows] = z.to(s["out"].dtype)
        return s["out"]
    top, at = z.amax(1, keepdim=True), z.argmax(1)          # the lowest index of the maximum
    none = top == -math.inf
    p = 1 / torch.exp(z - torch.where(none, 0, top)).sum(1)
    s["conf"][rows] = torch.where(none[:, 0], 0, p)
    s["argmax"][rows] = torch.where(none[:, 0], -1, at).to(torch.int32)
    return s["conf"], s["argmax"]


def _adjusted(s):
    """The live rows' logits under the rules, in float32."""
    c, rows, req = s["case"], s["rows"], s["req"]
    B, V = c["B"], c["V"]
    pos = torch.arange(s["T_max"], device="cuda")
    prefix = pos < s["o"][:, None]
    made = (prefix & (pos >= s["st"][:, 1:2])).float()
    tok = s["tokens"].long()
    seen = torch.zeros(B, V, device="cuda").scatter_add_(1, tok, prefix.float()) > 0
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, tok, made)
    rep, pres, freq, _ = s["params"][:, :, None].unbind(1)
    add = torch.zeros(B, V, device="cuda")
    if c["bias"]:
        add.scatter_add_(1, s["bias_id"].view(B, -1).long(), s["bias_val"].view(B, -1))
    add = add - torch.where(count > 0, pres, 0)
    add = add - freq * count
    z = s["logits"][rows].float()
    z = torch.where(seen[req], torch.where(z > 0, z / rep[req], z * rep[req]), z)
    z += add[req]
    if c["masks"]:
        v = torch.arange(V, device="cuda")
        allowed = (s["masks"][:, v >> 5] >> (v & 31)) & 1
        every = torch.ones(1, V, dtype=allowed.dtype, device="cuda")
        allowed = torch.cat([every, allowed]) > 0          # row 0: no mask
        z.masked_fill_(~allowed[s["row_mask"][rows].long() + 1], -math.inf)
    return z


def work(case):
    c = case
    # live rows: the middle of the range of windows, the first request's at its largest
    rows = c["bl"] * ((c["B"] - 1) * (c["w_lo"] + c["w_hi"]) / 2 + c["w_hi"])
    if c["kind"] == "norm":
        D, elt = c["D"], 2 if c["dtype"] == "bf16" else 4
        gate = {"none": 0, "all": 1, "request": c["B"], "row": rows}[c["gate"]]
        return {"bytes": elt * D * (4 * rows + gate + 2), "flops": rows * D * 11}
    if c["kind"] == "linear":
        N, K = c["N"], c["K"]
        return {"bytes": N * K / 2 + N * K / 32 + rows * K * 2 + rows * N * (2 if c["out"] == "bf16" else 4),
                "flops": 2 * rows * N * K}
    V, elt = c["V"], 2 if c["dtype"] == "bf16" else 4
    prefix = c["B"] * (c["hi"] - c["lo"]) / max(1e-9, math.log((c["hi"] + 1e-6) / c["lo"]))
    once = rows * V * elt + c["masks"] * V / 8 + 4 * prefix + c["B"] * c["bias"] * 8
    return {"bytes": once + (rows * V * elt if c["kind"] == "logits" else 8 * rows),
            "flops": rows * V * 4}


# --------------------------------------------------------------- in 64 bits ---
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    rows = s["rows"].cpu().numpy()
    req = s["req"].cpu().numpy()
    if c["kind"] == "norm":
        h_out = torch.zeros(s["cap"], c["D"], dtype=torch.float64, device="cuda")
        n_out = torch.zeros_like(h_out)
        for lo in range(0, len(rows), 2048):
            r = s["rows"][lo:lo + 2048]
            y, h = s["y"][r].double(), s["h"][r].double()
            if c["post"]:
                y = y / torch.sqrt((y * y).sum(1) / c["D"] + 1e-6)[:, None] * s["w_post"].double()
            if c["gate"] == "all":
                y = y * s["gate"].double()
            elif c["gate"] == "request":
                y = y * s["gate"].double()[s["req"][lo:lo + 2048]]
            elif c["gate"] == "row":
                y = y * s["gate"][r].double()
            # the residual scale is a float32 number
            h = h + float(np.float32(0.7)) * y
            h_out[r] = h
            n_out[r] = h / torch.sqrt((h * h).sum(1) / c["D"] + 1e-6)[:, None] * s["w_pre"].double()
        return h_out, n_out
    if c["kind"] == "linear":
        N, K = c["N"], c["K"]
        y = torch.zeros(s["cap"], N, dtype=torch.float64, device="cuda")
        x = s["x"][s["rows"]].double()
        for lo in range(0, N, 8192):
            codes = s["codes"][lo:lo + 8192].int()
            w = torch.empty(codes.shape[0], K, dtype=torch.float64, device="cuda")
            for half in range(2):
                q = (codes >> (4 * half)) & 15
                ex, man = (q >> 1) & 3, (q & 1).double()
                mag = torch.where(ex == 0, 0.5 * man, (1 + 0.5 * man) * torch.exp2(ex.double() - 1))
                w[:, half::2] = torch.where(q >= 8, -mag, mag)
            w *= torch.exp2(s["scales"][lo:lo + 8192].double() - 127).repeat_interleave(32, 1)
            y[s["rows"], lo:lo + w.shape[0]] = x @ w.t().contiguous()
        return y
    V = c["V"]
    st, o = s["st"].cpu().numpy(), s["o"].cpu().numpy()
    tok = s["tokens"].cpu().numpy()
    words = s["masks"].cpu().numpy().view(np.uint32) if c["masks"] else None
    of_row = s["row_mask"].cpu().numpy() if c["masks"] else None
    par = s["params"].double().cpu().numpy()
    out = torch.zeros(s["cap"], V, dtype=torch.float64, device="cuda") if c["kind"] == "logits" else None
    conf = torch.zeros(s["cap"], dtype=torch.float64, device="cuda")
    allowed = [torch.from_numpy(np.unpackbits(m.view(np.uint8), bitorder="little")[:V] > 0).cuda()
               for m in words] if c["masks"] else []
    for b in range(c["B"]):
        made = np.bincount(tok[b, st[b, 1]:o[b]], minlength=V)
        seen = np.bincount(tok[b, :o[b]], minlength=V) > 0
        add = -par[b, 2] * made - par[b, 1] * (made > 0)
        if c["bias"]:
            part = slice(b * c["bias"], (b + 1) * c["bias"])
            np.add.at(add, s["bias_id"][part].cpu().numpy(), s["bias_val"][part].double().cpu().numpy())
        seen, add = torch.from_numpy(seen).cuda(), torch.from_numpy(add).cuda()
        mine = rows[req == b]
        z = s["logits"][torch.from_numpy(mine).cuda()].double()
        z = torch.where(seen & (z > 0), z / par[b, 0], torch.where(seen, z * par[b, 0], z)) + add
        if c["masks"]:
            for i in np.flatnonzero(of_row[mine] >= 0):
                z[i].masked_fill_(~allowed[of_row[mine[i]]], -math.inf)
        mine = torch.from_numpy(mine).cuda()
        if out is not None:
            out[mine] = z
        else:
            lse = torch.logsumexp(z, 1)
            conf[mine] = torch.where(lse == -math.inf, 0.0, torch.exp(z.amax(1) - lse))
    return out if out is not None else (conf, None)
