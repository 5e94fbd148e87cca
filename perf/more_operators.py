"""The cases that the operators around a quantised KV cache are measured by:
positions with several axes on the way in, keys and values held in 4 or 8 bits,
and the attention that reads them.

    rotate  fb_rotary_axes: queries and fresh keys turned by their positions
            along several axes (time, height, width)
    store   fb_mx_write_window_kv + fb_mx_read_kv: the window's keys and values
            quantised into the paged cache, and read back from it
    read    fb_mx_read_kv: the committed prefixes as dense keys and values
    attend  fb_mx_attention: block-causal attention over the quantised cache

A group of 32 channels of one key or value has the scale 2^e, e the least for
which no element of the group passes the largest code (6 in E2M1, 448 in E4M3);
elements go to the nearest code, ties to the even one.

``own`` false: the operators in elementary torch operations; true: the
library's calls.  ``exact`` gives the outputs in float64.
"""
import math

import numpy as np
import torch

own = False

_BASE = dict(bl=32, W=4, w_lo=1, w_hi=4, layout="ragged", lo=128, hi=8192, Hq=32, Hkv=8, d=128,
             ps=32, dtype="bf16", bits=4)


def _case(kind, B, **kw):
    return dict(_BASE, kind=kind, B=B, **kw)


def listed():
    return [
        # One token of one request: latency alone.
        dict(_case("rotate", 1, bl=1, W=1, w_hi=1, lo=1024, hi=1024, sec="16 24 24",
                   pairing="halves"), name="rotate_token"),
        # Two axes over part of a head, neighbouring pairs, float32, blocks of 96, padded layout.
        dict(_case("rotate", 24, bl=96, W=3, w_hi=3, layout="padded", Hq=6, Hkv=2, d=64,
                   dtype="f32", sec="11 9", pairing="neighbours"), name="rotate_odd24"),
        # A serving batch's live rows, positions in time, height and width.
        dict(_case("rotate", 256, sec="16 24 24", pairing="halves"), name="rotate_serve256"),
        # One token's keys and values into the cache, and back.
        dict(_case("store", 1, bl=1, W=1, w_hi=1, lo=1024, hi=1024), name="store_token"),
        # Odd: blocks of 5 that start anywhere, pages of 8, float32, 8-bit codes, padded layout.
        dict(_case("store", 7, bl=5, W=3, w_hi=3, layout="padded", lo=5, hi=700, Hq=4, Hkv=2, d=64,
                   ps=8, dtype="f32", bits=8), name="store_odd"),
        # A serving batch's window, as every step writes it.
        dict(_case("store", 256), name="store_serve256"),
        # Long committed prefixes read back whole, for a layer that wants them dense.
        dict(_case("read", 8, w_lo=4, lo=16384, hi=32768), name="read_long8"),
        # One token over a short chat: latency.
        dict(_case("attend", 1, bl=1, W=1, w_hi=1, lo=1024, hi=1024), name="attend_token"),
        # Odd: float32, 8-bit codes, blocks of 5 over pages of 16, prefixes that end anywhere.
        dict(_case("attend", 7, bl=5, W=3, w_hi=3, layout="padded", lo=5, hi=700, Hq=6, Hkv=2, d=64,
                   ps=16, dtype="f32", bits=8), name="attend_odd"),
        # Single tokens of a batch over long contexts: one pass over the cache.
        dict(_case("attend", 64, bl=1, W=1, w_hi=1, lo=1024, hi=32768), name="attend_decode64"),
        # Whole windows of a few long-context requests, 8-bit codes.
        dict(_case("attend", 8, w_lo=4, lo=16384, hi=32768, bits=8), name="attend_long8"),
        # Whole windows of the serving batch: matrix products.
        dict(_case("attend", 256), name="attend_serve256"),
    ]


def _sections(c):
    """Pairs of each axis."""
    return [int(n) for n in c["sec"].split()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["rotate", "store", "read", "attend", "attend", "attend"])
    d = rng.choice([32, 64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
    bl = rng.choice([1, 1, 4, 5, 8, 16, 32, 32, 64, 96, 128])
    W = rng.randint(1, 4) if bl > 1 else 1
    B = max(1, min(256, _log_int(rng, 1, {"rotate": 24576, "store": 24576, "read": 64,
                                          "attend": 24576}[kind]) // (W * bl)))
    hi = _log_int(rng, 1, 32768)
    lo = rng.randint(1, hi) if kind != "read" else max(1, hi // 2)
    # no more cache than the largest listed batches hold, no more products
    while hi > 64 and (B * (hi + W * bl) * Hkv * d > 64 * 9000 * 8 * 128 or
                       B * W * bl * Hq * d * (hi + W * bl) > 256 * 64 * 32 * 128 * 2048):
        hi, lo = max(64, hi // 2), max(1, lo // 2)
    c = _case(kind, B, bl=bl, W=W, w_lo=rng.randint(1, W), w_hi=W, lo=min(lo, hi), hi=hi, d=d,
              Hq=Hq, Hkv=Hkv, ps=rng.choice([8, 16, 32, 32, 64, 128]),
              dtype=rng.choice(["bf16", "bf16", "f32"]), bits=rng.choice([4, 4, 8]),
              layout=rng.choice(["ragged", "ragged", "padded"]))
    if kind == "rotate":
        n, axes = rng.randint(4, d // 2), rng.randint(1, 4)
        cut = sorted(rng.randint(1, n - 1) for _ in range(axes - 1))
        c.update(sec=" ".join(str(b - a) for a, b in zip([0] + cut, cut + [n])),
                 pairing=rng.choice(["halves", "neighbours"]))
    return c


# ----------------------------------------------------------------- inputs ---
_T = {"bf16": torch.bfloat16, "f32": torch.float32}
_LARGEST = {4: 6.0, 8: 448.0}
_E_RANGE = {4: (-125, 125), 8: (-117, 119)}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _pow2(e):
    """2^e in float32, exactly, for -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x, bits):
    """Codes (uint8, two to a byte in 4 bits, the even element low) and scales of the
    last dimension's groups of 32."""
    g = x.float().unflatten(-1, (-1, 32))
    f, k = torch.frexp(g.abs().amax(-1))                   # amax = f 2^k, f in [1/2, 1)
    if bits == 4:
        e = k - 3 + (f > 0.75)
    else:
        e = k - 9 + (f > 0.875)
    e = e.to(torch.int32).clamp_(*_E_RANGE[bits])
    y = (g * _pow2(-e)[..., None]).clamp_(-_LARGEST[bits], _LARGEST[bits]).flatten(-2)
    if bits == 8:
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        n = (torch.round(a / step) * step * 2).to(torch.int64)    # 0 1 2 3 4 6 8 12
        table = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], device=x.device)
        q = (table[n] + 8 * (y < 0)).to(torch.uint8)
        codes = q[..., 0::2] | (q[..., 1::2] << 4)
    return codes, (e + 127).to(torch.uint8)


def _values(codes, scales, bits):
    """What codes and scales stand for, in float32."""
    if bits == 8:
        y = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
        y = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return (y.unflatten(-1, (-1, 32)) * _pow2(scales.int() - 127)[..., None]).flatten(-2)


def _batch(c, seed):
    """Request states, the packed rows that are live with their requests and positions,
    and a page table of shuffled pages."""
    rng = np.random.default_rng([seed, 1])
    B, bl, W, ps = c["B"], c["bl"], c["W"], c["ps"]
    w = rng.integers(c["w_lo"], c["w_hi"] + 1, size=B)
    w[0] = c["w_hi"]
    o = np.exp(rng.uniform(math.log(c["lo"]), math.log(c["hi"] + 0.999), size=B)).astype(np.int64)
    o = np.clip(o, c["lo"], c["hi"])
    L = rng.integers(0, o // bl + 1)            # committed blocks; the rest of the prefix is prompt
    st = np.zeros((B, 8), dtype=np.int32)
    st[:, 0] = st[:, 1] = o - L * bl            # gen_start, prompt_len
    st[:, 2] = L + W + 1                        # n_blocks
    st[:, 3], st[:, 4], st[:, 5] = L, L + w, 1  # L, R, active
    first = np.concatenate([[0], np.cumsum(w)[:-1]]) * bl if c["layout"] == "ragged" \
        else np.arange(B) * W * bl
    rows = np.concatenate([first[b] + np.arange(w[b] * bl) for b in range(B)])
    pos = np.concatenate([o[b] + np.arange(w[b] * bl) for b in range(B)])
    need = -(-(o + w * bl) // ps)
    table = np.full((B, int(need.max())), -1, dtype=np.int32)
    ids = rng.permutation(int(need.sum())).astype(np.int32)
    for b, at in enumerate(np.cumsum(need) - need):
        table[b, :need[b]] = ids[at:at + need[b]]
    return dict(st=torch.from_numpy(st).cuda(), T_max=int(o.max()) + (W + 2) * bl,
                n_max=int(st[:, 2].max()), rows=torch.from_numpy(rows).cuda(),
                req=torch.from_numpy(np.repeat(np.arange(B), w * bl)).cuda(),
                pos=torch.from_numpy(pos).cuda(), table=torch.from_numpy(table).cuda(),
                pages=int(need.sum()), o=o.tolist(), w=w.tolist(), first=first.tolist(),
                cap=B * W * bl)


def prepare(case, seed):
    c = case
    s = dict(_batch(c, seed), case=c)
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, cap, Hq, Hkv, d, t = c["B"], s["cap"], c["Hq"], c["Hkv"], c["d"], _T[c["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    if c["kind"] == "rotate":
        # text, images and frames in turn: time steps slowly, height and width sweep a grid
        p, sec = s["pos"], _sections(c)
        A = len(sec)
        axes = torch.stack([p if a == 0 else p // 7 ** a % 1024 for a in range(A)]).to(torch.int32)
        s["positions"] = torch.full((A, cap), -1, dtype=torch.int32, device="cuda")
        s["positions"][:, s["rows"]] = axes
        s["freq"] = [10000.0 ** (-2 * j / d) for j in range(sum(sec))]
        s["axis"] = [a for a, n in enumerate(sec) for _ in range(n)]
        s["q"], s["k"] = randn(cap, Hq, d).to(t), randn(cap, Hkv, d).to(t)
        s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
    else:
        shape, n = (s["pages"], Hkv, c["ps"]), d * c["bits"] // 8
        s["cache"] = [torch.zeros(*shape, m, dtype=torch.uint8, device="cuda")
                      for _ in "kv" for m in (n, d // 32)]
        # a few channels of the keys are large in every token, as trained projections leave them
        wide = 1 + 5 * (torch.rand(1, Hkv, 1, d, generator=g, device="cuda") > 0.95)
        if c["kind"] != "store":
            # a cache that earlier steps have filled
            few = max(1, (64 << 20) // (Hkv * c["ps"] * d))
            for at in range(0, s["pages"], few):
                m = min(few, s["pages"] - at)
                for i in (0, 2):
                    x = randn(m, Hkv, c["ps"], d)
                    codes, scales = _quantise(x * wide if i == 0 else x, c["bits"])
                    s["cache"][i][at:at + m], s["cache"][i + 1][at:at + m] = codes, scales
        if c["kind"] == "attend":
            s["q"] = randn(cap, Hq, d).to(t)
            s["out"] = torch.zeros_like(s["q"])
        else:
            # spans to read: the window, or the committed prefix
            own_w = [w * c["bl"] for w in s["w"]]
            spans = [[o, n] for o, n in zip(s["o"], own_w)] if c["kind"] == "store" \
                else [[0, o] for o in s["o"]]
            s["spans"] = torch.tensor(spans, dtype=torch.int32, device="cuda")
            T = c["W"] * c["bl"] if c["kind"] == "store" else c["hi"]
            s["span_list"] = spans
            s["k_out"] = torch.zeros(B, T, Hkv, d, dtype=t, device="cuda")
            s["v_out"] = torch.zeros_like(s["k_out"])
        if c["kind"] == "store":
            s["k"] = (randn(cap, Hkv, d) * wide[:, :, 0]).to(t)
            s["v"] = randn(cap, Hkv, d).to(t)
    if own:
        from paper_2607_17652_amd import binding as fb
        s["fb"] = fb
        buf = torch.zeros(fb.fb_pack_bytes(B, c["W"], c["bl"]), dtype=torch.uint8, device="cuda")
        s["pack"] = fb.fb_pack_init(buf, B, c["W"], c["bl"], c["layout"])
        fb.fb_pack_wavefronts(s["st"], None, s["n_max"], s["T_max"], s["pack"])
        s["shape"] = fb.make_shape(Hq, Hkv, d, c["dtype"], c["ps"], s["table"].shape[1], s["pages"])
        if c["kind"] == "rotate":
            s["rotary"] = fb.make_rotary(s["freq"], s["axis"], c["pairing"])
        else:
            s["mx"] = fb.make_mx_cache(c["bits"], *s["cache"])
        if c["kind"] == "attend":
            s["ws"] = torch.empty(fb.fb_mx_attention_workspace_bytes(s["pack"], s["shape"]),
                                  dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------- runs ---
def run(s):
    c = s["case"]
    kind, d = c["kind"], c["d"]
    if own:
        fb = s["fb"]
        if kind == "rotate":
            fb.fb_rotary_axes(s["q"], s["q_out"], s["k"], s["k_out"], s["positions"], s["pack"],
                              s["shape"], s["rotary"])
            return s["q_out"], s["k_out"]
        if kind == "attend":
            fb.fb_mx_attention(s["q"], s["mx"], s["table"], s["pack"], s["shape"], s["out"], s["ws"])
            return s["out"]
        if kind == "store":
            fb.fb_mx_write_window_kv(s["k"], s["v"], s["mx"], s["table"], s["pack"], s["shape"])
        fb.fb_mx_read_kv(s["mx"], s["table"], s["spans"], s["k_out"], s["v_out"], s["pack"],
                         s["shape"])
        return s["k_out"], s["v_out"]
    rows = s["rows"]
    if kind == "rotate":
        n = len(s["freq"])
        freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
        ax = torch.tensor(s["axis"], device="cuda")
        angle = s["positions"][:, rows].double()[ax].T * freq          # [rows, n]
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
            y = x[rows].float()
            if c["pairing"] == "halves":
                a, b = y[..., :n], y[..., n:2 * n]
                turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
            else:
                a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
                turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
            out[rows] = torch.cat([turned, y[..., 2 * n:]], -1).to(out.dtype)
        return s["q_out"], s["k_out"]
    if kind == "store":
        page = s["table"][s["req"], s["pos"] // c["ps"]].long()
        at = s["pos"] % c["ps"]
        for i, x in ((0, s["k"]), (2, s["v"])):
            codes, scales = _quantise(x[rows], c["bits"])
            s["cache"][i][page, :, at], s["cache"][i + 1][page, :, at] = codes, scales
    if kind != "attend":
        for b, (first, n) in enumerate(s["span_list"]):
            for i, out in ((0, s["k_out"]), (2, s["v_out"])):
                out[b, :n] = _dense(s, b, i, first, n).to(out.dtype)
        return s["k_out"], s["v_out"]
    bl, Hkv, g = c["bl"], c["Hkv"], c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        o, n, r0 = s["o"][b], s["w"][b] * bl, s["first"][b]
        k = _dense(s, b, 0, 0, o + n).permute(1, 2, 0).contiguous()     # [Hkv, d, keys]
        v = _dense(s, b, 2, 0, o + n).permute(1, 0, 2).contiguous()     # [Hkv, keys, d]
        q = s["q"][r0:r0 + n].float().view(n, Hkv, g, d).permute(1, 0, 2, 3).reshape(Hkv, n * g, d)
        z = q @ k * (1 / math.sqrt(d))
        seen = o + (torch.arange(n, device="cuda") // bl + 1) * bl      # keys of each row
        hidden = torch.arange(o + n, device="cuda") >= seen.repeat_interleave(g)[:, None]
        z.masked_fill_(hidden, -math.inf)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        y = p @ v / p.sum(-1, keepdim=True)
        s["out"][r0:r0 + n] = y.view(Hkv, n, g, d).permute(1, 0, 2, 3).reshape(n, -1, d).to(
            s["out"].dtype)
    return s["out"]


def _dense(s, b, i, first, n):
    """Positions [first, first + n) of request b's keys (i = 0) or values (2): [n, Hkv, d]."""
    c = s["case"]
    pos = torch.arange(first, first + n, device="cuda")
    page, at = s["table"][b, pos // c["ps"]].long(), pos % c["ps"]
    return _values(s["cache"][i][page, :, at], s["cache"][i + 1][page, :, at], c["bits"])


def work(case):
    c = case
    bl, B, elt = c["bl"], c["B"], 2 if c["dtype"] == "bf16" else 4
    # live rows: the middle of the range of windows, the first request's at its largest
    w = (c["w_lo"] + c["w_hi"]) / 2
    rows = bl * ((B - 1) * w + c["w_hi"])
    held = 2 * c["Hkv"] * (c["d"] * c["bits"] / 8 + c["d"] / 32)        # a token in the cache
    dense = 2 * c["Hkv"] * c["d"] * elt                                 # and outside
    prefix = (c["hi"] - c["lo"]) / max(1e-9, math.log((c["hi"] + 1e-6) / c["lo"]))
    prefix = prefix if c["hi"] > c["lo"] else c["hi"]
    if c["kind"] == "rotate":
        heads = c["Hq"] + c["Hkv"]
        return {"bytes": rows * (2 * heads * c["d"] * elt + 4 * len(_sections(c))),
                "flops": rows * heads * sum(_sections(c)) * 6}
    if c["kind"] == "store":
        return {"bytes": rows * (2 * dense + 2 * held), "flops": rows * 2 * c["Hkv"] * c["d"] * 4}
    if c["kind"] == "read":
        return {"bytes": B * prefix * (held + dense), "flops": B * prefix * 2 * c["Hkv"] * c["d"]}
    keys = prefix + bl * (w + 1) / 2                                    # the mean row's
    return {"bytes": B * (prefix + bl * w) * held + 2 * rows * c["Hq"] * c["d"] * elt,
            "flops": 4 * rows * c["Hq"] * c["d"] * keys}


# --------------------------------------------------------------- in 64 bits ---
def _grid(bits):
    """The code values >= 0, ascending."""
    if bits == 4:
        return [m / 2 for m in (0, 1, 2, 3)] + [2.0, 3.0, 4.0, 6.0]
    return [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16)
                                                for m in range(8)][:-1]


def _nearest64(x, bits):
    """What the quantised x stands for."""
    grid = torch.tensor(_grid(bits), dtype=torch.float64, device=x.device)
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().max(-1, keepdim=True).values
    e = torch.ceil(torch.log2(top / grid[-1]))
    lo, hi = _E_RANGE[bits]
    scale = 2.0 ** torch.where(top > 0, e, lo).clamp(lo, hi)
    a = (g.abs() / scale).clamp(max=float(grid[-1]))
    up = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)   # first code >= a
    dn = (up - 1).clamp(min=0)
    below, above = a - grid[dn], grid[up] - a
    pick = torch.where((above < below) | ((above == below) & (up % 2 == 0)), up, dn)
    return (torch.sign(g) * grid[pick] * scale).reshape(x.shape)


def _held64(s, b, i, n):
    """The first n keys or values of request b in float64: [n, Hkv, d]."""
    c = s["case"]
    ids = s["table"][b, :-(-n // c["ps"])].long()
    codes, scales = s["cache"][i][ids], s["cache"][i + 1][ids]
    grid = torch.tensor(_grid(c["bits"]), dtype=torch.float64, device=codes.device)
    if c["bits"] == 4:
        q = torch.empty(*codes.shape[:-1], c["d"], dtype=torch.int64, device=codes.device)
        q[..., 0::2], q[..., 1::2] = codes.long() % 16, codes.long() // 16
        y = torch.where(q >= 8, -grid[q % 8], grid[q % 8])
    else:
        q = codes.long()
        m = grid[(q % 128).clamp(max=len(grid) - 1)]
        y = torch.where(q >= 128, -m, m)
    y = y * (2.0 ** (scales.double() - 127)).repeat_interleave(32, -1)
    return y.transpose(1, 2).reshape(-1, c["Hkv"], c["d"])[:n]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    rows, d = s["rows"], c["d"]
    if c["kind"] == "rotate":
        outs = []
        theta = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
        p = s["positions"][torch.tensor(s["axis"], device="cuda")].double()     # [pairs, cap]
        turn = torch.polar(torch.ones_like(p[:, rows]), p[:, rows] * theta[:, None]).T[:, None]
        n = len(s["freq"])
        for x in (s["q"], s["k"]):
            y = x[rows].double()
            at = torch.arange(n, device="cuda")
            i, j = (at, at + n) if c["pairing"] == "halves" else (2 * at, 2 * at + 1)
            z = torch.complex(y[..., i], y[..., j]) * turn
            y[..., i], y[..., j] = z.real, z.imag
            full = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
            full[rows] = y
            outs.append(full)
        return tuple(outs)
    if c["kind"] == "store":
        outs = []
        for x in (s["k"], s["v"]):
            out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
            for b, (_, n) in enumerate(s["span_list"]):
                out[b, :n] = _nearest64(x[s["first"][b]:s["first"][b] + n], c["bits"])
            outs.append(out)
        return tuple(outs)
    if c["kind"] == "read":
        outs = []
        for i in (0, 2):
            out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
            for b, (_, n) in enumerate(s["span_list"]):
                out[b, :n] = _held64(s, b, i, n)
            outs.append(out)
        return tuple(outs)
    out = torch.zeros(s["cap"], c["Hq"], d, dtype=torch.float64, device="cuda")
    g = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        o, bl, r0 = s["o"][b], c["bl"], s["first"][b]
        k, v = (_held64(s, b, i, o + s["w"][b] * bl) for i in (0, 2))
        for h in range(c["Hkv"]):
            kt = k[:, h].t().contiguous()
            for t in range(s["w"][b]):                     # one block of the window at a time
                n, r = o + (t + 1) * bl, r0 + t * bl
                q = s["q"][r:r + bl, h * g:(h + 1) * g].double().reshape(bl * g, d)
                p = torch.softmax(q @ kt[:, :n] / math.sqrt(d), -1)
                out[r:r + bl, h * g:(h + 1) * g] = (p @ v[:n, h].contiguous()).view(bl, g, d)
    return out
