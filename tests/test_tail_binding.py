"""The binding of the model's tail refuses tensors that do not agree, before the library
sees a pointer: types, sizes, strides, host memory.  CPU only, with stand-ins for device
tensors; every call here holds one thing that is wrong."""
import pytest
import torch

from paper_2607_17652_amd import binding as fb

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
B, ROWS, D, N, K, V = 2, 24, 64, 40, 96, 1000


class Device:
    """A host tensor that says it is on the GPU."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


class Null:
    cuda_stream = 0


def device(*shape, dtype=F32):
    return Device(torch.zeros(*shape, dtype=dtype))


def strided(*shape, dtype=F32):
    return Device(torch.zeros(*shape[:-1], 2 * shape[-1], dtype=dtype)[..., ::2])


@pytest.fixture
def pack():
    p = fb.fb_pack_init(torch.zeros(1 << 16, dtype=U8), B, 3, 4, "ragged")
    assert p.row_cap == ROWS
    return p


def refused(why, call, *args):
    with pytest.raises(fb.FlowBlockError) as e:
        call(*args)
    assert e.value.code == fb.FB_E_INVAL and why in str(e.value), e.value


def wrong(shape, dtype, other):
    """(what is said, a tensor) for everything that can be wrong with one."""
    less = (shape[0] - 1,) + tuple(shape[1:])
    return [(f"holds {other}", device(*shape, dtype=other)), ("has", device(*less, dtype=dtype)),
            ("is not contiguous", strided(*shape, dtype=dtype)),
            ("is not on the GPU", torch.zeros(*shape, dtype=dtype))]


@pytest.mark.parametrize("dtype,other", [(BF, F32), (F32, BF)])
@pytest.mark.parametrize("gate", ["all", "request", "row"])
def test_residual_norm(pack, gate, dtype, other):
    shapes = dict(y=(ROWS, D), h=(ROWS, D), gate={"all": (D,), "request": (B, D), "row": (ROWS, D)}[gate],
                  w_post=(D,), w_pre=(D,), h_out=(ROWS, D), n_out=(ROWS, D))
    t = {k: device(*s, dtype=dtype) for k, s in shapes.items()}
    sh = fb.make_norm_shape(D, dtype, gate)
    for k, s in shapes.items():
        for why, bad in wrong(s, dtype, other):
            refused(f"{k} {why}", fb.fb_residual_norm, *dict(t, **{k: bad}).values(), pack, sh)
    # one row's gate seen as every row's
    if gate == "row":
        t["gate"] = Device(torch.zeros(1, D, dtype=dtype).expand(ROWS, D))
        refused("gate is not contiguous", fb.fb_residual_norm, *t.values(), pack, sh)
    # all of one type, the shape of another: read and written past their ends
    t = {k: device(*s, dtype=dtype) for k, s in shapes.items()}
    refused(f"holds {dtype}, not {other}", fb.fb_residual_norm, *t.values(), pack,
            fb.make_norm_shape(D, other, gate))


def test_arrays_that_may_not_be_absent_are_the_library_s_to_refuse(pack):
    sh = fb.make_norm_shape(D, "bf16")
    refused("h is NULL", fb.fb_residual_norm, None, None, None, None, None, None, None, pack, sh, Null)
    r = fb.make_rules(*rules().values())
    ws, z = device(1 << 20, dtype=U8), device(ROWS, V)
    refused("state or tokens", fb.fb_rules_build, r, None, device(B, 50, dtype=I32), V, pack, ws, Null)
    refused("out must be", fb.fb_logits_rules, z, None, pack, r, ws, Null)


def test_mx4_linear(pack):
    t = dict(x=device(ROWS, K, dtype=BF), codes=device(N, K // 2, dtype=U8),
             scales=device(N, K // 32, dtype=U8), y=device(ROWS, N))

    def call(**kw):
        a = dict(t, **kw)
        return fb.fb_mx4_linear, a["x"], a["codes"], a["scales"], pack, a["y"]
    for why, bad in wrong((ROWS, K), BF, torch.float16):
        refused(f"x {why}", *call(x=bad))
    for why, bad in wrong((ROWS, N), F32, BF)[1:]:
        refused(f"y {why}", *call(y=bad))
    for k, width in (("codes", K // 2), ("scales", K // 32)):
        refused(f"{k} has", *call(**{k: device(N, width + 1, dtype=U8)}))     # those of another K
        refused(f"{k} has", *call(**{k: device(N, width - 1, dtype=U8)}))
        refused(f"{k} holds torch.int32", *call(**{k: device(N, width, dtype=I32)}))
        refused(f"{k} is not contiguous", *call(**{k: strided(N, width, dtype=U8)}))
        refused(f"{k} is not on the GPU", *call(**{k: torch.zeros(N, width, dtype=U8)}))
    with pytest.raises(fb.FlowBlockError) as e:
        f, *a = call(y=device(ROWS, N, dtype=torch.float16))
        f(*a)
    assert e.value.code == fb.FB_E_UNSUPPORTED
    # bytes by another name pass
    assert fb._octets(device(N, K // 2, dtype=torch.float8_e4m3fn), N * K // 2, "codes")


RULES = dict(params=((B, 4), F32, BF), bias_start=((B + 1,), I32, torch.int64), bias_id=((8,), I32, torch.int64),
             bias_val=((8,), F32, torch.float64), masks=((3, 32), I32, torch.bool),
             row_mask=((ROWS,), I32, torch.int64))


def rules(**kw):
    return {k: kw.get(k, device(*s, dtype=d)) for k, (s, d, _) in RULES.items()}


@pytest.mark.parametrize("name", RULES)
def test_make_rules(name):
    shape, dtype, other = RULES[name]
    for why, bad in wrong(shape, dtype, other):
        if why != "has":
            refused(f"{name} {why}", fb.make_rules, *rules(**{name: bad}).values())
    fb.make_rules(*rules().values())
    fb.make_rules(*rules(masks=device(3, 32, dtype=torch.uint32)).values())
    # one mask as a vector is one mask, not as many as it has words
    assert fb.make_rules(*rules(masks=device(32, dtype=I32)).values()).n_masks == 1
    assert fb.make_rules(*rules().values()).n_masks == 3
    refused("bias_val has 7 elements, needs 8", fb.make_rules, *rules(bias_val=device(7)).values())


def test_rules_fit_the_pack_and_the_vocabulary(pack):
    ws, z = device(1 << 20, dtype=U8), device(ROWS, V)
    st, tok = device(B, 8, dtype=I32), device(B, 50, dtype=I32)

    def calls(r):
        yield fb.fb_vocab_reduce_rules, z, pack, r, ws, ws
        yield fb.fb_logits_rules, z, z, pack, r, ws
        yield fb.fb_rules_build, r, st, tok, V, pack, ws
    for name, bad in (("params has", dict(params=device(B - 1, 4))),
                      ("bias_start has", dict(bias_start=device(B, dtype=I32))),
                      ("masks have rows of 31 words", dict(masks=device(3, 31, dtype=I32))),
                      ("masks have rows of 33 words", dict(masks=device(3, 33, dtype=I32))),
                      ("row_mask has", dict(row_mask=device(ROWS - 1, dtype=I32)))):
        r = fb.make_rules(*rules(**bad).values())
        for call, *a in calls(r):
            if "mask" in name and call is fb.fb_rules_build:
                fb._rules(r, pack)          # which reads no masks
            else:
                refused(name, call, *a)


def test_rules_calls(pack):
    r = fb.make_rules(*rules().values())
    ws, z = device(1 << 20, dtype=U8), device(ROWS, V)
    st, tok = device(B, 8, dtype=I32), device(B, 50, dtype=I32)
    conf, top = device(ROWS), device(ROWS, dtype=I32)
    for why, bad in wrong((B, 8), I32, None)[1:]:
        refused(f"st {why}", fb.fb_rules_build, r, bad, tok, V, pack, ws)
    for why, bad in wrong((B, 50), I32, torch.int64):
        refused(f"tokens {why}", fb.fb_rules_build, r, st, bad, V, pack, ws)
    for why, bad in wrong((ROWS, V), F32, BF)[1:]:
        refused(f"logits {why}", fb.fb_vocab_reduce_rules, bad, pack, r, ws, ws, conf, top)
        refused(f"logits {why}", fb.fb_logits_rules, bad, z, pack, r, ws)
    for why, bad in wrong((ROWS, V), F32, BF):
        refused(f"out {why}", fb.fb_logits_rules, z, bad, pack, r, ws)
    for why, bad in wrong((ROWS,), F32, torch.float64):
        refused(f"conf {why}", fb.fb_vocab_reduce_rules, z, pack, r, ws, ws, bad, top)
    for why, bad in wrong((ROWS,), I32, torch.int64):
        refused(f"argmax {why}", fb.fb_vocab_reduce_rules, z, pack, r, ws, ws, conf, bad)
    for why, bad in wrong((1 << 10,), U8, None)[2:]:
        refused(f"ws {why}", fb.fb_rules_build, r, st, tok, V, pack, bad)
        refused(f"rules_ws {why}", fb.fb_vocab_reduce_rules, z, pack, r, bad, ws)
        refused(f"upd_ws {why}", fb.fb_vocab_reduce_rules, z, pack, r, ws, bad)
        refused(f"rules_ws {why}", fb.fb_logits_rules, z, z, pack, r, bad)
    for half in (device(ROWS, V, dtype=torch.float16),):
        with pytest.raises(fb.FlowBlockError) as e:
            fb.fb_logits_rules(half, half, pack, r, ws)
        assert e.value.code == fb.FB_E_UNSUPPORTED
