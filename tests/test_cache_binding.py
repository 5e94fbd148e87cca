"""The binding of the quantised cache and of the rotary refuses tensors that do not agree,
before the library sees a pointer.  CPU only, with stand-ins for device tensors; every
call here holds one thing that is wrong."""
import pytest
import torch

from paper_2607_17652_amd import binding as fb
from test_tail_binding import BF, F32, I32, U8, Device, Null, device, refused, wrong

B, ROWS, HQ, HKV, D, PS, MP, NP, T, A = 2, 24, 4, 2, 64, 8, 5, 9, 6, 3


@pytest.fixture
def pack():
    p = fb.fb_pack_init(torch.zeros(1 << 16, dtype=U8), B, 3, 4, "ragged")
    assert p.row_cap == ROWS
    return p


def shape(dtype):
    return fb.make_shape(HQ, HKV, D, dtype, PS, MP, NP)


def sizes(bits):
    n = D * bits // 8
    return dict(k_codes=(NP, HKV, PS, n), k_scales=(NP, HKV, PS, D // 32),
                v_codes=(NP, HKV, PS, n), v_scales=(NP, HKV, PS, D // 32))


def cache(bits, **other):
    t = {k: device(*s, dtype=U8) for k, s in sizes(bits).items()}
    return fb.make_mx_cache(bits, *dict(t, **other).values())


def calls(bits, dtype, pack):
    """(function, its tensors in order, shapes): cache and page table among them."""
    table = dict(page_table=(B, MP))
    return [
        (lambda t, c: fb.fb_mx_write_window_kv(t["k_new"], t["v_new"], c, t["page_table"], pack, shape(dtype), Null),
         dict(k_new=(ROWS, HKV, D), v_new=(ROWS, HKV, D)), table),
        (lambda t, c: fb.fb_mx_read_kv(c, t["page_table"], t["spans"], t["k_out"], t["v_out"], pack, shape(dtype),
                                       Null),
         dict(k_out=(B, T, HKV, D), v_out=(B, T, HKV, D)), dict(table, spans=(B, 2))),
        (lambda t, c: fb.fb_mx_attention(t["q"], c, t["page_table"], pack, shape(dtype), t["out"],
                                         device(64, dtype=U8), Null),
         dict(q=(ROWS, HQ, D), out=(ROWS, HQ, D)), table)]


@pytest.mark.parametrize("dtype,other", [(BF, F32), (F32, BF)])
@pytest.mark.parametrize("bits", [4, 8])
def test_tensors_of_the_cache_calls(pack, bits, dtype, other):
    for call, floats, ints in calls(bits, dtype, pack):
        good = {k: device(*s, dtype=dtype) for k, s in floats.items()}
        good.update({k: device(*s, dtype=I32) for k, s in ints.items()})
        for k, s in {**floats, **ints}.items():
            t, o = (dtype, other) if k in floats else (I32, F32)
            for why, bad in wrong(s, t, o):
                refused(f"{k} {why}", lambda: call(dict(good, **{k: bad}), cache(bits)))
        # a cache of fewer pages than the shape says
        for k, s in sizes(bits).items():
            less = cache(bits, **{k: device(NP - 1, *s[1:], dtype=U8)})
            refused(f"{k} has", lambda: call(good, less))


@pytest.mark.parametrize("bits", [4, 8])
def test_cache_tensors(bits):
    for k, s in sizes(bits).items():
        strided = Device(torch.zeros(*s[:-1], 2 * s[-1], dtype=U8)[..., ::2])
        for why, bad in (("holds torch.float32", device(*s)), ("is not contiguous", strided),
                         ("is not on the GPU", torch.zeros(*s, dtype=U8))):
            refused(f"{k} {why}", lambda: cache(bits, **{k: bad}))


def test_codes_of_another_width_are_too_few(pack):
    """Four-bit codes seen as eight-bit ones."""
    c = cache(4)
    c.format = fb.FB_MX8
    t = {k: device(ROWS, HKV, D, dtype=BF) for k in ("k", "v")}
    refused("k_codes has", fb.fb_mx_write_window_kv, t["k"], t["v"], c, device(B, MP, dtype=I32), pack,
            shape(BF), Null)


def test_read_outputs_of_other_lengths(pack):
    t = [device(B, n, HKV, D, dtype=BF) for n in (T, T + 1)]
    refused("differ", fb.fb_mx_read_kv, cache(4), device(B, MP, dtype=I32), device(B, 2, dtype=I32), *t, pack,
            shape(BF), Null)


@pytest.mark.parametrize("dtype,other", [(BF, F32), (F32, BF)])
def test_rotary(pack, dtype, other):
    floats = dict(q_in=(ROWS, HQ, D), q_out=(ROWS, HQ, D), k_in=(ROWS, HKV, D), k_out=(ROWS, HKV, D))
    good = {k: device(*s, dtype=dtype) for k, s in floats.items()}
    good["positions"] = device(A, ROWS, dtype=I32)
    rot = fb.make_rotary([1.0, 0.5, 0.25], [0, 1, 2])
    for k, s in dict(floats, positions=(A, ROWS)).items():
        t, o = (dtype, other) if k in floats else (I32, F32)
        for why, bad in wrong(s, t, o):
            refused(f"{k} {why}", fb.fb_rotary_axes, *dict(good, **{k: bad}).values(), pack, shape(dtype), rot,
                    Null)


@pytest.mark.parametrize("freq,axis", [([], []), ([1.0], []), ([1.0] * 65, [0] * 65), ([1.0], [8]), ([1.0], [-1])])
def test_make_rotary_refuses(freq, axis):
    refused("", fb.make_rotary, freq, axis)


def test_sections():
    freq, axis = fb.rotary_sections(64, (2, 0, 1), base=100.0)
    assert axis == [0, 0, 2] and freq == [100.0 ** (-2 * j / 64) for j in range(3)]
    r = fb.make_rotary(freq, axis, "neighbours")
    assert (r.n_axes, r.n_pairs, r.pairing) == (3, 3, 1) and list(r.axis[:3]) == axis
