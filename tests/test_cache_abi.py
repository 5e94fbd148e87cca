"""The quantised cache's calls and the rotary's refuse what the host can see to be wrong
before anything is launched, and their structs match the header.  CPU only."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_17652_amd import binding as fb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 1 << 40


def at(i, odd=0):
    """The i-th of some far apart addresses, never dereferenced."""
    return ctypes.c_void_p((i + 1 << 40) + odd)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2607_17652_amd import build
        build.build()
    return fb.lib()


@pytest.fixture
def pack(lib):
    h = fb.fb_pack()
    assert lib.fb_pack_init(ctypes.byref(h), at(0), BIG, 2, 2, 4, fb.FB_RAGGED) == fb.FB_OK
    return h


def shape(**kw):
    s = fb.make_shape(8, 2, 64, "bf16", 16, 4, 10)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def rotary(**kw):
    r = fb.make_rotary([0.5] * 8, [0, 1] * 4)
    for k, v in kw.items():
        if k in ("freq", "axis"):
            getattr(r, k)[v[0]] = v[1]
        else:
            setattr(r, k, v)
    return r


def cache(**kw):
    c = fb.fb_mx_cache(at(10), at(11, 1), at(12), at(13, 3), fb.FB_MX4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def refused(lib, what, rc):
    assert rc == getattr(fb, "FB_E_" + what), (rc, fb.fb_last_error())
    assert fb.fb_last_error()


def test_struct_layouts(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "flowblock_cache.h"',
             "int main(void) {"]
    structs = [fb.fb_rotary, fb.fb_mx_cache]
    for S in structs:
        lines.append(f'printf("{S.__name__} %zu\\n", sizeof({S.__name__}));')
        lines += [f'printf("{S.__name__}.{f} %zu\\n", offsetof({S.__name__}, {f}));'
                  for f, _ in S._fields_]
    names = ("FB_MX4", "FB_MX8", "FB_DERR_SPAN")
    lines += [f'printf("{n} %d\\n", {n});' for n in names]
    lines += [f'printf("{n} %d\\n", FB_PAIR_{n.upper()});' for n in fb.PAIRINGS] + ["return 0;", "}"]
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    for S in structs:
        assert int(got[S.__name__]) == ctypes.sizeof(S)
        for f, _ in S._fields_:
            assert int(got[f"{S.__name__}.{f}"]) == getattr(S, f).offset
    assert all(int(got[n]) == getattr(fb, n) for n in names)
    assert all(int(got[n]) == v for n, v in fb.PAIRINGS.items())


@pytest.mark.parametrize("want,change", [
    ("INVAL", dict(shape=None)), ("INVAL", dict(shape=dict(Hq=0))), ("INVAL", dict(shape=dict(Hq=7))),
    ("UNSUPPORTED", dict(shape=dict(head_dim=96))), ("UNSUPPORTED", dict(shape=dict(dtype=2))),
    ("UNSUPPORTED", dict(shape=dict(Hq=1 << 25, Hkv=1))), ("INVAL", dict(rot=None)), ("INVAL", dict(rot=dict(n_axes=0))), ("INVAL", dict(rot=dict(n_axes=9))),
    ("INVAL", dict(rot=dict(n_pairs=0))), ("INVAL", dict(rot=dict(n_pairs=33))),
    ("INVAL", dict(rot=dict(pairing=2))), ("INVAL", dict(rot=dict(axis=(7, 2)))),
    ("INVAL", dict(rot=dict(freq=(3, float("nan"))))), ("INVAL", dict(rot=dict(freq=(0, float("inf"))))),
    ("INVAL", dict(q_in=None)), ("INVAL", dict(q_out=None)), ("INVAL", dict(k_in=None)),
    ("INVAL", dict(k_out=None)), ("INVAL", dict(q_in=None, q_out=None, k_in=None, k_out=None)),
    ("INVAL", dict(pos=None)), ("INVAL", dict(pos=at(5, 2))), ("INVAL", dict(q_in=at(1, 8))),
    ("INVAL", dict(k_out=at(4, 2))),
    # outputs over inputs and each other: 16 rows of 8 x 64 and 2 x 64 bf16
    ("INVAL", dict(q_out=at(1, 16))), ("INVAL", dict(k_out=at(3, 4080))), ("INVAL", dict(q_out=at(3))),
    ("INVAL", dict(k_out=at(1, 16368))), ("INVAL", dict(k_out=at(2, 16)))])
def test_rotary_refuses(lib, pack, want, change):
    a = dict(q_in=at(1), q_out=at(2), k_in=at(3), k_out=at(4), pos=at(5))
    a.update({k: v for k, v in change.items() if k in a})
    sh = shape(**(change.get("shape", {}) or {})) if change.get("shape", {}) is not None else None
    ro = rotary(**(change.get("rot", {}) or {})) if change.get("rot", {}) is not None else None
    refused(lib, want, lib.fb_rotary_axes(*a.values(), pack, sh, ro, None))
    refused(lib, "INVAL", lib.fb_rotary_axes(at(1), at(2), at(3), at(4), at(5), None, shape(),
                                             rotary(), None))


CACHE = [("INVAL", dict(cache=None)), ("UNSUPPORTED", dict(cache=dict(format=6))),
         ("INVAL", dict(cache=dict(k_codes=None))), ("INVAL", dict(cache=dict(k_scales=None))),
         ("INVAL", dict(cache=dict(v_codes=None))), ("INVAL", dict(cache=dict(v_scales=None))),
         ("INVAL", dict(cache=dict(k_codes=at(10, 8)))), ("INVAL", dict(cache=dict(v_codes=at(12, 1)))),
         ("INVAL", dict(table=None)), ("INVAL", dict(table=at(14, 1))),
         ("INVAL", dict(shape=dict(page_size=12))), ("INVAL", dict(shape=dict(max_pages=0))),
         ("INVAL", dict(shape=dict(num_pages=0))), ("UNSUPPORTED", dict(shape=dict(head_dim=256))),
         ("UNSUPPORTED", dict(shape=dict(Hq=1 << 24, Hkv=1 << 24))),
         ("UNSUPPORTED", dict(shape=dict(Hq=1 << 28, Hkv=1))),
         ("INVAL", dict(shape=dict(sm_scale=float("inf"))))]


def parts(change):
    sh = shape(**change.get("shape", {}))
    c = change.get("cache", {})
    return sh, None if c is None else cache(**c), change.get("table", at(14))


@pytest.mark.parametrize("want,change", CACHE + [
    ("INVAL", dict(k=None)), ("INVAL", dict(v=None)), ("INVAL", dict(k=at(1, 8))),
    ("INVAL", dict(v=at(2, 2)))])
def test_write_refuses(lib, pack, want, change):
    sh, c, tab = parts(change)
    refused(lib, want, lib.fb_mx_write_window_kv(change.get("k", at(1)), change.get("v", at(2)), c, tab,
                                                 pack, sh, None))
    refused(lib, "INVAL", lib.fb_mx_write_window_kv(at(1), at(2), cache(), at(14), None, shape(), None))


@pytest.mark.parametrize("want,change", CACHE + [
    ("INVAL", dict(spans=None)), ("INVAL", dict(spans=at(3, 2))), ("INVAL", dict(T=0)),
    ("UNSUPPORTED", dict(T=(1 << 30) + 1)),
    ("INVAL", dict(k=None, v=None)), ("INVAL", dict(k=at(1, 8))), ("INVAL", dict(v=at(2, 4))),
    ("INVAL", dict(v=at(1, 2 * 5 * 2 * 64 * 2 - 16)))])
def test_read_refuses(lib, pack, want, change):
    sh, c, tab = parts(change)
    refused(lib, want, lib.fb_mx_read_kv(c, tab, change.get("spans", at(3)), change.get("T", 5),
                                         change.get("k", at(1)), change.get("v", at(2)), pack, sh, None))
    refused(lib, "INVAL", lib.fb_mx_read_kv(cache(), at(14), at(3), 5, at(1), at(2), None, shape(), None))


@pytest.mark.parametrize("want,change", CACHE + [
    ("INVAL", dict(q=None)), ("INVAL", dict(out=None)), ("INVAL", dict(q=at(1, 8))),
    ("INVAL", dict(out=at(2, 2))), ("INVAL", dict(out=at(1, 16))), ("WORKSPACE", dict(ws=None)),
    ("WORKSPACE", dict(less=1)), ("INVAL", dict(ws=at(3, 8)))])
def test_attention_refuses(lib, pack, want, change):
    sh, c, tab = parts(change)
    size = lib.fb_mx_attention_workspace_bytes(pack, sh)
    if "shape" in change:
        assert size == 0
    else:
        assert size > 0
    refused(lib, want, lib.fb_mx_attention(change.get("q", at(1)), c, tab, pack, sh,
                                           change.get("out", at(2)), change.get("ws", at(3)),
                                           size - change.get("less", 0), None))
    refused(lib, "INVAL", lib.fb_mx_attention(at(1), cache(), at(14), None, shape(), at(2), at(3), BIG, None))


def test_the_quantised_cache_takes_pages_of_any_power_of_two(lib, pack):
    """(the bf16 cache needs eight keys to a page)"""
    for ps in (1, 2, 4, 8, 1024):
        assert lib.fb_mx_attention_workspace_bytes(pack, shape(page_size=ps)) > 0
    assert lib.fb_mx_attention_workspace_bytes(None, shape()) == 0


def test_workspace_follows_the_form(lib, pack):
    """32 query rows to a unit where a request has no more, 128 otherwise."""
    few = lib.fb_mx_attention_workspace_bytes(pack, shape(Hq=8, Hkv=2))      # 8 rows x 4 heads
    more = lib.fb_mx_attention_workspace_bytes(pack, shape(Hq=10, Hkv=2))
    assert 5.9 < more / few < 6.1        # and three workgroups a CU, not two
