"""The model tail's calls refuse what the host can see to be wrong before
anything is launched, and their structs match the header.  CPU only."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_17652_amd import binding as fb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x100000)      # never dereferenced
Q = ctypes.c_void_p(0x40000000)
R = ctypes.c_void_p(0x80000000)
ODD = ctypes.c_void_p(0x100001)
OFF8 = ctypes.c_void_p(0x100008)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fb.LIB_PATH):
        from paper_2607_17652_amd import build
        build.build()
    return fb.lib()


@pytest.fixture
def pack(lib):
    h = fb.fb_pack()
    assert lib.fb_pack_init(ctypes.byref(h), P, BIG, 2, 2, 4, fb.FB_RAGGED) == fb.FB_OK
    return h


def test_struct_layouts(tmp_path):
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "flowblock_tail.h"',
             "int main(void) {", 'printf("p %zu\\n", sizeof(fb_rule_params));']
    structs = [fb.fb_norm_shape, fb.fb_logit_rules]
    for S in structs:
        lines.append(f'printf("{S.__name__} %zu\\n", sizeof({S.__name__}));')
        lines += [f'printf("{S.__name__}.{f} %zu\\n", offsetof({S.__name__}, {f}));'
                  for f, _ in S._fields_]
    lines += ["return 0;", "}"]
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    assert got["p"] == "16"
    for S in structs:
        assert int(got[S.__name__]) == ctypes.sizeof(S)
        for f, _ in S._fields_:
            assert int(got[f"{S.__name__}.{f}"]) == getattr(S, f).offset


@pytest.mark.parametrize("want,change", [
    ("INVAL", dict(h=None)), ("INVAL", dict(h_out=None)), ("INVAL", dict(D=0)),
    ("UNSUPPORTED", dict(D=16385)), ("UNSUPPORTED", dict(dtype=2)),
    ("INVAL", dict(gate_kind=4)), ("INVAL", dict(gate_kind=-1)),
    ("INVAL", dict(gate_kind=1)),                       # a layout, no gate
    ("INVAL", dict(gate=R)),                            # a gate, no layout
    ("INVAL", dict(eps=0.0)), ("INVAL", dict(eps=-1.0)), ("INVAL", dict(eps=float("nan"))),
    ("INVAL", dict(eps=float("inf"))), ("INVAL", dict(a=float("inf"))),
    ("INVAL", dict(a=float("nan"))),
    ("INVAL", dict(y=None)),                            # a plain norm with h_out
    ("INVAL", dict(y=None, h_out=None, w_post=R)),
    ("INVAL", dict(n_out=None)),                        # w_pre without n_out
    ("INVAL", dict(y=None, h_out=None, n_out=None, w_pre=None)),
    ("INVAL", dict(y=ODD)),
    ("INVAL", dict(n_out=Q)),                           # n_out == h_out
    ("INVAL", dict(h_out=OFF8)),                        # overlaps y (and h) without being h
    ("INVAL", dict(pack=None)),
])
def test_residual_norm_refuses(lib, pack, want, change):
    a = dict(y=P, h=R, gate=None, w_post=None, w_pre=R, h_out=Q,
             n_out=ctypes.c_void_p(0xc0000000), D=64, dtype=fb.FB_BF16, gate_kind=0, eps=1e-6,
             a=1.0, pack=ctypes.byref(pack))
    a.update(change)
    sh = fb.fb_norm_shape(a["D"], a["dtype"], a["gate_kind"], a["eps"], a["a"])
    rc = lib.fb_residual_norm(a["y"], a["h"], a["gate"], a["w_post"], a["w_pre"], a["h_out"],
                              a["n_out"], a["pack"], ctypes.byref(sh), None)
    assert rc == getattr(fb, "FB_E_" + want), fb.fb_last_error()
    assert fb.fb_last_error()


@pytest.mark.parametrize("want,change", [
    ("INVAL", dict(x=None)), ("INVAL", dict(codes=None)), ("INVAL", dict(scales=None)),
    ("INVAL", dict(y=None)), ("INVAL", dict(N=0)), ("INVAL", dict(K=0)), ("INVAL", dict(K=48)),
    ("UNSUPPORTED", dict(K=65568)), ("UNSUPPORTED", dict(N=(1 << 30) + 1)),
    ("UNSUPPORTED", dict(dtype=3)), ("INVAL", dict(x=OFF8)),
    ("INVAL", dict(codes=OFF8)), ("INVAL", dict(y=ODD)), ("INVAL", dict(y=P)),
    ("INVAL", dict(pack=None)),
])
def test_mx4_linear_refuses(lib, pack, want, change):
    a = dict(x=P, codes=Q, scales=ODD, N=64, K=64, y=R, dtype=fb.FB_BF16,
             pack=ctypes.byref(pack))
    a.update(change)
    rc = lib.fb_mx4_linear(a["x"], a["codes"], a["scales"], a["N"], a["K"], a["pack"], a["y"],
                           a["dtype"], None)
    assert rc == getattr(fb, "FB_E_" + want), fb.fb_last_error()


def rules(**kw):
    r = fb.fb_logit_rules(params=P, bias_start=P, bias_id=P, bias_val=P, masks=P, row_mask=P,
                          n_bias=4, n_masks=1)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_RULES = [dict(n_bias=-1), dict(n_masks=-1), dict(bias_id=None), dict(bias_val=None),
             dict(row_mask=None), dict(masks=None), dict(n_masks=0), dict(masks=ODD),
             dict(params=ODD)]


@pytest.mark.parametrize("change", BAD_RULES)
def test_rules_are_checked_by_every_call(lib, pack, change):
    r, ph = ctypes.byref(rules(**change)), ctypes.byref(pack)
    assert lib.fb_rules_build(r, P, P, 64, 1000, ph, P, BIG, None) == fb.FB_E_INVAL
    assert lib.fb_vocab_reduce_rules(P, 1000, 1, ph, r, P, BIG, P, BIG, None, None,
                                     None) == fb.FB_E_INVAL
    assert lib.fb_logits_rules(P, P, 1000, 1, ph, r, P, BIG, None) == fb.FB_E_INVAL


def test_rules_calls_refuse(lib, pack):
    r, ph = ctypes.byref(rules()), ctypes.byref(pack)
    need = lib.fb_rules_workspace_bytes(ph, 1000)
    assert need > 0 and need % 16 == 0
    assert lib.fb_rules_workspace_bytes(ph, 0) == 0
    assert lib.fb_rules_workspace_bytes(ph, (1 << 19) + 1) == 0
    assert lib.fb_rules_workspace_bytes(None, 1000) == 0
    upd = lib.fb_update_workspace_bytes(ph, 1000)

    def build(rules=r, st=P, tok=P, T=64, V=1000, p=ph, ws=P, nb=need):
        return lib.fb_rules_build(rules, st, tok, T, V, p, ws, nb, None)
    assert build(rules=None) == build(st=None) == build(tok=None) == build(T=0) == fb.FB_E_INVAL
    assert build(V=0) == build(p=None) == build(ws=OFF8) == fb.FB_E_INVAL
    assert build(V=(1 << 19) + 1) == fb.FB_E_UNSUPPORTED
    assert build(ws=None) == build(nb=need - 1) == fb.FB_E_WORKSPACE

    def reduce(z=P, V=1000, dt=1, p=ph, rules=r, ws=P, nb=need, uw=P, ub=upd, c=P, am=P):
        return lib.fb_vocab_reduce_rules(z, V, dt, p, rules, ws, nb, uw, ub, c, am, None)
    assert reduce(z=None) == reduce(z=OFF8) == reduce(V=0) == reduce(rules=None) == fb.FB_E_INVAL
    assert reduce(c=None) == reduce(am=None) == reduce(uw=OFF8) == fb.FB_E_INVAL
    assert reduce(dt=5) == fb.FB_E_UNSUPPORTED
    assert reduce(nb=need - 1) == reduce(ub=upd - 1) == reduce(ws=None) == fb.FB_E_WORKSPACE

    def write(z=P, out=Q, V=1000, dt=1, p=ph, rules=r, ws=P, nb=need):
        return lib.fb_logits_rules(z, out, V, dt, p, rules, ws, nb, None)
    assert write(z=None) == write(out=None) == write(out=OFF8) == write(V=0) == fb.FB_E_INVAL
    assert write(out=ctypes.c_void_p(0x100010)) == fb.FB_E_INVAL       # a shifted overlap
    assert "overlap" in fb.fb_last_error()
    assert write(dt=9) == fb.FB_E_UNSUPPORTED
    assert write(nb=16) == fb.FB_E_WORKSPACE
