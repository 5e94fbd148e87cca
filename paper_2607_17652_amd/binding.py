"""ctypes binding of libflowblock.so -- argument marshalling, and checks of what the
library cannot see of the tail's and the quantised cache's tensors.

Each function has the name of the C entry point it calls and takes torch
tensors where the C call takes device pointers; every step of the work runs
in the library's HIP kernels.  A non-zero status raises ``FlowBlockError``
with the library's message.  Loading fails loudly if the library is not built:
there is no fallback path.
"""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflowblock.so")

FB_OK = 0
FB_E_INVAL = -1
FB_E_UNSUPPORTED = -2
FB_E_WORKSPACE = -3
FB_E_HIP = -4

FB_DERR_NONE = 0
FB_DERR_STATE = 1
FB_DERR_PAGE = 2
FB_DERR_PLAN = 3
FB_DERR_RULE = 4
FB_DERR_SPAN = 5

FB_F32 = 0
FB_BF16 = 1
FB_I32 = -1       # for _type alone: no call takes it
FB_RAGGED = 0
FB_PADDED = 1
FB_EDIT_MASKED = 1
FB_FORCE_PROGRESS = 2
FB_SYNC_WINDOW = 4
FB_MX4 = 4
FB_MX8 = 8

LAYOUTS = {"ragged": FB_RAGGED, "padded": FB_PADDED}
PAIRINGS = {"halves": 0, "neighbours": 1}
GATES = {"none": 0, "all": 1, "request": 2, "row": 3}

# Every symbol include/*.h declares.
EXPORTS = [
    "fb_version", "fb_last_error", "fb_pack_bytes", "fb_pack_get_offsets",
    "fb_pack_init", "fb_pack_wavefronts", "fb_pack_read_status",
    "fb_write_window_kv", "fb_attention_workspace_bytes",
    "fb_wavefront_attention", "fb_attention_plan", "fb_wavefront_attention_planned",
    "fb_update_workspace_bytes", "fb_denoise_update",
    "fb_vocab_reduce", "fb_denoise_apply",
    "fb_synth_embed", "fb_synth_logits", "fb_decode_loop",
    "fb_lmhead_workspace_bytes", "fb_lmhead_reduce", "fb_window_prologue",
    "fb_hbm_read_probe", "fb_hbm_copy_probe", "fb_denoise_update_noalloc",
    "fb_residual_norm", "fb_mx4_linear", "fb_rules_workspace_bytes", "fb_rules_build",
    "fb_vocab_reduce_rules", "fb_logits_rules",
    "fb_rotary_axes", "fb_mx_write_window_kv", "fb_mx_read_kv",
    "fb_mx_attention_workspace_bytes", "fb_mx_attention",
]
FB_NOALLOC_SCRATCH_BYTES = 4 << 20
FB_PROBE_BLOCKS = 2048


class FlowBlockError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"flowblock status {code}: {msg}")
        self.code = code


class fb_pack(ctypes.Structure):
    _fields_ = [("buf", ctypes.c_void_p), ("B", ctypes.c_int32),
                ("W_max", ctypes.c_int32), ("bl", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("row_cap", ctypes.c_int32),
                ("tile_cap", ctypes.c_int32)]


class fb_pack_offsets(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in
                ("header", "tiles", "req_w", "req_row0", "row_req", "row_pos",
                 "row_tok", "total")]


class fb_attn_shape(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("kv_split", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("reserved", ctypes.c_int32 * 3)]


class fb_update_params(ctypes.Structure):
    _fields_ = [("tau_mask", ctypes.c_double), ("tau_edit", ctypes.c_double),
                ("theta_spawn", ctypes.c_double), ("mask_id", ctypes.c_int32),
                ("eos_id", ctypes.c_int32), ("S_pe", ctypes.c_int32),
                ("W", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("reserved", ctypes.c_int32 * 3)]


class fb_synth_model(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("levels", ctypes.c_float * 4)]


class fb_loop_args(ctypes.Structure):
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    _fields_ = [
        ("st", vp), ("tokens", vp), ("T_max", i32), ("n_max", i32), ("pe", vp),
        ("fin", vp), ("pack", ctypes.POINTER(fb_pack)),
        ("prm", ctypes.POINTER(fb_update_params)),
        ("model", ctypes.POINTER(fb_synth_model)), ("logits", vp), ("V", i32),
        ("logit_dtype", i32), ("pred", vp), ("conf", vp), ("argmax", vp),
        ("stats", vp), ("upd_ws", vp), ("upd_ws_bytes", sz),
        ("shape", ctypes.POINTER(fb_attn_shape)), ("q", vp), ("k_new", vp),
        ("v_new", vp), ("k_cache", vp), ("v_cache", vp), ("page_table", vp),
        ("attn_out", vp), ("attn_ws", vp), ("attn_ws_bytes", sz),
        ("embed_seed", ctypes.c_uint64), ("counters", vp), ("forwards", vp)]


class fb_norm_shape(ctypes.Structure):
    _fields_ = [("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("gate", ctypes.c_int32), ("eps", ctypes.c_float),
                ("res_scale", ctypes.c_float), ("reserved", ctypes.c_int32 * 3)]


class fb_logit_rules(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("params", "bias_start", "bias_id", "bias_val", "masks", "row_mask")] + \
        [("n_bias", ctypes.c_int32), ("n_masks", ctypes.c_int32)]
    tensors = (None,) * 6       # make_rules: what the pointers belong to


class fb_rotary(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("n_pairs", ctypes.c_int32),
                ("pairing", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("freq", ctypes.c_double * 64), ("axis", ctypes.c_uint8 * 64)]


class fb_mx_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")] + \
        [("format", ctypes.c_int32), ("reserved", ctypes.c_int32)]
    tensors = (None,) * 4       # make_mx_cache: what the pointers belong to


# numpy views of the device records
REQ_STATE_DTYPE = np.dtype([(n, "<i4") for n in
                            ("gen_start", "prompt_len", "n_blocks", "L", "R",
                             "active", "eos_hit", "reserved")])
REQ_STATS_DTYPE = np.dtype([("m2t", "<i4"), ("t2t", "<i4"), ("committed", "<i4"),
                            ("spawned", "<i4"), ("eos", "<i4"), ("done", "<i4"),
                            ("valid", "<i4"), ("reserved", "<i4"),
                            ("rho_frontier", "<f8")])
assert REQ_STATE_DTYPE.itemsize == 32 and REQ_STATS_DTYPE.itemsize == 40

_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is not built; run `python -m paper_2607_17652_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        P = ctypes.POINTER
        sig = {
            "fb_version": (ctypes.c_char_p, []),
            "fb_last_error": (ctypes.c_char_p, []),
            "fb_pack_bytes": (sz, [i32, i32, i32]),
            "fb_pack_get_offsets": (i32, [i32, i32, i32, P(fb_pack_offsets)]),
            "fb_pack_init": (i32, [P(fb_pack), vp, sz, i32, i32, i32, i32]),
            "fb_pack_wavefronts": (i32, [vp, vp, i32, i32, P(fb_pack), vp]),
            "fb_pack_read_status": (i32, [P(fb_pack), P(i32), P(i32), P(i32),
                                          P(i32), vp]),
            "fb_write_window_kv": (i32, [vp, vp, vp, vp, vp, P(fb_pack),
                                         P(fb_attn_shape), vp]),
            "fb_attention_workspace_bytes": (sz, [P(fb_pack), P(fb_attn_shape)]),
            "fb_wavefront_attention": (i32, [vp, vp, vp, vp, P(fb_pack),
                                             P(fb_attn_shape), vp, vp, sz, vp]),
            "fb_attention_plan": (i32, [P(fb_pack), P(fb_attn_shape), vp, sz, vp]),
            "fb_wavefront_attention_planned": (i32, [vp, vp, vp, vp, P(fb_pack),
                                                     P(fb_attn_shape), vp, vp, sz, vp]),
            "fb_update_workspace_bytes": (sz, [P(fb_pack), i32]),
            "fb_denoise_update": (i32, [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp,
                                        i32, P(fb_pack), P(fb_update_params), vp,
                                        vp, sz, vp]),
            "fb_vocab_reduce": (i32, [vp, i32, i32, P(fb_pack), vp, sz, vp]),
            "fb_denoise_apply": (i32, [i32, vp, i32, vp, vp, vp, vp, vp, i32,
                                       P(fb_pack), P(fb_update_params), vp, vp, sz,
                                       vp]),
            "fb_window_prologue": (i32, [vp, vp, vp, vp, vp, vp, vp, P(fb_pack),
                                         P(fb_attn_shape), ctypes.c_double, vp]),
            "fb_lmhead_workspace_bytes": (sz, [P(fb_pack), i32, i32]),
            "fb_lmhead_reduce": (i32, [vp, vp, i32, i32, P(fb_pack), vp, sz, vp, sz, vp]),
            "fb_synth_embed": (i32, [P(fb_pack), P(fb_attn_shape), ctypes.c_uint64,
                                     vp, vp, vp, vp]),
            "fb_synth_logits": (i32, [vp, vp, i32, P(fb_pack), P(fb_synth_model),
                                      i32, i32, vp, vp, vp]),
            "fb_decode_loop": (i32, [P(fb_loop_args), i32, i32, i32, P(i32), P(i32),
                                     vp]),
            "fb_hbm_read_probe": (i32, [vp, sz, vp, vp]),
            "fb_denoise_update_noalloc": (i32, [vp, i32, i32, vp, i32, vp, vp, vp, vp,
                                                vp, i32, P(fb_pack), P(fb_update_params),
                                                vp, vp]),
            "fb_hbm_copy_probe": (i32, [vp, vp, sz, vp]),
            "fb_residual_norm": (i32, [vp, vp, vp, vp, vp, vp, vp, P(fb_pack),
                                       P(fb_norm_shape), vp]),
            "fb_mx4_linear": (i32, [vp, vp, vp, i32, i32, P(fb_pack), vp, i32, vp]),
            "fb_rules_workspace_bytes": (sz, [P(fb_pack), i32]),
            "fb_rules_build": (i32, [P(fb_logit_rules), vp, vp, i32, i32, P(fb_pack), vp,
                                     sz, vp]),
            "fb_vocab_reduce_rules": (i32, [vp, i32, i32, P(fb_pack), P(fb_logit_rules), vp,
                                            sz, vp, sz, vp, vp, vp]),
            "fb_logits_rules": (i32, [vp, vp, i32, i32, P(fb_pack), P(fb_logit_rules), vp, sz,
                                      vp]),
            "fb_rotary_axes": (i32, [vp, vp, vp, vp, vp, P(fb_pack), P(fb_attn_shape),
                                     P(fb_rotary), vp]),
            "fb_mx_write_window_kv": (i32, [vp, vp, P(fb_mx_cache), vp, P(fb_pack),
                                            P(fb_attn_shape), vp]),
            "fb_mx_read_kv": (i32, [P(fb_mx_cache), vp, vp, i32, vp, vp, P(fb_pack),
                                    P(fb_attn_shape), vp]),
            "fb_mx_attention_workspace_bytes": (sz, [P(fb_pack), P(fb_attn_shape)]),
            "fb_mx_attention": (i32, [vp, P(fb_mx_cache), vp, P(fb_pack), P(fb_attn_shape), vp,
                                      vp, sz, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(rc):
    if rc != FB_OK:
        raise FlowBlockError(rc, lib().fb_last_error().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = _device = None     # torch's calls, once CUDA is up


def _stream(stream):
    """The stream's handle.  The current stream comes from torch's raw-handle
    call where CUDA is up: building its Stream object takes 2.8 us of the host,
    about a third of a call."""
    if stream is not None:
        return stream.cuda_stream
    global _raw_stream, _device
    if _raw_stream is not None:
        return _raw_stream(_device())
    import torch
    c = torch._C
    if torch.cuda.is_initialized() and hasattr(c, "_cuda_getCurrentRawStream"):
        _raw_stream, _device = c._cuda_getCurrentRawStream, c._cuda_getDevice
    return torch.cuda.current_stream().cuda_stream


_types, _codes = {}, {}      # dtype code -> torch type and back; the library's int32


def _load_types():
    import torch
    _types.update({FB_BF16: torch.bfloat16, FB_F32: torch.float32, FB_I32: torch.int32})
    _codes.update({torch.bfloat16: FB_BF16, torch.float32: FB_F32})


def _type(code):
    if not _types:
        _load_types()
    t = _types.get(code)
    if t is None:
        raise FlowBlockError(FB_E_UNSUPPORTED, f"dtype {code}")
    return t


def _dtype_code(t):
    if not _codes:
        _load_types()
    code = _codes.get(t.dtype)
    if code is None:
        raise FlowBlockError(FB_E_UNSUPPORTED, f"dtype {t.dtype}")
    return code


# ------------------------------------------------------------------ library
def fb_version():
    return lib().fb_version().decode()


def fb_last_error():
    return lib().fb_last_error().decode()


# ------------------------------------------------------------------ packing
def fb_pack_bytes(B, W_max, bl):
    return int(lib().fb_pack_bytes(B, W_max, bl))


def fb_pack_get_offsets(B, W_max, bl):
    off = fb_pack_offsets()
    _check(lib().fb_pack_get_offsets(B, W_max, bl, ctypes.byref(off)))
    return {n: int(getattr(off, n)) for n, _ in fb_pack_offsets._fields_}


class Pack:
    """A host fb_pack handle plus the device buffer it points into."""

    def __init__(self, handle, buf):
        self.handle = handle
        self.buf = buf
        self.B, self.row_cap = handle.B, handle.row_cap

    @property
    def tile_cap(self):
        return self.handle.tile_cap

    def ref(self):
        return ctypes.byref(self.handle)

    def view(self):
        """int32 device views of the packed batch (header, tiles, row maps)."""
        h = self.handle
        off = fb_pack_get_offsets(h.B, h.W_max, h.bl)
        b32 = self.buf.view(dtype=__import__("torch").int32)

        def sl(a, n):
            return b32[off[a] // 4: off[a] // 4 + n]
        return dict(header=sl("header", 16),
                    tiles=sl("tiles", h.tile_cap * 8).view(h.tile_cap, 8),
                    req_w=sl("req_w", h.B), req_row0=sl("req_row0", h.B),
                    row_req=sl("row_req", h.row_cap),
                    row_pos=sl("row_pos", h.row_cap),
                    row_tok=sl("row_tok", h.row_cap))


def fb_pack_init(buf, B, W_max, bl, layout):
    """buf: a uint8 CUDA tensor of at least fb_pack_bytes(B, W_max, bl) bytes."""
    if isinstance(layout, str):
        layout = LAYOUTS[layout]
    h = fb_pack()
    _check(lib().fb_pack_init(ctypes.byref(h), _ptr(buf),
                              buf.numel() * buf.element_size(), B, W_max, bl,
                              layout))
    return Pack(h, buf)


def fb_pack_wavefronts(st, tokens, n_max, T_max, pack, stream=None):
    _check(lib().fb_pack_wavefronts(_ptr(st), _ptr(tokens), n_max, T_max,
                                    pack.ref(), _stream(stream)))


def fb_pack_read_status(pack, stream=None):
    code, req, rows, tiles = (ctypes.c_int(), ctypes.c_int(), ctypes.c_int(),
                              ctypes.c_int())
    _check(lib().fb_pack_read_status(pack.ref(), ctypes.byref(code),
                                     ctypes.byref(req), ctypes.byref(rows),
                                     ctypes.byref(tiles), _stream(stream)))
    return dict(code=code.value, request=req.value, n_rows=rows.value,
                n_tiles=tiles.value)


# ---------------------------------------------------------------- attention
def make_shape(Hq, Hkv, head_dim, dtype, page_size, max_pages, num_pages,
               kv_split=0, sm_scale=0.0):
    if not isinstance(dtype, int):
        dtype = FB_BF16 if str(dtype) in ("bf16", "torch.bfloat16") else FB_F32
    return fb_attn_shape(Hq, Hkv, head_dim, dtype, page_size, max_pages,
                         num_pages, kv_split, sm_scale)


def fb_write_window_kv(k_new, v_new, k_cache, v_cache, page_table, pack, shape,
                       stream=None):
    _check(lib().fb_write_window_kv(_ptr(k_new), _ptr(v_new), _ptr(k_cache),
                                    _ptr(v_cache), _ptr(page_table), pack.ref(),
                                    ctypes.byref(shape), _stream(stream)))


def fb_window_prologue(q_in, q_out, k_new, v_new, k_cache, v_cache, page_table, pack, shape,
                       rope_base=10000.0, stream=None):
    _check(lib().fb_window_prologue(_ptr(q_in), _ptr(q_out), _ptr(k_new), _ptr(v_new),
                                    _ptr(k_cache), _ptr(v_cache), _ptr(page_table), pack.ref(),
                                    ctypes.byref(shape), float(rope_base), _stream(stream)))


def fb_attention_workspace_bytes(pack, shape):
    return int(lib().fb_attention_workspace_bytes(pack.ref(), ctypes.byref(shape)))


def fb_wavefront_attention(q, k_cache, v_cache, page_table, pack, shape, out,
                           ws, stream=None):
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().fb_wavefront_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache),
                                        _ptr(page_table), pack.ref(),
                                        ctypes.byref(shape), _ptr(out), _ptr(ws),
                                        nbytes, _stream(stream)))


def fb_attention_plan(pack, shape, ws, stream=None):
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().fb_attention_plan(pack.ref(), ctypes.byref(shape), _ptr(ws), nbytes,
                                   _stream(stream)))


def fb_wavefront_attention_planned(q, k_cache, v_cache, page_table, pack, shape, out,
                                   ws, stream=None):
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().fb_wavefront_attention_planned(_ptr(q), _ptr(k_cache), _ptr(v_cache),
                                                _ptr(page_table), pack.ref(),
                                                ctypes.byref(shape), _ptr(out), _ptr(ws),
                                                nbytes, _stream(stream)))


# ------------------------------------------------------------------- update
def make_params(tau_mask, tau_edit, theta, mask_id, eos_id, S_pe, W,
                edit_masked=False, force_progress=False, sync_window=False):
    flags = (FB_EDIT_MASKED if edit_masked else 0) | \
        (FB_FORCE_PROGRESS if force_progress else 0) | \
        (FB_SYNC_WINDOW if sync_window else 0)
    return fb_update_params(tau_mask, tau_edit, theta, mask_id, eos_id, S_pe, W,
                            flags)


def fb_update_workspace_bytes(pack, V):
    return int(lib().fb_update_workspace_bytes(pack.ref(), V))


def fb_denoise_update(logits, tokens, conf, argmax, st, pe, fin, pack, params,
                      stats, ws, stream=None):
    """logits [row_cap, V]; tokens int32 [B, T_max]; pe/fin uint8 [B, n_max];
    st: int32 [B, 8] (fb_req_state records); stats: uint8 [B*40] or None."""
    V = logits.shape[-1]
    T_max = tokens.shape[-1]
    n_max = pe.shape[-1]
    nbytes = ws.numel() * ws.element_size()
    _check(lib().fb_denoise_update(_ptr(logits), V, _dtype_code(logits),
                                   _ptr(tokens), T_max, _ptr(conf), _ptr(argmax),
                                   _ptr(st), _ptr(pe), _ptr(fin), n_max,
                                   pack.ref(), ctypes.byref(params), _ptr(stats),
                                   _ptr(ws), nbytes, _stream(stream)))


def fb_denoise_update_noalloc(logits, tokens, conf, argmax, st, pe, fin, pack, params,
                              stats, stream=None):
    """fb_denoise_update without a workspace argument: the library's own
    per-device array serves as the workspace (nothing is allocated)."""
    _check(lib().fb_denoise_update_noalloc(_ptr(logits), logits.shape[-1],
                                           _dtype_code(logits), _ptr(tokens),
                                           tokens.shape[-1], _ptr(conf), _ptr(argmax),
                                           _ptr(st), _ptr(pe), _ptr(fin), pe.shape[-1],
                                           pack.ref(), ctypes.byref(params), _ptr(stats),
                                           _stream(stream)))


def fb_vocab_reduce(logits, pack, ws, stream=None):
    nbytes = ws.numel() * ws.element_size()
    _check(lib().fb_vocab_reduce(_ptr(logits), logits.shape[-1], _dtype_code(logits),
                                 pack.ref(), _ptr(ws), nbytes, _stream(stream)))


def fb_denoise_apply(V, tokens, conf, argmax, st, pe, fin, pack, params, stats, ws,
                     stream=None):
    nbytes = ws.numel() * ws.element_size()
    _check(lib().fb_denoise_apply(V, _ptr(tokens), tokens.shape[-1], _ptr(conf),
                                  _ptr(argmax), _ptr(st), _ptr(pe), _ptr(fin),
                                  pe.shape[-1], pack.ref(), ctypes.byref(params),
                                  _ptr(stats), _ptr(ws), nbytes, _stream(stream)))


def fb_lmhead_workspace_bytes(pack, V, D):
    return int(lib().fb_lmhead_workspace_bytes(pack.ref(), V, D))


def fb_lmhead_reduce(hidden, weight, pack, lm_ws, upd_ws, stream=None):
    """hidden bf16 [row_cap, D]; weight bf16 [V, D]; the reduction lands in
    upd_ws for fb_denoise_apply."""
    D = hidden.shape[-1]
    V = weight.shape[0]
    _check(lib().fb_lmhead_reduce(_ptr(hidden), _ptr(weight), D, V, pack.ref(), _ptr(lm_ws),
                                  lm_ws.numel() * lm_ws.element_size(), _ptr(upd_ws),
                                  upd_ws.numel() * upd_ws.element_size(), _stream(stream)))


def stats_to_numpy(stats_tensor, B):
    raw = stats_tensor.cpu().numpy().view(np.uint8)[: B * REQ_STATS_DTYPE.itemsize]
    return raw.view(REQ_STATS_DTYPE)


# ------------------------------------------------------- the model's tail
# These calls take many tensors that have to agree.  What the library cannot see of
# them is checked here: the element type, that they are dense and on the GPU, and that
# they hold all that the call reads or writes.  (Structs go to the library as they are:
# ctypes passes their address in 0.27 us less than a reference made here.)
def _dense(t, dtype, n, name):
    """The pointer of t (None: NULL), which holds n elements of `dtype` or more."""
    if t is None:
        return None
    if t.dtype is dtype and t.numel() >= n and t.is_contiguous() and t.is_cuda:
        return t.data_ptr()
    return _refuse(t, dtype, n, name)


def _refuse(t, dtype, n, name):
    if dtype is not None and t.dtype is not dtype:
        why = f"holds {t.dtype}, not {dtype}"
    elif t.numel() < n:
        why = f"has {t.numel()} elements, needs {n}"
    elif not t.is_contiguous():
        why = "is not contiguous"
    else:
        why = "is not on the GPU"
    raise FlowBlockError(FB_E_INVAL, f"{name} {why}")


def _octets(t, n, name):
    """The pointer of t, n bytes in elements of one byte, whatever they are called."""
    if t.nbytes == n == t.numel() and t.is_contiguous() and t.is_cuda:
        return t.data_ptr()
    if t.element_size() != 1:
        raise FlowBlockError(FB_E_INVAL, f"{name} holds {t.dtype}, not bytes")
    if t.numel() != n:
        raise FlowBlockError(FB_E_INVAL, f"{name} has {t.numel()} bytes, not {n}")
    return _refuse(t, None, n, name)


def _space(ws, name):
    """The pointer of a workspace; the library compares its size."""
    if ws.is_contiguous() and ws.is_cuda:
        return ws.data_ptr()
    return _refuse(ws, None, 0, name)


def make_norm_shape(D, dtype, gate="none", eps=1e-6, res_scale=1.0):
    if not isinstance(dtype, int):
        dtype = FB_BF16 if str(dtype) in ("bf16", "torch.bfloat16") else FB_F32
    return fb_norm_shape(D, dtype, GATES[gate] if isinstance(gate, str) else gate, eps,
                         res_scale)


def fb_residual_norm(y, h, gate, w_post, w_pre, h_out, n_out, pack, shape, stream=None):
    """u = rms(y) w_post, h_out = h + a g u, n_out = rms(h_out) w_pre on the live
    rows; any of y, gate, w_post, w_pre, h_out, n_out may be None as the header says.
    All are of the shape's type."""
    t, D = _type(shape.dtype), shape.D
    n = pack.row_cap * D
    if gate is not None:
        gate = _dense(gate, t, {1: D, 2: pack.B * D, 3: n}.get(shape.gate, 0), "gate")
    _check(lib().fb_residual_norm(_dense(y, t, n, "y"), _dense(h, t, n, "h"), gate,
                                  _dense(w_post, t, D, "w_post"), _dense(w_pre, t, D, "w_pre"),
                                  _dense(h_out, t, n, "h_out"), _dense(n_out, t, n, "n_out"),
                                  pack.handle, shape, _stream(stream)))


def fb_mx4_linear(x, codes, scales, pack, y, stream=None):
    """x bf16 [row_cap, K]; codes uint8 [N, K/2] (E2M1, element 2i in the low half
    of byte i); scales uint8 [N, K/32] (E8M0); y [row_cap, N], bf16 or fp32."""
    N, K, rows = codes.shape[0], x.shape[-1], pack.row_cap
    _check(lib().fb_mx4_linear(_dense(x, _type(FB_BF16), rows * K, "x"),
                               _octets(codes, N * K // 2, "codes"),
                               _octets(scales, N * K // 32, "scales"), N, K, pack.handle,
                               _dense(y, y.dtype, rows * N, "y"), _dtype_code(y),
                               _stream(stream)))


def make_rules(params=None, bias_start=None, bias_id=None, bias_val=None, masks=None,
               row_mask=None):
    """params fp32 [B, 4] (repetition, presence, frequency, 0); bias_start int32
    [B+1] with bias_id int32 and bias_val fp32; masks int32 [n_masks,
    ceil(V/32)] with row_mask int32 [row_cap].  Keeps its tensors alive."""
    import torch
    n_bias = 0 if bias_id is None else bias_id.numel()
    n_masks = 0 if masks is None else masks.numel() // max(1, masks.shape[-1])
    word = torch.int32 if masks is None or masks.dtype is not torch.uint32 else torch.uint32
    r = fb_logit_rules(_dense(params, torch.float32, 0, "params"),
                       _dense(bias_start, torch.int32, 0, "bias_start"),
                       _dense(bias_id, torch.int32, 0, "bias_id"),
                       _dense(bias_val, torch.float32, n_bias, "bias_val"),
                       _dense(masks, word, 0, "masks"),
                       _dense(row_mask, torch.int32, 0, "row_mask"), n_bias, n_masks)
    r.tensors = (params, bias_start, bias_id, bias_val, masks, row_mask)
    return r


def _rules(rules, pack, V=0):
    """The rules, which fit the pack and, for the calls that read masks,
    the vocabulary."""
    params, start, _, _, masks, row_mask = rules.tensors
    if params is not None and params.numel() < 4 * pack.B:
        _refuse(params, None, 4 * pack.B, "params")
    if start is not None and start.numel() <= pack.B:
        _refuse(start, None, pack.B + 1, "bias_start")
    if V and masks is not None:
        if masks.shape[-1] != (V + 31) // 32:
            raise FlowBlockError(FB_E_INVAL, f"masks have rows of {masks.shape[-1]} words, not "
                                             f"the {(V + 31) // 32} of {V} tokens")
        if row_mask is not None and row_mask.numel() < pack.row_cap:
            _refuse(row_mask, None, pack.row_cap, "row_mask")
    return rules


def fb_rules_workspace_bytes(pack, V):
    return int(lib().fb_rules_workspace_bytes(pack.handle, V))


def fb_rules_build(rules, st, tokens, V, pack, ws, stream=None):
    B, T_max = pack.B, tokens.shape[-1]
    if st is not None and st.nbytes < 32 * B:
        raise FlowBlockError(FB_E_INVAL, f"st has {st.nbytes} bytes, needs {32 * B}")
    _check(lib().fb_rules_build(_rules(rules, pack), st if st is None else _space(st, "st"),
                                _dense(tokens, _type(FB_I32), B * T_max, "tokens"), T_max, V,
                                pack.handle, _space(ws, "ws"), ws.nbytes, _stream(stream)))


def fb_vocab_reduce_rules(logits, pack, rules, rules_ws, upd_ws, conf=None, argmax=None,
                          stream=None):
    """The reduction under the rules lands in upd_ws for fb_denoise_apply, and, if
    given, in conf fp32 and argmax int32 [row_cap]."""
    V, rows = logits.shape[-1], pack.row_cap
    _check(lib().fb_vocab_reduce_rules(_dense(logits, logits.dtype, rows * V, "logits"), V,
                                       _dtype_code(logits), pack.handle,
                                       _rules(rules, pack, V), _space(rules_ws, "rules_ws"),
                                       rules_ws.nbytes, _space(upd_ws, "upd_ws"), upd_ws.nbytes,
                                       _dense(conf, _type(FB_F32), rows, "conf"),
                                       _dense(argmax, _type(FB_I32), rows, "argmax"),
                                       _stream(stream)))


def fb_logits_rules(logits, out, pack, rules, rules_ws, stream=None):
    V, t = logits.shape[-1], logits.dtype
    n = pack.row_cap * V
    _check(lib().fb_logits_rules(_dense(logits, t, n, "logits"), _dense(out, t, n, "out"), V,
                                 _dtype_code(logits), pack.handle, _rules(rules, pack, V),
                                 _space(rules_ws, "rules_ws"), rules_ws.nbytes,
                                 _stream(stream)))


# ---------------------------------------------------- the quantised cache
# Checked as the tail's calls are: type, density and size of every tensor against the
# pack, the shape and the cache.
def make_rotary(freq, axis, pairing="halves"):
    """Pair j turns by positions[axis[j]][row] * freq[j]; its elements are j and
    len(freq) + j ("halves") or 2j and 2j + 1 ("neighbours")."""
    n = len(freq)
    if n != len(axis) or not 1 <= n <= 64:
        raise FlowBlockError(FB_E_INVAL, f"{n} frequencies and {len(axis)} axes: need 1 .. 64 of "
                                         "each")
    if min(axis) < 0 or max(axis) > 7:
        raise FlowBlockError(FB_E_INVAL, "axes are 0 .. 7")
    r = fb_rotary(max(axis) + 1, n, PAIRINGS[pairing] if isinstance(pairing, str) else pairing)
    r.freq[:n], r.axis[:n] = freq, axis
    return r


def rotary_sections(head_dim, sections, base=10000.0):
    """(freq, axis) of make_rotary for heads whose first sections[0] pairs turn by axis 0,
    the next sections[1] by axis 1, and so on, pair j at base^(-2j/head_dim).  (A model that
    turns part of a head may count its frequencies over that width: pass it as head_dim.)"""
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    return [base ** (-2.0 * j / head_dim) for j in range(len(axis))], axis


def fb_rotary_axes(q_in, q_out, k_in, k_out, positions, pack, shape, rotary, stream=None):
    """q [row_cap, Hq, d] and k [row_cap, Hkv, d] (either pair may be None) turned by
    positions int32 [n_axes, row_cap]."""
    t, row = _type(shape.dtype), pack.row_cap * shape.head_dim
    nq, nk = row * shape.Hq, row * shape.Hkv
    _check(lib().fb_rotary_axes(_dense(q_in, t, nq, "q_in"), _dense(q_out, t, nq, "q_out"),
                                _dense(k_in, t, nk, "k_in"), _dense(k_out, t, nk, "k_out"),
                                _dense(positions, _type(FB_I32), rotary.n_axes * pack.row_cap,
                                       "positions"),
                                pack.handle, shape, rotary, _stream(stream)))


def make_mx_cache(format, k_codes, k_scales, v_codes, v_scales):
    """format FB_MX4 or FB_MX8; codes uint8 [num_pages, Hkv, page_size, d * format / 8],
    scales uint8 [num_pages, Hkv, page_size, d / 32].  Keeps its tensors alive."""
    t = (k_codes, k_scales, v_codes, v_scales)
    names = ("k_codes", "k_scales", "v_codes", "v_scales")
    c = fb_mx_cache(*(_octets(x, x.numel(), n) for x, n in zip(t, names)), format)
    c.tensors = t
    return c


def _mx_cache(cache, page_table, pack, shape):
    """The cache and the page table's pointer, which fit the shape."""
    slots = shape.num_pages * shape.Hkv * shape.page_size
    sizes = (slots * shape.head_dim * cache.format // 8, slots * (shape.head_dim // 32))
    for t, n, name in zip(cache.tensors, sizes * 2, ("k_codes", "k_scales", "v_codes", "v_scales")):
        if t is not None and t.numel() < n:
            _refuse(t, None, n, name)
    return cache, _dense(page_table, _type(FB_I32), pack.B * shape.max_pages, "page_table")


def fb_mx_write_window_kv(k_new, v_new, cache, page_table, pack, shape, stream=None):
    t, n = _type(shape.dtype), pack.row_cap * shape.Hkv * shape.head_dim
    _check(lib().fb_mx_write_window_kv(_dense(k_new, t, n, "k_new"), _dense(v_new, t, n, "v_new"),
                                       *_mx_cache(cache, page_table, pack, shape), pack.handle,
                                       shape, _stream(stream)))


def fb_mx_read_kv(cache, page_table, spans, k_out, v_out, pack, shape, stream=None):
    """spans int32 [B, 2]: first position and count; k_out, v_out [B, T, Hkv, d] (one may
    be None)."""
    out = k_out if k_out is not None else v_out
    T = 0 if out is None else out.shape[1]
    if k_out is not None and v_out is not None and v_out.shape[1] != T:
        raise FlowBlockError(FB_E_INVAL, f"k_out {tuple(k_out.shape)} and v_out "
                                         f"{tuple(v_out.shape)} differ")
    t, n = _type(shape.dtype), pack.B * T * shape.Hkv * shape.head_dim
    _check(lib().fb_mx_read_kv(*_mx_cache(cache, page_table, pack, shape),
                               _dense(spans, _type(FB_I32), 2 * pack.B, "spans"), T,
                               _dense(k_out, t, n, "k_out"), _dense(v_out, t, n, "v_out"),
                               pack.handle, shape, _stream(stream)))


def fb_mx_attention_workspace_bytes(pack, shape):
    return int(lib().fb_mx_attention_workspace_bytes(pack.handle, shape))


def fb_mx_attention(q, cache, page_table, pack, shape, out, ws, stream=None):
    t, n = _type(shape.dtype), pack.row_cap * shape.Hq * shape.head_dim
    _check(lib().fb_mx_attention(_dense(q, t, n, "q"), *_mx_cache(cache, page_table, pack, shape),
                                 pack.handle, shape, _dense(out, t, n, "out"), _space(ws, "ws"),
                                 ws.nbytes, _stream(stream)))


# ------------------------------------------------------ multi-step loop
def make_model(seed, levels):
    m = fb_synth_model()
    m.seed = seed
    for i, a in enumerate(levels):
        m.levels[i] = a
    return m


def fb_synth_embed(pack, shape, seed, q, k_new, v_new, stream=None):
    _check(lib().fb_synth_embed(pack.ref(), ctypes.byref(shape), seed, _ptr(q),
                                _ptr(k_new), _ptr(v_new), _stream(stream)))


def fb_synth_logits(st, tokens, pack, model, pred, logits, stream=None):
    """st int32 [B, 8]; tokens int32 [B, T_max]; pred int32 [row_cap, 2];
    logits [row_cap, V] (bf16 or fp32)."""
    _check(lib().fb_synth_logits(_ptr(st), _ptr(tokens), tokens.shape[-1],
                                 pack.ref(), ctypes.byref(model), logits.shape[-1],
                                 _dtype_code(logits), _ptr(pred), _ptr(logits),
                                 _stream(stream)))


def fb_decode_loop(args, max_steps, check_every, use_graph, stream=None):
    """args: an fb_loop_args (its pointer fields must stay alive for the call).
    Returns (steps enqueued, done)."""
    steps, done = ctypes.c_int(), ctypes.c_int()
    _check(lib().fb_decode_loop(ctypes.byref(args), max_steps, check_every,
                                1 if use_graph else 0, ctypes.byref(steps),
                                ctypes.byref(done), _stream(stream)))
    return steps.value, bool(done.value)


# ------------------------------------------------------------- HBM probes
def fb_hbm_read_probe(src, out, stream=None):
    """Stream `src` (a contiguous device tensor) once; out: int32 or uint32
    tensor of FB_PROBE_BLOCKS words receiving per-workgroup XORs."""
    _check(lib().fb_hbm_read_probe(_ptr(src), src.numel() * src.element_size(),
                                   _ptr(out), _stream(stream)))


def fb_hbm_copy_probe(src, dst, stream=None):
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < nbytes:
        raise FlowBlockError(FB_E_INVAL, "dst smaller than src")
    _check(lib().fb_hbm_copy_probe(_ptr(src), _ptr(dst), nbytes, _stream(stream)))
