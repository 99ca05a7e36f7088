"""ctypes binding of libdlm (include/dlm.h): argument marshalling only.

Every function has the name of the C entry point it calls.  Device buffers are
torch tensors (torch only allocates memory and supplies the stream); host
arrays are plain int lists.  A missing library is an error: there is no
fallback path.
"""
import ctypes as C
import functools
import os
import struct

import torch  # loaded first so that libdlm binds to the HIP runtime torch already opened

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdlm.so")
_lib = None

DLM_F32, DLM_BF16 = 0, 1
ERRORS = {-1: "DLM_EINVAL", -2: "DLM_ESHAPE", -3: "DLM_ECAPACITY", -4: "DLM_ENOMEM", -5: "DLM_EHIP"}
_ECAPACITY = -3


class DlmError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


class dlm_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "mask_id", "dtype")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class dlm_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("wqkv", C.POINTER(C.c_void_p)), ("wo", C.POINTER(C.c_void_p)),
                ("w_gate_up", C.POINTER(C.c_void_p)), ("w_down", C.POINTER(C.c_void_p)), ("norm1", C.POINTER(C.c_void_p)),
                ("norm2", C.POINTER(C.c_void_p)), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class dlm_q8_weight(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "k", "gated")] + [("data", C.c_void_p)]


class dlm_kv8_cache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_slots", "max_len", "n_kv", "head_dim", "format")] + [("data", C.c_void_p)]


_I32P = C.POINTER(C.c_int32)


class dlm_step_desc(C.Structure):
    _fields_ = [("n_seqs", C.c_int32)] + [(n, _I32P) for n in
                ("slot", "row_offsets", "span_start", "commit_len", "kl_first", "kl_count", "save_first", "save_count", "tok_start", "suffix_len")] + \
               [(n, C.c_void_p) for n in ("tokens", "logits", "max_logit", "lse", "entropy", "kl", "conf", "argmax")]


class dlm_boundary_params(C.Structure):
    _fields_ = [("lam", C.c_float), ("l_min", C.c_int32), ("smooth_radius", C.c_int32), ("norm_mode", C.c_int32), ("rule", C.c_int32)]


class dlm_select_params(C.Structure):
    _fields_ = [("tau_low", C.c_float), ("tau_high", C.c_float), ("gamma", C.c_float), ("mode", C.c_int32)]


EXPORTS = ["dlm_last_error", "dlm_model_create", "dlm_model_destroy", "dlm_state_create", "dlm_state_destroy", "dlm_state_reset",
           "dlm_state_kv_len", "dlm_step", "block_boundary", "select_parallel", "dlm_vocab_stats_workspace", "dlm_vocab_stats",
           "dlm_gemm_nt", "dlm_attention", "dlm_profile_enable", "dlm_profile_read", "dlm_probe_hbm_read", "dlm_probe_mfma",
           "dlm_state_fuse_stats", "dlm_vocab_stats_static", "dlm_plan_attention",
           "dlm_plan_vocab_stats", "dlm_plan_gemm", "dlm_qk_norm_rope", "dlm_kv8_bytes", "dlm_kv8_write", "dlm_kv8_read",
           "dlm_kv8_attention_workspace", "dlm_kv8_attention", "dlm_q8_rows", "dlm_add_norm_q8", "dlm_q8_weight_bytes",
           "dlm_q8_weight_pack", "dlm_q8_gemm_workspace", "dlm_q8_gemm", "dlm_plan_q8_gemm"]


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2604_15750_amd.build` (there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        L.dlm_last_error.restype = C.c_char_p
        L.dlm_vocab_stats_workspace.restype = C.c_size_t
        L.dlm_vocab_stats_workspace.argtypes = [C.c_int]
        L.dlm_model_create.argtypes = [C.POINTER(dlm_config), C.POINTER(dlm_weights), C.c_void_p, C.POINTER(C.c_void_p)]
        L.dlm_model_destroy.argtypes = [C.c_void_p]
        L.dlm_model_destroy.restype = None
        L.dlm_state_create.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_void_p)]
        L.dlm_state_destroy.argtypes = [C.c_void_p]
        L.dlm_state_destroy.restype = None
        L.dlm_state_reset.argtypes = [C.c_void_p, C.c_int]
        L.dlm_state_kv_len.argtypes = [C.c_void_p, C.c_int]
        L.dlm_step.argtypes = [C.c_void_p, C.POINTER(dlm_step_desc), C.c_void_p]
        # (the host arrays and parameters of the two decisions are void pointers: they are handed over as bytes)
        L.block_boundary.argtypes = [C.c_void_p] * 5 + [C.c_int] + [C.c_void_p] * 5
        L.select_parallel.argtypes = [C.c_void_p, C.c_int, C.c_int] + [C.c_void_p] * 7 + \
                                     [C.c_int, C.c_int, C.c_void_p, C.c_int] + [C.c_void_p] * 4
        L.dlm_vocab_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int] + [C.c_void_p] * 7 + \
                                     [C.c_size_t, C.c_void_p]
        L.dlm_vocab_stats_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int] + [C.c_void_p] * 7
        L.dlm_gemm_nt.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p]
        L.dlm_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p] + [C.c_int] * 6 + [C.c_void_p]
        L.dlm_probe_hbm_read.argtypes = [C.c_void_p, C.c_size_t, C.c_int, C.POINTER(C.c_double), C.c_void_p]
        L.dlm_probe_mfma.argtypes = [C.c_int, C.POINTER(C.c_double), C.c_void_p]
        L.dlm_plan_attention.argtypes = [C.c_int] * 4 + [_I32P]
        L.dlm_plan_vocab_stats.argtypes = [C.c_int] * 3 + [_I32P]
        L.dlm_plan_gemm.argtypes = [C.c_int] * 4 + [_I32P]
        L.dlm_state_fuse_stats.argtypes = [C.c_void_p, C.c_int]
        L.dlm_profile_enable.argtypes = [C.c_void_p, C.c_uint]
        L.dlm_profile_read.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int]
        L.dlm_qk_norm_rope.argtypes = [C.c_void_p, C.c_int64] + [C.c_int] * 5 + [C.c_void_p] * 2 + [C.c_float] * 2 + [C.c_void_p] * 2 + [C.c_int64, C.c_void_p]
        L.dlm_kv8_bytes.argtypes = [C.c_int] * 4
        L.dlm_kv8_bytes.restype = C.c_size_t
        for f in (L.dlm_kv8_write, L.dlm_kv8_read):
            f.argtypes = [C.c_void_p] * 3 + [C.c_int64, C.c_int] + [C.c_void_p] * 3 + [C.c_int, C.c_void_p]
        L.dlm_kv8_attention_workspace.argtypes = [C.c_int] * 3
        L.dlm_kv8_attention_workspace.restype = C.c_size_t
        L.dlm_kv8_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int, C.c_int] + [C.c_void_p] * 3 + \
                                       [C.c_int, C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.dlm_q8_rows.argtypes = [C.c_void_p, C.c_int64] + [C.c_int] * 3 + [C.c_void_p, C.c_int64] + [C.c_void_p] * 2
        L.dlm_add_norm_q8.argtypes = [C.c_void_p, C.c_int64] + [C.c_int] * 3 + [C.c_void_p, C.c_int64] * 2 + [C.c_int, C.c_void_p, C.c_float, C.c_void_p, C.c_int64] + \
                                     [C.c_void_p] * 2
        L.dlm_plan_q8_gemm.argtypes = [C.c_int] * 4 + [_I32P]
        L.dlm_q8_weight_bytes.argtypes = [C.c_int] * 3
        L.dlm_q8_weight_bytes.restype = C.c_size_t
        L.dlm_q8_weight_pack.argtypes = [C.c_void_p] * 2 + [C.c_int64] + [C.c_void_p] * 2
        L.dlm_q8_gemm_workspace.argtypes = [C.c_int] * 4
        L.dlm_q8_gemm_workspace.restype = C.c_size_t
        L.dlm_q8_gemm.argtypes = [C.c_void_p] * 2 + [C.c_int64, C.c_void_p, C.c_int, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


def _check(rc):
    if rc < 0:
        raise DlmError(rc, lib().dlm_last_error().decode())
    return rc


def _ptr(t):
    return None if t is None else t.data_ptr()


def _enough(v, n):
    """The library reads n entries of a host array, whatever its length: one that is shorter is refused here."""
    if v is not None and len(v) < n:
        raise ValueError(f"a host array of {len(v)} entries where the call reads {n}")
    return v


def _ints(v, n=0):
    if v is None:
        return None
    k = len(v)
    if k < n:
        _enough(v, n)
    return (C.c_int32 * k)(*map(int, v))


# The two decisions are bound by what their calls cost the host: plain arguments go through a small extension (csrc/decisions_py.c),
# any others through ctypes, host arrays and parameters as bytes (marshalling alone 3.8 and 6.1 us with ctypes structs and a format
# string per array, 2.7 and 4.8 as bytes, 1.2 and 2.1 through the extension; both decisions of one sequence x 8 rows 11.8 -> 10.0 us a
# pass, of 16 x 64 12.3 -> 10.3, on another box 10.3 -> 9.6 and 10.7 -> 9.7).
@functools.lru_cache(maxsize=None)
def _decisions():
    """The extension, bound to the library; None where it has not been built."""
    try:
        from . import _decisions as m
    except ImportError:
        return None
    L = lib()
    m.bind(C.cast(L.block_boundary, C.c_void_p).value, C.cast(L.select_parallel, C.c_void_p).value, torch.float32, torch.bfloat16)
    return m


@functools.lru_cache(maxsize=64)
def _int_packer(n):
    return struct.Struct(f"{n}i").pack


def _packed(v):
    """A host array as bytes (a ctypes array of 16 takes 2.1 us, this 0.3).  What struct does not take as a 32-bit integer goes
    the way of _ints."""
    if v is None:
        return None
    try:
        return _int_packer(len(v))(*v)
    except (struct.error, TypeError, OverflowError):
        return bytes(_ints(v))


_pack_boundary, _pack_select = struct.Struct("f4i").pack, struct.Struct("3fi").pack


def _params(pack, cls, v):
    """A parameter struct as bytes; values that struct does not take go the way of the ctypes struct."""
    try:
        return pack(*v)
    except (struct.error, TypeError, OverflowError):
        return bytes(cls(*v))


# what torch.cuda.current_stream() asks, without its Stream object (0.3 us against 2.7); a private name, so the public way stays beside it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


_DTYPE_CODES = {torch.float32: DLM_F32, torch.bfloat16: DLM_BF16}


def dtype_code(t):
    return _DTYPE_CODES[t if isinstance(t, torch.dtype) else t.dtype]


class Model:
    """dlm_model_create / dlm_model_destroy.  cfg: dict of inputs.model_config; W: dict of device tensors.
    weight_copies=False sets DLM_W_STEPS=0 for the call: no step-major second copies of the layer matrices."""

    def __init__(self, cfg, W, weight_copies=True):
        self.cfg = dict(cfg)
        dt = DLM_F32 if cfg["dtype"] == "f32" else DLM_BF16
        c = dlm_config(cfg["n_layers"], cfg["d_model"], cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["d_ffn"],
                       cfg["vocab"], cfg["mask_id"], dt, cfg["rms_eps"], cfg["rope_theta"])
        arr = lambda ts: (C.c_void_p * len(ts))(*[t.data_ptr() for t in ts])
        keep = [arr(W[k]) for k in ("wqkv", "wo", "w_gate_up", "w_down", "norm1", "norm2")]
        w = dlm_weights(W["embed"].data_ptr(), *keep, W["final_norm"].data_ptr(), W["lm_head"].data_ptr())
        h = C.c_void_p()
        before = os.environ.get("DLM_W_STEPS")
        if not weight_copies:
            os.environ["DLM_W_STEPS"] = "0"
        try:
            _check(lib().dlm_model_create(C.byref(c), C.byref(w), _stream(), C.byref(h)))
        finally:
            if not weight_copies:
                if before is None:
                    del os.environ["DLM_W_STEPS"]
                else:
                    os.environ["DLM_W_STEPS"] = before
        torch.cuda.current_stream().synchronize()  # the caller may now drop W
        self.handle = h
        self.torch_dtype = torch.float32 if dt == DLM_F32 else torch.bfloat16

    def close(self):
        if self.handle and lib is not None:  # at interpreter shutdown the module's globals may already be gone
            lib().dlm_model_destroy(self.handle)
            self.handle = None

    __del__ = close


class State:
    """dlm_state_create / dlm_state_destroy."""

    def __init__(self, model, max_seqs, max_seq_len, max_rows, max_lookahead):
        self.model = model
        h = C.c_void_p()
        _check(lib().dlm_state_create(model.handle, max_seqs, max_seq_len, max_rows, max_lookahead, C.byref(h)))
        self.handle = h
        self.max_rows = max_rows

    def reset(self, slot):
        _check(lib().dlm_state_reset(self.handle, slot))

    def kv_len(self, slot):
        return _check(lib().dlm_state_kv_len(self.handle, slot))

    def fuse_stats(self, enable):
        """dlm_state_fuse_stats: statistics of qualifying passes from the LM head's epilogue (default) or from the streamed reduction."""
        _check(lib().dlm_state_fuse_stats(self.handle, int(bool(enable))))

    PROFILE_CLASSES = ("gemm_qkv", "gemm_o", "gemm_gate_up", "gemm_down", "gemm_lm_head", "attention", "vocab_stats", "other")

    def profile_enable(self, classes):
        """classes: True (all), False (none) or an iterable of names from PROFILE_CLASSES."""
        if classes is True:
            mask = (1 << len(self.PROFILE_CLASSES)) - 1
        elif not classes:
            mask = 0
        else:
            mask = sum(1 << self.PROFILE_CLASSES.index(c) for c in classes)
        _check(lib().dlm_profile_enable(self.handle, mask))

    def profile_read(self, reset=True):
        """{class name: (milliseconds, launches)} since the last reset."""
        k = len(self.PROFILE_CLASSES)
        ms = (C.c_double * k)()
        n = (C.c_int64 * k)()
        _check(lib().dlm_profile_read(self.handle, k, ms, n, int(reset)))
        return {name: (ms[i], n[i]) for i, name in enumerate(self.PROFILE_CLASSES)}

    def close(self):
        if self.handle and lib is not None:
            lib().dlm_state_destroy(self.handle)
            self.handle = None

    __del__ = close


class StepOutputs:
    """Caller-owned output buffers of dlm_step for up to `rows` rows."""

    def __init__(self, rows, vocab, dtype, device):
        self.logits = torch.empty((rows, vocab), dtype=dtype, device=device)
        f = lambda: torch.empty(rows, dtype=torch.float32, device=device)
        self.max_logit, self.lse, self.entropy, self.kl, self.conf = f(), f(), f(), f(), f()
        self.argmax = torch.empty(rows, dtype=torch.int32, device=device)


def dlm_step(state, tokens, out, row_offsets, span_start, commit_len, tok_start, slot=None, kl_first=None, kl_count=None,
             save_first=None, save_count=None, suffix_len=None):
    """tokens: device int32 tensor; out: StepOutputs; the rest: host int lists (see include/dlm.h)."""
    n = len(span_start)
    keep = [_ints(slot, n), _ints(row_offsets, n + 1)]
    keep += [_ints(v, n) for v in (span_start, commit_len, kl_first, kl_count, save_first, save_count, tok_start, suffix_len)]
    d = dlm_step_desc(n, *keep, tokens.data_ptr(), out.logits.data_ptr(), out.max_logit.data_ptr(), out.lse.data_ptr(),
                      out.entropy.data_ptr(), out.kl.data_ptr(), out.conf.data_ptr(), out.argmax.data_ptr())
    _check(lib().dlm_step(state.handle, C.byref(d), _stream()))


def block_boundary(I, H, win_start, win_len, L_out, lam, l_min, smooth_radius=1, norm_mode=0, rule=0, cold=None, S_out=None,
                   margin_out=None):
    ext = _decisions()
    if ext is not None:
        rc = ext.boundary(I, H, win_start, win_len, cold, L_out, S_out, margin_out, lam, l_min, smooth_radius, norm_mode, rule, _stream())
        if rc is not None:  # (None: not plain arguments, nothing has been called)
            if rc < 0:
                _check(rc)
            return
    n = len(win_start)
    _check(lib().block_boundary(_ptr(I), _ptr(H), _packed(win_start), _packed(_enough(win_len, n)), _packed(_enough(cold, n)), n,
                                _params(_pack_boundary, dlm_boundary_params, (lam, l_min, smooth_radius, norm_mode, rule)), _ptr(L_out),
                                _ptr(S_out), _ptr(margin_out), _stream()))


def select_parallel(logits, lse, conf, argmax, tokens, row_start, tok_start, block_len, mask_id, tau_low, tau_high, gamma, mode,
                    selected_out, n_selected_out, apply_tokens=True, margin_out=None):
    ext = _decisions()
    if ext is not None:
        rc = ext.select(logits, lse, conf, argmax, tokens, row_start, tok_start, block_len, mask_id, tau_low, tau_high, gamma, mode,
                        selected_out, n_selected_out, apply_tokens, margin_out, _stream())
        if rc is not None:
            if rc < 0:
                _check(rc)
            return
    n = len(row_start)
    _check(lib().select_parallel(_ptr(logits), logits.size(-1), dtype_code(logits), _ptr(lse), _ptr(conf), _ptr(argmax), _ptr(tokens),
                                 _packed(row_start), _packed(_enough(tok_start, n)), _packed(_enough(block_len, n)), n, mask_id,
                                 _params(_pack_select, dlm_select_params, (tau_low, tau_high, gamma, mode)), int(apply_tokens),
                                 _ptr(selected_out), _ptr(n_selected_out), _ptr(margin_out), _stream()))


def dlm_vocab_stats(logits, mask_id, prev=None, workspace=None, prev_lse=None):
    rows, vocab = logits.shape
    dev = logits.device
    f = lambda: torch.empty(rows, dtype=torch.float32, device=dev)
    out = dict(max_logit=f(), lse=f(), entropy=f(), kl=f(), conf=f(), argmax=torch.empty(rows, dtype=torch.int32, device=dev))
    if workspace is None:
        workspace = torch.empty(lib().dlm_vocab_stats_workspace(rows), dtype=torch.uint8, device=dev)
    _check(lib().dlm_vocab_stats(_ptr(logits), _ptr(prev), _ptr(prev_lse), rows, vocab, dtype_code(logits), mask_id, _ptr(out["max_logit"]),
                                 _ptr(out["lse"]), _ptr(out["entropy"]), _ptr(out["kl"]), _ptr(out["conf"]), _ptr(out["argmax"]),
                                 _ptr(workspace), workspace.numel(), _stream()))
    return out


def dlm_vocab_stats_static(logits, mask_id, prev=None, out=None, prev_lse=None):
    """dlm_vocab_stats_static: the partial states live in the library's file-scope scratch.  `out`: a dict of preallocated
    output tensors as dlm_vocab_stats returns (so that the call allocates nothing at all); None: new ones."""
    rows, vocab = logits.shape
    dev = logits.device
    if out is None:
        f = lambda: torch.empty(rows, dtype=torch.float32, device=dev)
        out = dict(max_logit=f(), lse=f(), entropy=f(), kl=f(), conf=f(), argmax=torch.empty(rows, dtype=torch.int32, device=dev))
    _check(lib().dlm_vocab_stats_static(_ptr(logits), _ptr(prev), _ptr(prev_lse), rows, vocab, dtype_code(logits), mask_id, _ptr(out["max_logit"]),
                                        _ptr(out["lse"]), _ptr(out["entropy"]), _ptr(out["kl"]), _ptr(out["conf"]), _ptr(out["argmax"]),
                                        _stream()))
    return out


def dlm_gemm_nt(x, w):
    M, K = x.shape
    N = w.shape[0]
    y = torch.empty((M, N), dtype=x.dtype, device=x.device)
    _check(lib().dlm_gemm_nt(_ptr(x), _ptr(w), _ptr(y), M, N, K, dtype_code(x), _stream()))
    return y


def probe_hbm_read(buf, reps=10):
    """GB/s of a plain streaming read of the device tensor `buf` (see include/dlm.h)."""
    out = C.c_double()
    _check(lib().dlm_probe_hbm_read(_ptr(buf), C.c_size_t(buf.numel() * buf.element_size()), reps, C.byref(out), _stream()))
    return out.value


def probe_mfma(reps=5):
    """TFLOP/s of independent half-precision matrix-core products out of registers, on operands of pseudo-random values."""
    out = C.c_double()
    _check(lib().dlm_probe_mfma(reps, C.byref(out), _stream()))
    return out.value


def dlm_attention(q, k, v):
    A, n_q, hd = q.shape
    T, n_kv, _ = k.shape
    out = torch.empty_like(q)
    _check(lib().dlm_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(out), A, T, n_q, n_kv, hd, dtype_code(q), _stream()))
    return out


# ---- the 8-bit KV cache, and what feeds and reads it (include/dlm.h) ---------------------------------------------------------------

KV8_FORMATS = ("e4m3", "i8")


# Calls that need no refusal go through an extension (csrc/kv8_py.cpp); what it declines (None) comes the way below it, which says what it refuses.
@functools.lru_cache(maxsize=None)
def _kv8_calls():
    """The extension, bound to the library; None where it has not been built, or for another torch, whose tensors it would misread."""
    try:
        from . import _kv8 as m
    except ImportError:
        return None
    if getattr(m, "torch_version", None) != str(torch.__version__):
        return None
    L = lib()
    m.bind(*(C.cast(f, C.c_void_p).value for f in (L.dlm_kv8_write, L.dlm_kv8_read, L.dlm_kv8_attention, L.dlm_qk_norm_rope)))
    return m


def _taken(rc):
    """Whether the extension made the call; its error raised."""
    if rc is None:
        return False
    if rc < 0:
        _check(rc)
    return True


def _int32s(name, v, n):
    """A host list as the bytes of 32-bit integers, at least n of them; what is none is refused."""
    if v is None:
        return None
    if len(v) < n:
        raise ValueError(f"{name}: {len(v)} entries where {n} are read")
    try:
        return _int_packer(len(v))(*v)
    except (struct.error, TypeError):
        pass
    whole = [int(x) if not isinstance(x, str) and x == int(x) else None for x in v]
    if any(x is None or not -2**31 <= x < 2**31 for x in whole):
        raise ValueError(f"{name}: {v} are not 32-bit integers")
    return _int_packer(len(v))(*whole)


def _device():
    return torch.cuda.current_device()


def _gpu_of(name, t):
    """The index of the current GPU, which t is on."""
    dev = t.get_device()  # (-1: on none)
    if dev < 0 or dev != _device():
        raise ValueError(f"{name}: not on the current GPU")
    return dev


def _on_gpu(name, t, dev):
    if t.get_device() != dev:
        raise ValueError(f"{name}: not on the current GPU")


def _row_stride(name, t, dev, tail, dtypes):
    """The stride between the rows (first axis) of a tensor on GPU `dev` whose rows are contiguous; tail: their shape, None for any."""
    if t.get_device() != dev:
        raise ValueError(f"{name}: not on the current GPU")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: {t.dtype}, not one of {dtypes}")
    have = t.shape
    if len(have) != len(tail) + 1:
        raise ValueError(f"{name}: {len(have)} dimensions where {len(tail) + 1} are read")
    width, dense = 1, t.is_contiguous()
    strides = None if dense else t.stride()
    for i in range(len(tail), 0, -1):
        n = have[i]
        if tail[i - 1] is not None and tail[i - 1] != n:
            raise ValueError(f"{name}: rows of shape {tuple(have[1:])} where {tail} is read")
        if not dense and strides[i] != width and n != 1:
            raise ValueError(f"{name}: strides {strides}: a row is not contiguous")
        width *= n
    return width if dense or have[0] < 2 else strides[0]


def _vector(name, t, dev, n, dtype):
    if t.get_device() != dev:
        raise ValueError(f"{name}: not on the current GPU")
    if t.dtype is not dtype or t.dim() != 1 or t.size(0) != n or not t.is_contiguous():
        raise ValueError(f"{name}: not a contiguous vector of {n} x {dtype}")


_FLOATS = (torch.float32, torch.bfloat16)


class Kv8Cache:
    """A cache of K and V at 8 bits (dlm_kv8_cache) with its memory: `slots` sequences of up to max_len positions.
    format: "e4m3" or "i8"."""

    def __init__(self, slots, max_len, n_kv, head_dim, format="e4m3", device="cuda"):
        n = lib().dlm_kv8_bytes(slots, max_len, n_kv, head_dim) if all(0 < x < 2**31 for x in (slots, max_len, n_kv, head_dim)) else 0
        if n == 0:
            raise DlmError(-2, f"a cache of {slots} slots x {max_len} positions x {n_kv} heads of {head_dim}")
        self.slots, self.max_len, self.n_kv, self.head_dim, self.format = slots, max_len, n_kv, head_dim, format
        code = KV8_FORMATS.index(format)
        self._data = torch.zeros(n, dtype=torch.uint8, device=device)
        self._desc = dlm_kv8_cache(slots, max_len, n_kv, head_dim, code, self._data.data_ptr())
        self._ref = C.addressof(self._desc)

    @property
    def data(self):
        """The memory (one address for life: to be filled in place, not replaced)."""
        return self._data


def _kv8_spans(cache, k, v, row_offsets, start, slot):
    n, dev, tail = len(start), _gpu_of("k", k), (cache.n_kv, cache.head_dim)
    off = _int32s("row_offsets", row_offsets, n + 1)
    stride = _row_stride("k", k, dev, tail, _FLOATS)
    if _row_stride("v", v, dev, tail, (k.dtype,)) != stride:
        raise ValueError("k and v have different strides between rows")
    rows = k.shape[0]
    if rows != v.shape[0] or row_offsets[n] > rows:
        raise ValueError(f"{rows} rows of k and {v.shape[0]} of v where {row_offsets[n]} are read")
    _on_gpu("cache", cache._data, dev)
    return cache._ref, k.data_ptr(), v.data_ptr(), stride, _DTYPE_CODES[k.dtype], off, _int32s("start", start, n), _int32s("slot", slot, n), n, _stream()


def dlm_kv8_write(cache, k, v, row_offsets, start, slot=None):
    """k, v: device tensors [rows, n_kv, head_dim] (rows may be strided: columns of a wider matrix); the rest: host int lists."""
    ext = _kv8_calls()
    if ext is not None and _taken(ext.span(0, cache._ref, cache._data, k, v, row_offsets, start, slot, _device(), _stream())):
        return
    args = _kv8_spans(cache, k, v, row_offsets, start, slot)
    if k.shape[0]:  # (a tensor without rows has no address)
        _check(lib().dlm_kv8_write(*args))


def dlm_kv8_read(cache, row_offsets, start, slot=None, k=None, v=None, dtype=torch.bfloat16):
    """The values of cached positions, (k, v): into the given tensors [rows, n_kv, head_dim], or into new ones of `dtype`."""
    if (k is None) != (v is None):
        raise ValueError("k and v are given together")
    if k is None:
        if len(row_offsets) <= len(start):
            raise ValueError(f"row_offsets: {len(row_offsets)} entries where {len(start) + 1} are read")
        rows = max(0, int(row_offsets[len(start)]))
        k, v = (torch.empty((rows, cache.n_kv, cache.head_dim), dtype=dtype, device=cache._data.device) for _ in "kv")
    ext = _kv8_calls()
    if ext is not None and _taken(ext.span(1, cache._ref, cache._data, k, v, row_offsets, start, slot, _device(), _stream())):
        return k, v
    args = _kv8_spans(cache, k, v, row_offsets, start, slot)
    if k.shape[0]:
        _check(lib().dlm_kv8_read(*args))
    return k, v


def dlm_kv8_attention(cache, q, row_offsets, n_keys, slot=None, mask=None, out=None, workspace=None):
    """q: device tensor [rows, n_q, head_dim] (rows may be strided); mask: device int32 [rows, words], bits as in include/dlm.h; out:
    contiguous, of q's shape and dtype (None: a new one); workspace: a contiguous device tensor of at least
    dlm_kv8_attention_workspace bytes that nothing else uses meanwhile (None: a new one); the rest: host int lists.  Returns out."""
    ext = _kv8_calls()
    if ext is not None and out is not None:
        # (-1: not for the extension)
        size = 0 if workspace is None else workspace.numel() * workspace.element_size() if workspace.is_contiguous() else -1
        if _taken(ext.attention(cache._ref, cache._data, q, row_offsets, n_keys, slot, mask, out, workspace, size, _device(), _stream())):
            return out
    n, dev = len(n_keys), _gpu_of("q", q)
    stride = _row_stride("q", q, dev, (None, cache.head_dim), _FLOATS)
    rows, n_q, hd = q.shape
    off = _int32s("row_offsets", row_offsets, n + 1)
    packed = int(row_offsets[n])
    if packed > rows:
        raise ValueError(f"{rows} rows of q where {packed} are read")
    if out is None:
        out = torch.empty((rows, n_q, hd), dtype=q.dtype, device=q.device)
    elif _row_stride("out", out, dev, (n_q, hd), (q.dtype,)) != n_q * hd or out.shape[0] != rows:
        raise ValueError("out is not contiguous, or has not q's rows")
    words = 0
    if mask is not None:
        words = mask.shape[-1]
        if _row_stride("mask", mask, dev, (words,), (torch.int32,)) != words or mask.shape[0] < packed or words >= 2**31:
            raise ValueError(f"mask: {tuple(mask.shape)} for {packed} rows, or not contiguous")
    _on_gpu("cache", cache._data, dev)
    if rows == 0:
        return out
    L = lib()
    size = L.dlm_kv8_attention_workspace(packed, n_q, hd)
    if workspace is None:
        workspace = torch.empty(size, dtype=torch.uint8, device=q.device) if size else None
    else:
        _on_gpu("workspace", workspace, dev)
        if not workspace.is_contiguous():
            raise ValueError("workspace is not contiguous")
        size = workspace.numel() * workspace.element_size()
    _check(L.dlm_kv8_attention(cache._ref, q.data_ptr(), stride, out.data_ptr(), _DTYPE_CODES[q.dtype], n_q, off, _int32s("n_keys", n_keys, n),
                               _int32s("slot", slot, n), n, _ptr(mask), words, _ptr(workspace), size, _stream()))
    return out


def dlm_qk_norm_rope(x, positions, n_q, n_kv, head_dim, q_gain=None, k_gain=None, eps=1e-5, theta=10000.0, out=None):
    """x: device tensor [rows, columns] whose first (n_q + n_kv) * head_dim columns are the query and key heads (rows may be
    strided); positions: device int32 [rows]; gains: [head_dim] of x's dtype, or None; out: as x (x itself: in place; None: a new
    tensor of those columns alone).  Returns out."""
    ext = _kv8_calls()
    if ext is not None and out is not None and _taken(ext.rope(x, positions, n_q, n_kv, head_dim, q_gain, k_gain, eps, theta, out, _device(), _stream())):
        return out
    width, dev, dtype = (n_q + n_kv) * head_dim, _gpu_of("x", x), x.dtype
    stride = _row_stride("x", x, dev, (None,), _FLOATS)
    rows, columns = x.shape
    if out is None:
        out = torch.empty((rows, width), dtype=dtype, device=x.device)
    out_stride = stride if out is x else _row_stride("out", out, dev, (None,), (dtype,))
    if rows == 1:  # (a row has no stride: one that holds either, in multiples of 16 bytes)
        stride = out_stride = max(columns, out.shape[1]) + 7 & ~7
    if rows >= 2**31 or min(n_q, n_kv, head_dim) < 0 or columns < width or out.shape[1] < width or out.shape[0] != rows:
        raise ValueError(f"rows of {columns} and {out.shape[1]} columns where {width} are read and written, or not as many rows of out")
    _vector("positions", positions, dev, rows, torch.int32)
    if q_gain is not None:
        _vector("q_gain", q_gain, dev, head_dim, dtype)
    if k_gain is not None:
        _vector("k_gain", k_gain, dev, head_dim, dtype)
    if rows == 0:
        return out
    _check(lib().dlm_qk_norm_rope(x.data_ptr(), stride, rows, n_q, n_kv, head_dim, _DTYPE_CODES[x.dtype], _ptr(q_gain), _ptr(k_gain), eps, theta,
                                  positions.data_ptr(), out.data_ptr(), out_stride, _stream()))
    return out


# ---- linear layers in 8-bit integers (include/dlm.h) ---------------------------------------------------------------------------------

def _matrix(name, t, dev, rows, width, dtypes):
    """The stride between the rows of [rows, width] (None: any); a single row, which has none, gets one that holds it in multiples of 16 bytes."""
    stride = _row_stride(name, t, dev, (width,), dtypes)
    if rows is not None and t.shape[0] != rows:
        raise ValueError(f"{name}: {t.shape[0]} rows where {rows} are read")
    if t.shape[0] == 1:
        step = 16 // t.element_size()
        stride = -(-t.shape[1] // step) * step
    return stride


def _new_rows(rows, width, dtype, device):
    """New rows at a stride of a multiple of 16 bytes."""
    step = 16 // dtype.itemsize
    return torch.empty((rows, -(-width // step) * step), dtype=dtype, device=device)[:, :width]


def _codes(name, t, dev, rows, width):
    """As _matrix, of codes that are read: their rows' bytes up to a multiple of 16 have to be the tensor's memory."""
    stride = _matrix(name, t, dev, rows, width, (torch.int8,))
    width = t.shape[1]
    if width % 16 and t.shape[0]:
        if t.untyped_storage().nbytes() < t.storage_offset() + (t.shape[0] - 1) * stride + -(-width // 16) * 16:
            raise ValueError(f"{name}: the last row's bytes up to a multiple of 16 are not the tensor's memory")
    return stride


# Calls with all their outputs given go through an extension (csrc/q8_py.cpp), as those of the 8-bit cache do.
@functools.lru_cache(maxsize=None)
def _q8_calls():
    """The extension, bound to the library; None where it has not been built, or for another torch, whose tensors it would misread."""
    try:
        from . import _q8 as m
    except ImportError:
        return None
    if getattr(m, "torch_version", None) != str(torch.__version__):
        return None
    L = lib()
    m.bind(*(C.cast(f, C.c_void_p).value for f in (L.dlm_q8_rows, L.dlm_add_norm_q8, L.dlm_q8_gemm)))
    return m


def _code_outputs(x, dev, codes, scale):
    rows, width = x.shape
    if codes is None:
        codes = _new_rows(rows, width, torch.int8, x.device)
    if scale is None:
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    stride = _matrix("codes", codes, dev, rows, width, (torch.int8,))
    _vector("scale", scale, dev, rows, torch.float32)
    return codes, stride, scale


def dlm_q8_rows(x, codes=None, scale=None):
    """Rows in 8-bit integers: x: device tensor [rows, width] (rows may be strided); codes: int8 [rows, width], scale: fp32 [rows] (None: new ones).
    Returns (codes, scale)."""
    ext = _q8_calls()
    if ext is not None and _taken(ext.rows(x, codes, scale, _device(), _stream())):
        return codes, scale
    dev = _gpu_of("x", x)
    stride = _matrix("x", x, dev, None, None, _FLOATS)
    codes, code_stride, scale = _code_outputs(x, dev, codes, scale)
    rows, width = x.shape
    if rows and max(rows, width) < 2**31:
        _check(lib().dlm_q8_rows(x.data_ptr(), stride, rows, width, _DTYPE_CODES[x.dtype], codes.data_ptr(), code_stride, scale.data_ptr(), _stream()))
    elif rows:
        raise ValueError(f"x: {rows} rows of {width}")
    return codes, scale


def dlm_add_norm_q8(x, gain, residual=None, h=None, eps=1e-5, codes=None, scale=None):
    """The residual's addition, RMSNorm and the rows in 8-bit integers: x: device tensor [rows, width]; gain: [width] of x's dtype; residual: [rows,
    width] of x's dtype or fp32, or None (no addition); h: residual + x, of the residual's dtype (None: a new tensor; the residual or x itself: in place);
    codes, scale: as dlm_q8_rows.  Returns (codes, scale, h); h is x where there is no residual."""
    ext = _q8_calls()
    if ext is not None and _taken(ext.norm(x, gain, residual, h, eps, codes, scale, _device(), _stream())):
        return codes, scale, x if residual is None else h
    dev = _gpu_of("x", x)
    stride = _matrix("x", x, dev, None, None, _FLOATS)
    rows, width = x.shape
    _vector("gain", gain, dev, width, x.dtype)
    r_stride = h_stride = h_code = 0
    if residual is not None:
        r_stride = _matrix("residual", residual, dev, rows, width, (torch.float32, x.dtype))
        if h is None:
            h = _new_rows(rows, width, residual.dtype, x.device)
        h_stride = _matrix("h", h, dev, rows, width, (residual.dtype,))
        h_code = _DTYPE_CODES[residual.dtype]
    elif h is not None:
        raise ValueError("h is given without a residual")
    codes, code_stride, scale = _code_outputs(x, dev, codes, scale)
    if rows and max(rows, width) < 2**31:
        _check(lib().dlm_add_norm_q8(x.data_ptr(), stride, rows, width, _DTYPE_CODES[x.dtype], _ptr(residual), r_stride, _ptr(h), h_stride, h_code, gain.data_ptr(), eps,
                                     codes.data_ptr(), code_stride, scale.data_ptr(), _stream()))
    elif rows:
        raise ValueError(f"x: {rows} rows of {width}")
    return codes, scale, x if residual is None else h


class Q8Weight:
    """A weight in 8-bit integers (dlm_q8_weight) with its memory, packed from codes (int8 [n, k]) and scales (fp32 [n]), one per output channel.  gated: the
    first n / 2 channels are the gate's, the others the up channels, and a product with it has n / 2 outputs."""

    def __init__(self, codes, scale, gated=False):
        dev = _gpu_of("codes", codes)
        stride = _codes("codes", codes, dev, None, None)
        self.n, self.k = codes.shape
        self.gated = bool(gated)
        size = lib().dlm_q8_weight_bytes(self.n, self.k, int(self.gated)) if max(self.n, self.k) < 2**31 else 0
        if size == 0:
            raise DlmError(-2, f"a weight of {self.n} x {self.k}" + (", gated" if gated else ""))
        _vector("scale", scale, dev, self.n, torch.float32)
        self._data = torch.empty(size, dtype=torch.uint8, device=codes.device)
        self._desc = dlm_q8_weight(self.n, self.k, int(self.gated), self._data.data_ptr())
        self._ref = C.addressof(self._desc)
        _check(lib().dlm_q8_weight_pack(self._ref, codes.data_ptr(), stride, scale.data_ptr(), _stream()))

    @classmethod
    def quantise(cls, weight, gated=False):
        """Of a weight [n, k] in fp32 or bf16, each channel quantised as dlm_q8_rows does."""
        return cls(*dlm_q8_rows(weight), gated=gated)

    @property
    def outputs(self):
        return self.n // 2 if self.gated else self.n

    @property
    def data(self):
        """The memory (one address for life)."""
        return self._data

    def workspace(self, rows):
        """A new workspace for products of up to `rows` rows, or None where they need none."""
        size = lib().dlm_q8_gemm_workspace(rows, self.n, self.k, int(self.gated)) if 0 < rows < 2**31 else 0
        return torch.empty(size, dtype=torch.uint8, device=self._data.device) if size else None


def dlm_q8_gemm(weight, x, x_scale, out=None, dtype=torch.bfloat16, workspace=None):
    """The product of rows of codes (int8 [rows, k], scales fp32 [rows]) with a Q8Weight: into out [rows, weight.outputs] (fp32 or bf16; rows may be strided), or
    into a new tensor of `dtype`; workspace: one of weight.workspace(as many rows or more) that nothing else uses meanwhile (None: a new one of what this launch
    needs, if it needs one).  Returns out."""
    ext, refused = _q8_calls(), False
    if ext is not None:
        rc = ext.gemm(weight._ref, weight._data, x, x_scale, out, workspace, _device(), _stream())
        refused = rc == _ECAPACITY and workspace is None
        if not refused and _taken(rc):
            return out
    dev = _gpu_of("x", x)
    stride = _codes("x", x, dev, None, weight.k)
    rows = x.shape[0]
    _vector("x_scale", x_scale, dev, rows, torch.float32)
    if out is None:
        out = _new_rows(rows, weight.outputs, dtype, x.device)
    out_stride = _matrix("out", out, dev, rows, weight.outputs, _FLOATS)
    _on_gpu("weight", weight._data, dev)
    if rows >= 2**31:
        raise ValueError(f"x: {rows} rows")
    if rows == 0:
        return out

    def call(ws):
        size = 0 if ws is None else ws.numel() * ws.element_size()
        return lib().dlm_q8_gemm(weight._ref, x.data_ptr(), stride, x_scale.data_ptr(), rows, out.data_ptr(), out_stride, _DTYPE_CODES[out.dtype], _ptr(ws), size, _stream())

    if workspace is not None:
        _on_gpu("workspace", workspace, dev)
        if not workspace.is_contiguous():
            raise ValueError("workspace is not contiguous")
        _check(call(workspace))
        return out
    # Most launches need none.  One that does is refused with nothing launched, for the price of its plan, which is asked for then; weight.workspace looks through the
    # plans of fewer rows too, for the most that any of them needs (a call into a new out 20 us of host time instead of 62 at 2822 x 512 x 16000; at 2822 x 3584 x 18944
    # 12 instead of 31, and no workspace instead of 63 MiB)
    rc = _ECAPACITY if refused else call(None)
    if rc == _ECAPACITY:
        plan = (C.c_int32 * 6)()
        known = lib().dlm_plan_q8_gemm(rows, weight.n, weight.k, int(weight.gated), plan) == 0
        rc = call(torch.empty(plan[5] << 10, dtype=torch.uint8, device=x.device) if known and plan[5] else None)  # (None: too large a call, refused again)
    _check(rc)
    return out


def plan_attention(max_seq_rows, n_seqs, n_q, head_dim):
    """How the attention of such a pass is launched (include/dlm.h): wavefronts of a workgroup, workgroups that share a head's
    output dims, 16-query tiles of a workgroup."""
    out = (C.c_int32 * 3)()
    _check(lib().dlm_plan_attention(max_seq_rows, n_seqs, n_q, head_dim, out))
    return dict(zip(("waves", "shares", "tiles"), out))


def plan_vocab_stats(rows, vocab, dtype):
    """How the streamed vocabulary reduction is launched (include/dlm.h): threads of a workgroup, chunks of a row."""
    out = (C.c_int32 * 2)()
    _check(lib().dlm_plan_vocab_stats(rows, vocab, dtype_code(dtype), out))
    return dict(zip(("threads", "chunks"), out))


EPILOGUES = ("direct", "qkv", "swiglu", "resid", "sum", "stats")


def plan_gemm(M, N, K, epilogue):
    """How a bf16 model's product is launched (include/dlm.h); epilogue: a name from EPILOGUES."""
    out = (C.c_int32 * 7)()
    _check(lib().dlm_plan_gemm(M, N, K, EPILOGUES.index(epilogue), out))
    return dict(zip(("kernel", "rows", "cols", "splits", "k_parts", "workgroups", "ssq_parts"), (("skinny", "mid", "macro")[out[0]], *out[1:])))


def plan_q8_gemm(rows, n, k, gated=False):
    """How a product of 8-bit rows with a Q8Weight [n, k] is launched (include/dlm.h)."""
    out = (C.c_int32 * 6)()
    _check(lib().dlm_plan_q8_gemm(rows, n, k, int(gated), out))
    return dict(zip(("kernel", "rows", "cols", "splits", "workgroups", "workspace_kib"), (("streamed", "tiled", "banded")[out[0]], *out[1:])))
