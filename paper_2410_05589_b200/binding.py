"""Thin ctypes binding of the C ABI in include/ps.h.

Argument marshalling only: torch tensors supply device memory and the CUDA stream; every
step of the path runs in the library's kernels.  There is no CPU fallback: if the shared
library is missing or no CUDA device is present, calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import threading
import warnings

import torch

from . import build as _build

PS_OK = 0
STATUS_NAMES = {0: "PS_OK", -1: "PS_ERR_INVALID_ARG", -2: "PS_ERR_UNSUPPORTED", -3: "PS_ERR_CAPACITY",
                -4: "PS_ERR_CUDA", -5: "PS_ERR_TIMEOUT", -6: "PS_ERR_NONFINITE"}
PS_DTYPE_F32, PS_DTYPE_BF16 = 0, 1
PS_FLAG_FC_BIAS, PS_FLAG_UNFUSED_KERNELS, PS_FLAG_MMA_SYNC_GEMM, PS_FLAG_NO_FC = 1, 2, 4, 8
PS_FLAG_STAGE_LAUNCHES = 16
PS_MAX_BATCH, PS_MAX_MASKS, PS_MAX_TOP_N = 128, 15, 8

WEIGHT_NAMES = (
    "embed", "mask_embed", "mask_feat", "w_fc", "b_fc", "g_in", "w_q", "w_k", "w_v", "w_o",
    "g_post", "w_gate", "w_up", "w_down", "g_final", "w_lm",
)

EXPORTS = (
    "ps_workspace_bytes", "ps_init", "ps_kv_append", "ps_draft_step", "ps_verify", "ps_round_host",
    "ps_kv_len", "ps_kv_reset", "ps_kv_export", "ps_kv_import", "ps_poll", "ps_launch_count",
    "ps_last_error", "ps_destroy", "ps_philox_fill", "ps_profile", "ps_profile_read",
    "ps_verify_static", "ps_debug_buffer", "ps_verify_tree", "ps_draft_step_sampled", "ps_group_forward",
    "ps_build_tree", "ps_debug_wait_expires", "ps_debug_check_guards", "ps_debug_late_copy",
    "ps_debug_gemm_plan", "ps_debug_append_pass_rows",
    "ps_group_attn_workspace_bytes", "ps_group_attn", "ps_group_attn_backward", "ps_lm_loss_workspace_bytes",
    "ps_lm_loss", "ps_lm_loss_backward", "ps_embed_rows", "ps_embed_rows_workspace_bytes", "ps_embed_rows_backward",
    "ps_train_poll", "ps_debug_train_wait_expires",
)


class PsError(RuntimeError):
    def __init__(self, status: int, text: str = ""):
        self.status = status
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {text}")


class ps_config(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("hidden", C.c_int), ("n_heads", C.c_int), ("n_kv_heads", C.c_int),
        ("head_dim", C.c_int), ("ffn", C.c_int), ("vocab", C.c_int), ("k_masks", C.c_int),
        ("max_batch", C.c_int), ("max_ctx", C.c_int), ("rope_base", C.c_float),
        ("rms_eps", C.c_float), ("flags", C.c_int),
    ]


class ps_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES]


class ps_group_attn_args(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("B", C.c_int), ("k_masks", C.c_int), ("n_heads", C.c_int), ("n_kv_heads", C.c_int),
        ("head_dim", C.c_int), ("n_ctx", C.POINTER(C.c_int)), ("n_groups", C.POINTER(C.c_int)), ("scale", C.c_float),
        ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
        ("ldq", C.c_size_t), ("ldk", C.c_size_t), ("ldv", C.c_size_t),
        ("out", C.c_void_p), ("ldo", C.c_size_t), ("lse", C.c_void_p), ("dout", C.c_void_p), ("lddo", C.c_size_t),
        ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p),
        ("lddq", C.c_size_t), ("lddk", C.c_size_t), ("lddv", C.c_size_t),
    ]


_lib = None


def load_library(path: str | None = None) -> C.CDLL:
    """Loads libps_b200.so (building it with nvcc if the in-tree copy is stale)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or _build.build()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path}: the CUDA library is not built")
    lib = C.CDLL(path)
    vp, ip = C.c_void_p, C.POINTER(C.c_int)
    lib.ps_workspace_bytes.restype = C.c_size_t
    lib.ps_workspace_bytes.argtypes = [C.POINTER(ps_config)]
    lib.ps_init.argtypes = [C.POINTER(vp), C.POINTER(ps_config), C.POINTER(ps_weights), vp, C.c_size_t, vp]
    lib.ps_kv_append.argtypes = [vp, C.c_int, ip, ip, ip, vp, vp, vp]
    lib.ps_draft_step.argtypes = [vp, C.c_int, ip, vp, vp, C.c_int, vp, vp, vp, vp, vp, vp, vp]
    lib.ps_verify.argtypes = [vp, C.c_int, C.c_int, C.c_int, vp, vp, vp, C.c_float, C.c_uint64,
                              C.c_uint64, vp, vp, vp, vp]
    lib.ps_round_host.argtypes = [vp, C.c_int, ip, vp, vp, vp, C.c_float, C.c_uint64, C.c_uint64,
                                  vp, vp, vp, vp]
    lib.ps_draft_step_sampled.argtypes = [vp, C.c_int, ip, vp, vp, C.c_float, C.c_uint64, C.c_uint64, vp,
                                          C.c_int, vp, vp, vp, vp, vp, vp, vp]
    lib.ps_group_forward.argtypes = [vp, C.c_int, C.c_int, vp, vp, C.c_int, vp, vp, vp, vp, vp, vp, vp]
    lib.ps_verify_tree.argtypes = [vp, C.c_int, C.c_int, ip, vp, vp, vp, C.c_float, C.c_uint64, C.c_uint64,
                                   vp, vp, vp, vp, vp]
    lib.ps_build_tree.argtypes = [vp, C.c_int, C.c_int, ip, ip, vp, C.c_int, vp, vp, vp]
    lib.ps_debug_wait_expires.argtypes = [vp, C.c_longlong, vp]
    lib.ps_debug_check_guards.argtypes = [vp, vp, ip]
    lib.ps_debug_gemm_plan.argtypes = [C.c_int, C.c_int, C.c_int, ip, C.c_int, C.c_int, C.c_int, C.c_size_t, C.c_int, ip]
    lib.ps_debug_append_pass_rows.argtypes = [C.POINTER(ps_config), C.c_int, C.c_int, C.c_int]
    lib.ps_debug_late_copy.argtypes = [vp, vp, vp, C.c_size_t, C.c_int, vp]
    lib.ps_kv_len.argtypes = [vp, C.c_int, ip]
    lib.ps_kv_reset.argtypes = [vp, C.c_int]
    lib.ps_kv_export.argtypes = [vp, C.c_int, vp, vp, vp]
    lib.ps_kv_import.argtypes = [vp, C.c_int, C.c_int, vp, vp, vp]
    lib.ps_poll.argtypes = [vp, vp]
    lib.ps_launch_count.restype = C.c_longlong
    lib.ps_launch_count.argtypes = [vp]
    lib.ps_last_error.restype = C.c_char_p
    lib.ps_last_error.argtypes = [vp]
    lib.ps_destroy.restype = None
    lib.ps_destroy.argtypes = [vp]
    lib.ps_philox_fill.argtypes = [C.POINTER(C.c_uint32), vp, vp, C.c_int, vp]
    lib.ps_profile.argtypes = [vp, C.c_int]
    lib.ps_profile_read.argtypes = [vp, C.c_int, C.c_char_p, C.POINTER(C.c_float), ip, ip]
    lib.ps_debug_buffer.argtypes = [vp, C.c_char_p, C.POINTER(vp), C.POINTER(C.c_size_t)]
    lib.ps_verify_static.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, vp, vp, vp, C.c_float,
                                     C.c_uint64, C.c_uint64, vp, vp, vp, vp, C.c_char_p, C.c_size_t, vp]
    ga, sz, f = C.POINTER(ps_group_attn_args), C.c_size_t, C.c_float
    lib.ps_group_attn_workspace_bytes.restype = sz
    lib.ps_group_attn_workspace_bytes.argtypes = [ga, C.c_int]
    lib.ps_group_attn.argtypes = [ga, vp, sz, vp, C.c_char_p, sz, vp]
    lib.ps_group_attn_backward.argtypes = [ga, vp, sz, vp, C.c_char_p, sz, vp]
    lib.ps_lm_loss_workspace_bytes.restype = sz
    lib.ps_lm_loss_workspace_bytes.argtypes = [C.c_int] * 5
    lib.ps_lm_loss.argtypes = [C.c_int] * 4 + [vp, sz, vp, vp, vp, vp, vp, sz, vp, C.c_char_p, sz, vp]
    lib.ps_lm_loss_backward.argtypes = [C.c_int] * 4 + [vp, sz, vp, vp, vp, vp, vp, sz, vp, vp, sz, vp, C.c_char_p, sz, vp]
    lib.ps_embed_rows.argtypes = [C.c_int] * 5 + [vp, vp, vp, f, vp, sz, C.c_char_p, sz, vp]
    lib.ps_embed_rows_workspace_bytes.restype = sz
    lib.ps_embed_rows_workspace_bytes.argtypes = [C.c_int] * 5
    lib.ps_embed_rows_backward.argtypes = [C.c_int] * 5 + [vp, f, vp, sz, vp, vp, vp, sz, C.c_char_p, sz, vp]
    lib.ps_train_poll.argtypes = [vp]
    lib.ps_debug_train_wait_expires.argtypes = [C.c_int, C.c_longlong, vp, vp]
    _lib = lib
    return lib


# What a call costs on the host matters where its kernels take some ten microseconds: addresses and streams go
# to the library as plain integers (its argument types make pointers of them), and the current stream is asked
# for by its handle, without an object around it (13B, append of 12 rows and export of the four
# slots, which the host bounds: 73.8 -> 60.9 us).
def _dptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _iarr(xs):
    return (C.c_int * len(xs))(*map(int, xs))


# (not public names: a torch may lack them; the public ways take 0.3 us longer a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


_CUDA = torch.device("cuda")   # (the current device, like the name)


def workspace_bytes(cfg: ps_config) -> int:
    return load_library().ps_workspace_bytes(C.byref(cfg))


def philox_fill(key, ctr: torch.Tensor) -> torch.Tensor:
    """out[i] = Philox-4x32-10(key, ctr[i]); ctr: CUDA int32/uint32 tensor [n][4]."""
    lib = load_library()
    out = torch.empty_like(ctr)
    k = (C.c_uint32 * 2)(int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF)
    rc = lib.ps_philox_fill(k, _dptr(ctr), _dptr(out), ctr.shape[0], _stream())
    if rc != PS_OK:
        raise PsError(rc)
    return out


def verify_static(draft_tokens: torch.Tensor, draft_logits, target_logits: torch.Tensor,
                  temperature: float, seed: int, offset: int, out: dict, nonfinite_flag=None,
                  stream=None) -> dict:
    """ps_verify_static: the acceptance test for callers that may not allocate device memory.

    Needs no Drafter and no workspace; the kernel's scratch is a fixed array inside the library
    (one per GPU, shared by all calls, so calls must not overlap on a GPU).  ``out`` must hold the
    caller's preallocated CUDA int32 tensors ``accept_len`` [B], ``out_tokens`` [B][n_draft+1] and
    ``n_out`` [B]: this wrapper allocates nothing either.
    """
    lib = load_library()
    B, n_draft = draft_tokens.shape
    _, n_target, vocab = target_logits.shape
    err = C.create_string_buffer(256)
    rc = lib.ps_verify_static(vocab, B, n_draft, n_target, _dptr(draft_tokens), _dptr(draft_logits),
                              _dptr(target_logits), float(temperature), seed, offset,
                              _dptr(out["accept_len"]), _dptr(out["out_tokens"]), _dptr(out["n_out"]),
                              _dptr(nonfinite_flag), err, 256, _stream(stream))
    if rc != PS_OK:
        raise PsError(rc, err.value.decode())
    return out


# ---- training operators ----------------------------------------------------------------------------
# Functions of tensors: they need no Drafter.  Outputs and workspaces are allocated per call on the stream the
# call runs on (pass ``out`` to reuse outputs), so that calls on several streams and captured graphs share nothing.
# ``status`` (int32, zeroed by the caller) has bit 1 set by a call whose device-side wait expired; calls without one report to
# a word of the device that ``train_poll`` reads.  With ``stream`` the caller orders it behind what wrote the inputs, and keeps
# inputs and outputs until it is done with them, as with any tensor that is used on another stream than its own.
# Outputs are values without an autograd graph: a step calls the ``*_backward`` functions, itself or from a
# torch.autograd.Function whose forward and backward call the two.
_DTYPE_CODE = {torch.float32: PS_DTYPE_F32, torch.bfloat16: PS_DTYPE_BF16}


class _Here:
    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_HERE = _Here()


def _on(device, stream):
    """Makes the tensors' device current, and ``stream`` where one is given (of that device: a stream of another one would
    make that one current, and the kernels would run there)."""
    if stream is None:
        if device.index == _device():
            return _HERE
    elif stream.device != device:
        _refuse(f"the stream is of another device ({stream.device}) than the tensors ({device})")
    both = contextlib.ExitStack()
    both.enter_context(torch.cuda.device(device))
    if stream is not None:
        both.enter_context(torch.cuda.stream(stream))
    return both


# (What these checks cost on the host is most of what a small call costs: texts are put together only for a refusal, a
# tensor's device is read once.)
def _refuse(text):
    raise PsError(-1, text)


def _tensors(device, *tensors, dtype=None):
    """CUDA tensors of one device (None is skipped) and, with ``dtype``, of one type."""
    for t in tensors:
        if t is not None:
            if t.device != device:
                _refuse(f"tensors lie on different devices ({device}, {t.device})")
            if dtype is not None and t.dtype != dtype:
                _refuse(f"expected {dtype}, got {t.dtype}")


def _first(t, name):
    """Device and type code of the tensor that sets both."""
    if not t.is_cuda:
        _refuse("tensors must lie on a CUDA device")
    code = _DTYPE_CODE.get(t.dtype)
    if code is None:
        _refuse(f"{name}: float32 or bfloat16, got {t.dtype}")
    return t.device, code


def _rows(t, width, name):
    """Row stride in elements of a tensor of rows that are dense; a view of a wider buffer may have a larger one."""
    if t.is_contiguous() and t.numel() == width * t.shape[0]:
        return width
    shape, stride = t.shape, t.stride()
    w = 1
    for i in range(len(shape) - 1, 0, -1):
        if shape[i] != 1 and stride[i] != w:
            _refuse(f"{name}: rows must be dense")
        w *= shape[i]
    if w != width:
        _refuse(f"{name}: rows of {w} values, expected {width}")
    if shape[0] <= 1:
        return width
    if stride[0] < width:
        _refuse(f"{name}: rows overlap")
    return stride[0]


_err = threading.local()


def _op(fn, *args):
    try:
        err = _err.text
    except AttributeError:
        err = _err.text = C.create_string_buffer(256)
    rc = fn(*args, err, 256, _stream())
    if rc != PS_OK:
        raise PsError(rc, err.value.decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scratch(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None   # (0: the call says why)


def _values_only(name, *tensors):
    """Says so where autograd would stop at the outputs without a word (not within a Function, nor under no_grad)."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                warnings.warn(f"{name}: the outputs carry no autograd graph although an input requires a gradient; call {name}_backward "
                              f"for it, from a torch.autograd.Function for instance (under torch.no_grad() this is not said)",
                              stacklevel=3)
                return


def _check_status(status, device):
    if status is not None:
        _tensors(device, status, dtype=torch.int32)
        if status.numel() < 1:
            _refuse("status [1] int32")


def train_poll(device=None) -> int:
    """ps_train_poll: waits for the device's current stream and returns (and clears) what calls there without ``status`` have
    reported: PS_OK, or PS_ERR_TIMEOUT if a bounded wait of any of them expired, whose outputs are not to be used."""
    with torch.cuda.device(device):
        return load_library().ps_train_poll(_stream())


def _dense_like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _group_args(q, k, v, n_ctx, n_groups, k_masks, scale):
    device, code = _first(q, "q")
    _tensors(device, k, v, dtype=q.dtype)
    qs, ks = q.shape, k.shape
    if len(qs) != 3 or len(ks) != 3 or ks != v.shape or ks[2] != qs[2]:
        _refuse("q [rows][n_heads][head_dim], k and v [rows][n_kv_heads][head_dim]")
    if len(n_ctx) != len(n_groups):
        _refuse("n_ctx and n_groups have one entry per sequence")
    rows = sum(n_groups) * (k_masks + 1)
    if qs[0] != rows or ks[0] != rows + sum(n_ctx):
        _refuse("the rows do not add up to the sequences")
    d = qs[2]
    wq, wk = qs[1] * d, ks[1] * d
    a = ps_group_attn_args(code, len(n_ctx), k_masks, qs[1], ks[1], d, _iarr(n_ctx), _iarr(n_groups),
                           d ** -0.5 if scale is None else scale, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                           _rows(q, wq, "q"), _rows(k, wk, "k"), _rows(v, wk, "v"), None, wq, None, None, wq, None, None, None,
                           wq, wk, wk)
    return a, device, wq, wk


def _check_lse(lse, q):
    if lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (q.shape[1], q.shape[0]):
        _refuse("lse [n_heads][rows] float32")


def group_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, n_ctx, n_groups, k_masks: int, scale=None,
                    out: dict | None = None, status=None, stream=None) -> dict:
    """ps_group_attn: attention under the mask of parallel groups.

    q [group rows][n_heads][head_dim]; k, v [context and group rows][n_kv_heads][head_dim], float32 or bfloat16, views
    with a larger row stride allowed; n_ctx, n_groups: host lists, one entry per sequence; scale: head_dim ** -0.5 by
    default.  Returns ``out`` (like q) and ``lse`` [n_heads][group rows] float32, without an autograd graph; ``out`` may carry
    them preallocated.
    """
    _values_only("group_attention", q, k, v)
    a, device, wq, _ = _group_args(q, k, v, n_ctx, n_groups, k_masks, scale)
    lib = load_library()
    with _on(device, stream):
        o = out if out is not None else {}
        if "out" not in o:
            o["out"] = _dense_like(q)
        if "lse" not in o:
            o["lse"] = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=device)
        y, lse = o["out"], o["lse"]
        _tensors(device, y, dtype=q.dtype)
        _tensors(device, lse)
        _check_status(status, device)
        _check_lse(lse, q)
        if y.shape != q.shape:
            _refuse("out has another shape than q")
        a.out, a.lse, a.ldo = y.data_ptr(), lse.data_ptr(), _rows(y, wq, "out")
        n = lib.ps_group_attn_workspace_bytes(C.byref(a), 0)
        ws = _scratch(n, device)
        _op(lib.ps_group_attn, C.byref(a), _ptr(ws), n, _ptr(status))
    return o


def group_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                             lse: torch.Tensor, n_ctx, n_groups, k_masks: int, scale=None, grads: dict | None = None,
                             status=None, stream=None) -> dict:
    """ps_group_attn_backward: ``dq``, ``dk``, ``dv`` (like q, k, v) from dout, with out and lse of the forward call.
    ``grads`` may carry them preallocated, as views of wider buffers too."""
    a, device, wq, wk = _group_args(q, k, v, n_ctx, n_groups, k_masks, scale)
    lib = load_library()
    with _on(device, stream):
        o = grads if grads is not None else {}
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            if name not in o:
                o[name] = _dense_like(like)
            elif o[name].shape != like.shape:
                _refuse(f"{name} has another shape than its tensor")
        dq, dk, dv = o["dq"], o["dk"], o["dv"]
        _tensors(device, dout, out, dq, dk, dv, dtype=q.dtype)
        _tensors(device, lse)
        _check_status(status, device)
        _check_lse(lse, q)
        if dout.shape != q.shape or out.shape != q.shape:
            _refuse("dout and out have the shape of q")
        a.out, a.lse, a.dout = out.data_ptr(), lse.data_ptr(), dout.data_ptr()
        a.ldo, a.lddo = _rows(out, wq, "out"), _rows(dout, wq, "dout")
        a.dq, a.dk, a.dv = dq.data_ptr(), dk.data_ptr(), dv.data_ptr()
        a.lddq, a.lddk, a.lddv = _rows(dq, wq, "dq"), _rows(dk, wk, "dk"), _rows(dv, wk, "dv")
        n = lib.ps_group_attn_workspace_bytes(C.byref(a), 1)
        ws = _scratch(n, device)
        _op(lib.ps_group_attn_backward, C.byref(a), _ptr(ws), n, _ptr(status))
    return o


def _loss_args(x, w, labels):
    device, code = _first(x, "x")
    _tensors(device, w, dtype=x.dtype)
    _tensors(device, labels)
    xs, wsh = x.shape, w.shape
    if len(xs) != 2 or len(wsh) != 2 or wsh[1] != xs[1] or not w.is_contiguous():
        _refuse("x [rows][hidden], w [vocab][hidden] dense")
    if labels.dtype != torch.int32 or not labels.is_contiguous() or tuple(labels.shape) != (xs[0],):
        _refuse("labels [rows] int32")
    return device, (code, xs[0], xs[1], wsh[0])


def _check_rows_of_floats(labels, **tensors):
    for name, t in tensors.items():
        if t.dtype != torch.float32 or not t.is_contiguous() or t.shape != labels.shape:
            _refuse(f"{name} [rows] float32")


def lm_loss(x: torch.Tensor, w: torch.Tensor, labels: torch.Tensor, out: dict | None = None, status=None,
            stream=None) -> dict:
    """ps_lm_loss: softmax cross entropy of the logits x w^T, which never exist as a whole.

    x [rows][hidden] (a view with a larger row stride allowed), w [vocab][hidden], float32 or bfloat16; labels [rows]
    int32, any value outside the vocabulary (-100) for rows that count for nothing.  Returns ``loss`` and ``lse``
    [rows] float32, 0 for those rows, without an autograd graph."""
    _values_only("lm_loss", x, w)
    device, size = _loss_args(x, w, labels)
    lib = load_library()
    with _on(device, stream):
        o = out if out is not None else {}
        for name in ("loss", "lse"):
            if name not in o:
                o[name] = torch.empty(x.shape[0], dtype=torch.float32, device=device)
        loss, lse = o["loss"], o["lse"]
        _tensors(device, loss, lse)
        _check_status(status, device)
        _check_rows_of_floats(labels, loss=loss, lse=lse)
        n = lib.ps_lm_loss_workspace_bytes(*size, 0)
        ws = _scratch(n, device)
        _op(lib.ps_lm_loss, *size, x.data_ptr(), _rows(x, x.shape[1], "x"), w.data_ptr(), labels.data_ptr(), loss.data_ptr(),
            lse.data_ptr(), _ptr(ws), n, _ptr(status))
    return o


def lm_loss_backward(x: torch.Tensor, w: torch.Tensor, labels: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                     want_dx: bool = True, want_dw: bool = True, grads: dict | None = None, status=None,
                     stream=None) -> dict:
    """ps_lm_loss_backward: ``dx`` (like x) and ``dw`` (like w) from dloss [rows] float32, the gradient of the caller's
    scalar with respect to each row's loss (1 / rows that count, for their mean), and lse of the forward call.
    ``grads`` may carry them preallocated."""
    device, size = _loss_args(x, w, labels)
    lib = load_library()
    with _on(device, stream):
        o = grads if grads is not None else {}
        for name, like, want in (("dx", x, want_dx), ("dw", w, want_dw)):
            if want and name not in o:
                o[name] = _dense_like(like)
        dx, dw = o.get("dx") if want_dx else None, o.get("dw") if want_dw else None
        _tensors(device, dx, dw, dtype=x.dtype)
        _tensors(device, lse, dloss)
        _check_status(status, device)
        _check_rows_of_floats(labels, lse=lse, dloss=dloss)
        if dx is not None and dx.shape != x.shape:
            _refuse("dx has another shape than x")
        if dw is not None and (dw.shape != w.shape or not dw.is_contiguous()):
            _refuse("dw like w, dense")
        n = lib.ps_lm_loss_workspace_bytes(*size, 1)
        ws = _scratch(n, device)
        _op(lib.ps_lm_loss_backward, *size, x.data_ptr(), _rows(x, x.shape[1], "x"), w.data_ptr(), labels.data_ptr(), lse.data_ptr(),
            dloss.data_ptr(), _ptr(dx), x.shape[1] if dx is None else _rows(dx, x.shape[1], "dx"), _ptr(dw), _ptr(ws), n, _ptr(status))
    return o


def embed_rows(ids: torch.Tensor, table: torch.Tensor, mask_rows=None, scale: float = 1.0, out=None,
               stream=None) -> torch.Tensor:
    """ps_embed_rows: scaled rows of table [vocab][hidden] (ids below vocab) and of mask_rows [k_masks][hidden] (ids from
    vocab on); any other id gives a row of zeros.  ids [rows] int32; ``out`` [rows][hidden] may be a view with a
    larger row stride, such as the embedding half of the fc layer's input.  The result carries no autograd graph."""
    _values_only("embed_rows", table, mask_rows)
    device, code = _first(table, "table")
    _tensors(device, mask_rows, out, dtype=table.dtype)
    _tensors(device, ids)
    if table.dim() != 2 or not table.is_contiguous() or ids.dim() != 1 or ids.dtype != torch.int32 or not ids.is_contiguous():
        _refuse("table [vocab][hidden] dense, ids [rows] int32")
    V, H = table.shape
    if mask_rows is not None and (mask_rows.dim() != 2 or mask_rows.shape[1] != H or not mask_rows.is_contiguous()):
        _refuse("mask_rows [k_masks][hidden] dense")
    lib = load_library()
    with _on(device, stream):
        if out is None:
            out = torch.empty((ids.shape[0], H), dtype=table.dtype, device=device)
        elif tuple(out.shape) != (ids.shape[0], H):
            _refuse("out [rows][hidden]")
        _op(lib.ps_embed_rows, code, ids.shape[0], H, V, 0 if mask_rows is None else mask_rows.shape[0], ids.data_ptr(),
            table.data_ptr(), _ptr(mask_rows), scale, out.data_ptr(), _rows(out, H, "out"))
    return out


def embed_rows_backward(ids: torch.Tensor, dout: torch.Tensor, vocab: int, k_masks: int = 0, scale: float = 1.0,
                        want_table: bool = True, want_mask: bool = True, grads: dict | None = None, stream=None) -> dict:
    """ps_embed_rows_backward: ``d_table`` [vocab][hidden] and ``d_mask`` [k_masks][hidden], the scaled sums of the rows of
    dout [rows][hidden] per id, zeros for ids without a row.  ``grads`` may carry them preallocated."""
    device, code = _first(dout, "dout")
    _tensors(device, ids)
    if dout.dim() != 2 or ids.dtype != torch.int32 or not ids.is_contiguous() or tuple(ids.shape) != (dout.shape[0],):
        _refuse("dout [rows][hidden], ids [rows] int32")
    n_rows, H = dout.shape
    lib = load_library()
    with _on(device, stream):
        o = grads if grads is not None else {}
        got = []
        for name, n, want in (("d_table", vocab, want_table), ("d_mask", k_masks, want_mask and k_masks > 0)):
            t = None
            if want:
                if name not in o:
                    o[name] = torch.empty((n, H), dtype=dout.dtype, device=device)
                t = o[name]
                _tensors(device, t, dtype=dout.dtype)
                if tuple(t.shape) != (n, H) or not t.is_contiguous():
                    _refuse(f"{name} [{n}][hidden] dense")
            got.append(t)
        n = lib.ps_embed_rows_workspace_bytes(code, n_rows, H, vocab, k_masks)
        ws = _scratch(n, device)
        _op(lib.ps_embed_rows_backward, code, n_rows, H, vocab, k_masks, ids.data_ptr(), scale, dout.data_ptr(),
            _rows(dout, H, "dout"), _ptr(got[0]), _ptr(got[1]), _ptr(ws), n)
    return o


class Drafter:
    """One ps_ctx: a drafter with its KV caches on the current CUDA device.

    ``weights`` maps the names of ps_weights to CUDA tensors (float32 for dtype 0, bfloat16
    for dtype 1); the workspace is a torch uint8 tensor owned by this object.
    """

    def __init__(self, *, dtype: int, hidden: int, n_heads: int, n_kv_heads: int, head_dim: int,
                 ffn: int, vocab: int, k_masks: int, max_batch: int, max_ctx: int,
                 weights: dict, rope_base: float = 10000.0, rms_eps: float = 1e-5, flags: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2410_05589_b200 needs a CUDA device; there is no CPU path")
        self.lib = load_library()
        if weights.get("b_fc") is not None:
            flags |= PS_FLAG_FC_BIAS
        self.cfg = ps_config(dtype, hidden, n_heads, n_kv_heads, head_dim, ffn, vocab, k_masks,
                             max_batch, max_ctx, rope_base, rms_eps, flags)
        self.torch_dtype = torch.float32 if dtype == PS_DTYPE_F32 else torch.bfloat16
        self.weights = {}
        w = ps_weights()
        for n in WEIGHT_NAMES:
            t = weights.get(n)
            if t is not None:
                assert t.dtype == self.torch_dtype and t.is_cuda, n
                t = t.contiguous()
                self.weights[n] = t
                setattr(w, n, t.data_ptr())
        nbytes = self.lib.ps_workspace_bytes(C.byref(self.cfg))
        if nbytes == 0:
            raise PsError(-2, "configuration rejected by ps_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=_CUDA)
        h = C.c_void_p()
        rc = self.lib.ps_init(C.byref(h), C.byref(self.cfg), C.byref(w), _dptr(self.workspace),
                              nbytes, _stream())
        if rc != PS_OK:
            raise PsError(rc, "ps_init")
        self.h = h
        self.rows = k_masks + 1

    def close(self):
        if getattr(self, "h", None):
            self.lib.ps_destroy(self.h)
            self.h = None

    def __del__(self):
        self.close()

    def _check(self, rc):
        if rc != PS_OK:
            raise PsError(rc, (self.lib.ps_last_error(self.h) or b"").decode())

    # ---- cache -------------------------------------------------------------------------
    def kv_len(self, slot: int) -> int:
        n = C.c_int()
        self._check(self.lib.ps_kv_len(self.h, slot, C.byref(n)))
        return n.value

    def kv_reset(self, slot: int) -> None:
        self._check(self.lib.ps_kv_reset(self.h, slot))

    def kv_append(self, seq_slot, n_new, hidden: torch.Tensor, tokens: torch.Tensor, stream=None):
        off = [0]
        for n in n_new:
            off.append(off[-1] + int(n))
        self._check(self.lib.ps_kv_append(self.h, len(seq_slot), _iarr(seq_slot), _iarr(n_new),
                                          _iarr(off), _dptr(hidden), _dptr(tokens), _stream(stream)))

    def kv_export(self, slot: int):
        n = self.kv_len(slot)
        w = self.cfg.n_kv_heads * self.cfg.head_dim
        K = torch.empty((n, w), dtype=self.torch_dtype, device=_CUDA)
        V = torch.empty((n, w), dtype=self.torch_dtype, device=_CUDA)
        self._check(self.lib.ps_kv_export(self.h, slot, _dptr(K), _dptr(V), _stream()))
        return K, V

    def kv_import(self, slot: int, K: torch.Tensor, V: torch.Tensor):
        self._check(self.lib.ps_kv_import(self.h, slot, K.shape[0], _dptr(K), _dptr(V), _stream()))

    # ---- the hot path ------------------------------------------------------------------
    def draft_step(self, seq_slot, hidden_last: torch.Tensor, token_last: torch.Tensor, top_n: int = 1,
                   want_logits: bool = True, want_feat: bool = False, out: dict | None = None,
                   stream=None) -> dict:
        """ps_draft_step.  ``out`` may carry preallocated output tensors to reuse."""
        B, R, V, H = len(seq_slot), self.rows, self.cfg.vocab, self.cfg.hidden
        o = out if out is not None else {}
        dev = _CUDA
        if "row_max" not in o:
            o["top_ids"] = torch.empty((B, R, max(top_n, 1)), dtype=torch.int32, device=dev)
            o["top_logit"] = torch.empty((B, R, max(top_n, 1)), dtype=torch.float32, device=dev)
            o["row_max"] = torch.empty((B, R), dtype=torch.float32, device=dev)
            o["row_lse"] = torch.empty((B, R), dtype=torch.float32, device=dev)
            o["logits"] = torch.empty((B, R, V), dtype=torch.float32, device=dev) if want_logits else None
            o["feat"] = torch.empty((B, R, H), dtype=torch.float32, device=dev) if want_feat else None
        self._check(self.lib.ps_draft_step(
            self.h, B, _iarr(seq_slot), _dptr(hidden_last), _dptr(token_last), top_n,
            _dptr(o["top_ids"]), _dptr(o["top_logit"]), _dptr(o["row_max"]), _dptr(o["row_lse"]),
            _dptr(o.get("logits")), _dptr(o.get("feat")), _stream(stream)))
        return o

    def group_forward(self, slot: int, hidden: torch.Tensor, tokens: torch.Tensor, top_n: int = 1,
                      want_logits: bool = True, want_feat: bool = False, stream=None) -> dict:
        """ps_group_forward: the group-wise training layout, forward only.  hidden [n][H], tokens
        [n] int32; outputs shaped [n][k+1]..."""
        n, R, V, H = tokens.shape[0], self.rows, self.cfg.vocab, self.cfg.hidden
        dev = _CUDA
        o = {"top_ids": torch.empty((n, R, max(top_n, 1)), dtype=torch.int32, device=dev),
             "top_logit": torch.empty((n, R, max(top_n, 1)), dtype=torch.float32, device=dev),
             "row_max": torch.empty((n, R), dtype=torch.float32, device=dev),
             "row_lse": torch.empty((n, R), dtype=torch.float32, device=dev),
             "logits": torch.empty((n, R, V), dtype=torch.float32, device=dev) if want_logits else None,
             "feat": torch.empty((n, R, H), dtype=torch.float32, device=dev) if want_feat else None}
        self._check(self.lib.ps_group_forward(
            self.h, slot, n, _dptr(hidden), _dptr(tokens), top_n, _dptr(o["top_ids"]), _dptr(o["top_logit"]),
            _dptr(o["row_max"]), _dptr(o["row_lse"]), _dptr(o["logits"]), _dptr(o["feat"]), _stream(stream)))
        return o

    def draft_step_sampled(self, seq_slot, hidden_last: torch.Tensor, token_last: torch.Tensor,
                           temperature: float, seed: int, offset: int, top_n: int = 1,
                           want_logits: bool = True, want_feat: bool = False, out: dict | None = None,
                           stream=None) -> dict:
        """ps_draft_step_sampled: ps_draft_step plus ``sampled`` [B][k+1] int32, one token per row
        drawn from softmax(logits / temperature)."""
        B, R, V, H = len(seq_slot), self.rows, self.cfg.vocab, self.cfg.hidden
        o = out if out is not None else {}
        dev = _CUDA
        if "row_max" not in o:
            o["top_ids"] = torch.empty((B, R, max(top_n, 1)), dtype=torch.int32, device=dev)
            o["top_logit"] = torch.empty((B, R, max(top_n, 1)), dtype=torch.float32, device=dev)
            o["row_max"] = torch.empty((B, R), dtype=torch.float32, device=dev)
            o["row_lse"] = torch.empty((B, R), dtype=torch.float32, device=dev)
            o["logits"] = torch.empty((B, R, V), dtype=torch.float32, device=dev) if want_logits else None
            o["feat"] = torch.empty((B, R, H), dtype=torch.float32, device=dev) if want_feat else None
        if "sampled" not in o:
            o["sampled"] = torch.empty((B, R), dtype=torch.int32, device=dev)
        self._check(self.lib.ps_draft_step_sampled(
            self.h, B, _iarr(seq_slot), _dptr(hidden_last), _dptr(token_last), float(temperature), seed, offset,
            _dptr(o["sampled"]), top_n, _dptr(o["top_ids"]), _dptr(o["top_logit"]), _dptr(o["row_max"]),
            _dptr(o["row_lse"]), _dptr(o.get("logits")), _dptr(o.get("feat")), _stream(stream)))
        return o

    def verify(self, draft_tokens: torch.Tensor, draft_logits, target_logits: torch.Tensor,
               temperature: float, seed: int, offset: int, out: dict | None = None, stream=None) -> dict:
        """ps_verify.  draft_tokens [B][n_draft] int32, target_logits [B][n_target][V] float32."""
        B, n_draft = draft_tokens.shape
        n_target = target_logits.shape[1]
        assert target_logits.shape[2] == self.cfg.vocab and target_logits.dtype == torch.float32
        o = out if out is not None else {}
        if "accept_len" not in o:
            o["accept_len"] = torch.empty(B, dtype=torch.int32, device=_CUDA)
            o["out_tokens"] = torch.empty((B, n_draft + 1), dtype=torch.int32, device=_CUDA)
            o["n_out"] = torch.empty(B, dtype=torch.int32, device=_CUDA)
        self._check(self.lib.ps_verify(
            self.h, B, n_draft, n_target, _dptr(draft_tokens), _dptr(draft_logits),
            _dptr(target_logits), float(temperature), seed, offset, _dptr(o["accept_len"]),
            _dptr(o["out_tokens"]), _dptr(o["n_out"]), _stream(stream)))
        return o

    def verify_tree(self, parent, tokens: torch.Tensor, draft_logits, target_logits: torch.Tensor,
                    temperature: float, seed: int, offset: int, out: dict | None = None, stream=None) -> dict:
        """ps_verify_tree.  parent: host list [n_nodes]; tokens [B][n_nodes] int32; draft_logits
        [B][D][V] float32 (D = 1 + largest depth) or None at temperature 0; target_logits
        [B][n_nodes+1][V] float32."""
        B, n_nodes = tokens.shape
        assert len(parent) == n_nodes and target_logits.shape == (B, n_nodes + 1, self.cfg.vocab)
        depth = []
        for i, p in enumerate(parent):
            depth.append(0 if p < 0 or p >= i else depth[p] + 1)   # a malformed tree is the library's to reject
        D = max(depth) + 1
        if draft_logits is not None:
            assert draft_logits.shape == (B, D, self.cfg.vocab) and draft_logits.dtype == torch.float32
        o = out if out is not None else {}
        if "accept_len" not in o:
            o["accept_len"] = torch.empty(B, dtype=torch.int32, device=_CUDA)
            o["out_tokens"] = torch.empty((B, D + 1), dtype=torch.int32, device=_CUDA)
            o["n_out"] = torch.empty(B, dtype=torch.int32, device=_CUDA)
            o["path"] = torch.empty((B, D), dtype=torch.int32, device=_CUDA)
        self._check(self.lib.ps_verify_tree(
            self.h, B, n_nodes, _iarr(parent), _dptr(tokens), _dptr(draft_logits), _dptr(target_logits),
            float(temperature), seed, offset, _dptr(o["accept_len"]), _dptr(o["out_tokens"]),
            _dptr(o["n_out"]), _dptr(o["path"]), _stream(stream)))
        return o

    def build_tree(self, parent, rank, top_ids: torch.Tensor, sampled_ids=None, out=None, stream=None):
        """ps_build_tree.  parent, rank: host lists [n_nodes]; top_ids [B][k+1][top_n] int32 (a draft
        step's output); sampled_ids [B][k+1] int32 or None.  Returns tokens [B][n_nodes] int32."""
        B, R, top_n = top_ids.shape
        assert R == self.rows and top_ids.dtype == torch.int32 and top_ids.is_contiguous()
        n_nodes = len(parent)
        assert len(rank) == n_nodes
        tokens = out if out is not None else torch.empty((B, n_nodes), dtype=torch.int32, device=_CUDA)
        self._check(self.lib.ps_build_tree(self.h, B, n_nodes, _iarr(parent), _iarr(rank), _dptr(top_ids), top_n,
                                           _dptr(sampled_ids), _dptr(tokens), _stream(stream)))
        return tokens

    def round_host(self, seq_slot, hidden_last: torch.Tensor, token_last: torch.Tensor,
                   target_logits: torch.Tensor, temperature: float, seed: int, offset: int,
                   out: dict | None = None, stream=None) -> dict:
        """ps_round_host: all tensors are HOST tensors (pinned for asynchronous copies)."""
        B, R = len(seq_slot), self.rows
        for t in (hidden_last, token_last, target_logits):
            assert not t.is_cuda and t.is_contiguous()
        o = out if out is not None else {}
        if "accept_len" not in o:
            o["accept_len"] = torch.empty(B, dtype=torch.int32).pin_memory()
            o["out_tokens"] = torch.empty((B, R + 1), dtype=torch.int32).pin_memory()
            o["n_out"] = torch.empty(B, dtype=torch.int32).pin_memory()
        hp = lambda t: C.c_void_p(t.data_ptr())
        self._check(self.lib.ps_round_host(
            self.h, B, _iarr(seq_slot), hp(hidden_last), hp(token_last), hp(target_logits),
            float(temperature), seed, offset, hp(o["accept_len"]), hp(o["out_tokens"]),
            hp(o["n_out"]), _stream(stream)))
        return o

    def check_guards(self, stream=None) -> int:
        """ps_debug_check_guards: number of workspace slices whose guard words were overwritten."""
        n = C.c_int(-1)
        self._check(self.lib.ps_debug_check_guards(self.h, _stream(stream), C.byref(n)))
        return n.value

    def debug_wait_expires(self, limit_cycles: int, stream=None) -> None:
        """ps_debug_wait_expires: a bounded device wait that runs out (sets the status word)."""
        self._check(self.lib.ps_debug_wait_expires(self.h, int(limit_cycles), _stream(stream)))

    def debug_late_copy(self, dst: torch.Tensor, src: torch.Tensor, delay_us: int, stream=None) -> None:
        """ps_debug_late_copy: dst <- src by a kernel that lets the launches behind it start early."""
        assert dst.dtype == src.dtype and dst.numel() == src.numel()
        self._check(self.lib.ps_debug_late_copy(self.h, _dptr(dst), _dptr(src), dst.numel() * dst.element_size(),
                                                int(delay_us), _stream(stream)))

    def poll(self) -> int:
        """Waits for the stream and returns the device status (PS_OK, PS_ERR_NONFINITE, ...)."""
        return self.lib.ps_poll(self.h, _stream())

    def profile(self, enable) -> None:
        """ps_profile: False / 0 off, True / 1 an event per stage, 2 an event per launch."""
        self._check(self.lib.ps_profile(self.h, int(enable)))

    def profile_read(self) -> dict:
        """{stage: (total_ms, intervals)} since profiling was enabled or last read."""
        n_max = 32
        names = C.create_string_buffer(32 * n_max)
        ms = (C.c_float * n_max)()
        cnt = (C.c_int * n_max)()
        n = C.c_int()
        self._check(self.lib.ps_profile_read(self.h, n_max, names, ms, cnt, C.byref(n)))
        raw = names.raw
        return {raw[32 * i:32 * i + 32].split(b"\0")[0].decode(): (ms[i], cnt[i]) for i in range(n.value)}

    def debug_buffer(self, name: str, dtype, shape) -> torch.Tensor:
        """Copy of an intermediate buffer of the last draft step (test helper)."""
        ptr, nbytes = C.c_void_p(), C.c_size_t()
        self._check(self.lib.ps_debug_buffer(self.h, name.encode(), C.byref(ptr), C.byref(nbytes)))
        base = self.workspace.data_ptr()
        off = ptr.value - base
        n = 1
        for d in shape:
            n *= d
        elt = torch.empty((), dtype=dtype).element_size()
        assert 0 <= off and n * elt <= nbytes.value and off + n * elt <= self.workspace.numel()
        return self.workspace[off:off + n * elt].view(dtype).view(*shape).clone()

    def launch_count(self) -> int:
        return self.lib.ps_launch_count(self.h)
