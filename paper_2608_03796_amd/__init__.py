"""Fused chunked top-K KL distillation loss on AMD MI355X (gfx950).

Python binding of libkdtopk.so (C ABI in include/kdtopk.h). The binding only
marshals arguments: PyTorch provides device memory and the current stream;
every step of the loss runs in the library's HIP kernels. There is no CPU or
PyTorch fallback: if the library is missing, the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkdtopk.so")

KD_F32 = 0
KD_BF16 = 1
KD_MX4 = 2
KD_FLAG_TEACHER_LOGPROBS = 1
KD_FLAG_GRAD_HIDDEN_F32 = 2

STATUS = {
    0: "KD_OK", 1: "KD_ERR_NULL_PTR", 2: "KD_ERR_BAD_SHAPE", 3: "KD_ERR_BAD_ARG",
    4: "KD_ERR_UNSUPPORTED", 5: "KD_ERR_WORKSPACE_TOO_SMALL", 6: "KD_ERR_BAD_INDEX",
    7: "KD_ERR_DEVICE",
}
EXPORTED = ("kd_topk_kl_workspace_size", "kd_topk_kl_fwd_bwd", "kd_topk_kl_fwd_bwd_noalloc",
            "kd_topk_kl_fwd",
            "kd_topk_kl_bwd", "kd_topk_kl_check_indices", "kd_scale_grads", "kd_status_string",
            "kd_abi_version", "kd_profile_enable", "kd_profile_read",
            "kd_topk_entries_workspace_size", "kd_topk_entries", "kd_teacher_cache_write",
            "kd_teacher_cache_read", "kd_checkpoint_write", "kd_checkpoint_read",
            "kd_topk_kl_bwd_checkpoint",
            "kd_verify_draft_workspace_size", "kd_verify_draft", "kd_mx4_write", "kd_mx4_read",
            "kd_mx4_logits_workspace_size", "kd_mx4_logits",
            "kd_cross_entropy_workspace_size", "kd_cross_entropy_fwd_bwd", "kd_cross_entropy_fwd",
            "kd_cross_entropy_bwd")


class KdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)}")


class KdProblem(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int64), ("V", ctypes.c_int64),
                ("chunk", ctypes.c_int64), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("flags", ctypes.c_int32)]


class KdKernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double), ("flops", ctypes.c_double)]


class KdRows(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("V", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("K", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32)]


class KdDraft(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("T", ctypes.c_int64), ("V", ctypes.c_int64),
                ("ld_target", ctypes.c_int64), ("ld_draft", ctypes.c_int64),
                ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("temperature", ctypes.c_double), ("flags", ctypes.c_int32)]


class KdLabelProblem(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int64), ("V", ctypes.c_int64),
                ("chunk", ctypes.c_int64), ("dtype", ctypes.c_int32), ("z_loss", ctypes.c_float),
                ("flags", ctypes.c_int32)]


class KdMx4Head(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("D", ctypes.c_int64), ("V", ctypes.c_int64),
                ("ld_hidden", ctypes.c_int64), ("ld_out", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libkdtopk.so (built by paper_2608_03796_amd.build). Raises if absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is not built; run `python -m paper_2608_03796_amd.build`")
    lib = ctypes.CDLL(p)
    vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    lib.kd_topk_kl_workspace_size.argtypes = [ctypes.POINTER(KdProblem), ctypes.POINTER(sz)]
    lib.kd_topk_kl_workspace_size.restype = ctypes.c_int
    lib.kd_topk_kl_fwd_bwd.argtypes = [ctypes.POINTER(KdProblem), vp, vp, vp, vp, vp, vp, vp, vp,
                                       vp, ctypes.c_int, vp, sz, vp]
    lib.kd_topk_kl_fwd_bwd.restype = ctypes.c_int
    lib.kd_topk_kl_fwd_bwd_noalloc.argtypes = [ctypes.POINTER(KdProblem), vp, vp, vp, vp, vp,
                                               vp, vp, vp, vp, ctypes.c_int, vp]
    lib.kd_topk_kl_fwd_bwd_noalloc.restype = ctypes.c_int
    lib.kd_topk_kl_fwd.argtypes = [ctypes.POINTER(KdProblem), vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                   sz, vp]
    lib.kd_topk_kl_fwd.restype = ctypes.c_int
    lib.kd_topk_kl_bwd.argtypes = [ctypes.POINTER(KdProblem), vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                   vp, ctypes.c_int, vp, sz, vp]
    lib.kd_topk_kl_bwd.restype = ctypes.c_int
    lib.kd_topk_kl_check_indices.argtypes = [ctypes.POINTER(KdProblem), vp, vp, sz, vp]
    lib.kd_topk_kl_check_indices.restype = ctypes.c_int
    lib.kd_scale_grads.argtypes = [vp, vp, ctypes.c_int32, vp, i64, vp, ctypes.c_int32, vp, i64,
                                   vp]
    lib.kd_scale_grads.restype = ctypes.c_int
    lib.kd_status_string.argtypes = [ctypes.c_int]
    lib.kd_status_string.restype = ctypes.c_char_p
    lib.kd_abi_version.argtypes = []
    lib.kd_abi_version.restype = ctypes.c_int
    lib.kd_profile_enable.argtypes = [ctypes.c_int]
    lib.kd_profile_enable.restype = ctypes.c_int
    lib.kd_profile_read.argtypes = [ctypes.POINTER(KdKernelTime), ctypes.c_int]
    lib.kd_profile_read.restype = ctypes.c_int
    lib.kd_topk_kl_bwd_checkpoint.argtypes = [ctypes.POINTER(KdProblem), vp, vp, vp, vp, vp, vp,
                                              vp, vp, vp, vp, ctypes.c_int, vp, sz, vp]
    lib.kd_topk_kl_bwd_checkpoint.restype = ctypes.c_int
    i32 = ctypes.c_int32
    rows, draft = ctypes.POINTER(KdRows), ctypes.POINTER(KdDraft)
    head, labels = ctypes.POINTER(KdMx4Head), ctypes.POINTER(KdLabelProblem)
    for name, argtypes in (
            ("kd_topk_entries_workspace_size", [rows, ctypes.POINTER(sz)]),
            ("kd_topk_entries", [rows, vp, vp, vp, vp, sz, vp]),
            ("kd_teacher_cache_write", [rows, vp, vp, vp, vp, sz, vp]),
            ("kd_teacher_cache_read", [i64, i32, vp, vp, vp, i64, vp, vp, vp, vp]),
            ("kd_checkpoint_write", [i64, i64, i32, vp, vp, vp, vp]),
            ("kd_checkpoint_read", [i64, i64, i32, vp, vp, vp, vp]),
            ("kd_verify_draft_workspace_size", [draft, ctypes.POINTER(sz)]),
            ("kd_verify_draft", [draft] + [vp] * 11 + [sz, vp]),
            ("kd_mx4_write", [i64, i64, i32, vp, vp, vp, vp]),
            ("kd_mx4_read", [i64, i64, i32, vp, vp, vp, vp]),
            ("kd_mx4_logits_workspace_size", [head, ctypes.POINTER(sz)]),
            ("kd_mx4_logits", [head] + [vp] * 6 + [sz, vp]),
            ("kd_cross_entropy_workspace_size", [labels, ctypes.POINTER(sz)]),
            ("kd_cross_entropy_fwd_bwd", [labels] + [vp] * 7 + [ctypes.c_int, vp, sz, vp]),
            ("kd_cross_entropy_fwd", [labels] + [vp] * 7 + [sz, vp]),
            ("kd_cross_entropy_bwd", [labels] + [vp] * 8 + [ctypes.c_int, vp, sz, vp])):
        getattr(lib, name).argtypes = argtypes
        getattr(lib, name).restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def problem(N, D, V, K, chunk, tau, dtype, flags=0) -> KdProblem:
    return KdProblem(int(N), int(D), int(V), int(chunk), int(K), int(dtype), float(tau), int(flags))


def _flags(teacher_logprobs=False, grad_hidden_f32=False) -> int:
    return (KD_FLAG_TEACHER_LOGPROBS if teacher_logprobs else 0) | \
        (KD_FLAG_GRAD_HIDDEN_F32 if grad_hidden_f32 else 0)


def _dtype_code(t) -> int:
    import torch
    if t == torch.bfloat16:
        return KD_BF16
    if t == torch.float32:
        return KD_F32
    raise TypeError(f"unsupported dtype {t}")


def workspace_size(N, D, V, K, chunk, tau=1.0, dtype=KD_BF16) -> int:
    lib = load_library()
    pr = problem(N, D, V, K, chunk, tau, dtype)
    out = ctypes.c_size_t(0)
    rc = lib.kd_topk_kl_workspace_size(ctypes.byref(pr), ctypes.byref(out))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_workspace_size")
    return int(out.value)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream_handle(device):
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def alloc_workspace(N, D, V, K, chunk, tau, dtype, device):
    import torch
    n = workspace_size(N, D, V, K, chunk, tau, dtype)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _check_inputs(hidden, W, teacher_idx, teacher_logit, ignore, checkpoint=False):
    """Dtypes, shapes, devices and layouts of the inputs. The library takes
    plain pointers, so every size it will index with is checked here. With
    checkpoint, hidden is a checkpoint's codes and W gives the dtype."""
    import torch
    if hidden.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if hidden.dim() != 2 or W.dim() != 2:
        raise ValueError("hidden must be [N, D] and W [V, D]")
    if W.dtype != hidden.dtype and not checkpoint:
        raise TypeError("hidden and W must share a dtype")
    for name, t, want in (("teacher_idx", teacher_idx, torch.int32),
                          ("teacher_logit", teacher_logit, torch.float32)):
        if t.dtype != want:
            raise TypeError(f"{name} must be {want}")
    if ignore is not None and ignore.dtype != torch.uint8:
        raise TypeError("ignore must be uint8")
    N, D = hidden.shape
    if W.shape[1] != D:
        raise ValueError(f"W is {tuple(W.shape)}, expected [V, {D}]")
    if teacher_idx.dim() != 2 or teacher_idx.shape[0] != N:
        raise ValueError(f"teacher_idx is {tuple(teacher_idx.shape)}, expected [{N}, K]")
    K = teacher_idx.shape[1]
    if tuple(teacher_logit.shape) != (N, K):
        raise ValueError(f"teacher_logit is {tuple(teacher_logit.shape)}, expected [{N}, {K}]")
    if ignore is not None and tuple(ignore.shape) != (N,):
        raise ValueError(f"ignore is {tuple(ignore.shape)}, expected [{N}]")
    tensors = [hidden, W, teacher_idx, teacher_logit] + ([ignore] if ignore is not None else [])
    for t in tensors:
        if not t.is_contiguous():
            raise ValueError("inputs must be contiguous")
        if t.device != hidden.device:
            raise ValueError("inputs must be on one device")
    return N, D, W.shape[0], K, _dtype_code(W.dtype)


def _check_tensor(name, t, shape, dtype, device):
    """A caller-provided output or extra input: exact shape, dtype, device, layout."""
    if t.shape != tuple(shape) or t.dtype != dtype or t.device != device \
            or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} "
                         f"on {device} (got {t.dtype} {tuple(t.shape)} on {t.device})")


def _check_workspace(workspace, device):
    import torch
    if workspace.dtype != torch.uint8 or workspace.device != device \
            or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")


def fwd_bwd(hidden, W, teacher_idx, teacher_logit, tau: float = 1.0, ignore=None,
            chunk: int = 4096, grad_hidden: bool = True, grad_W: bool = True,
            loss_per_token: bool = False, grad_W_out=None, accumulate_grad_W: bool = False,
            workspace=None, out=None, teacher_logprobs: bool = False,
            grad_hidden_f32: bool = False):
    """One call of kd_topk_kl_fwd_bwd on the current stream.

    hidden [N, D] and W [V, D] (bf16 or fp32, same dtype), teacher_idx [N, K]
    int32, teacher_logit [N, K] fp32 (log-probabilities of a partial-mass
    teacher when teacher_logprobs), ignore [N] uint8 or None. Returns a dict
    with 'loss' (0-d fp32 tensor), and 'loss_per_token', 'grad_hidden',
    'grad_W' when requested. grad_hidden is in hidden's dtype, or fp32 with
    grad_hidden_f32. `out` may carry preallocated output tensors (keys as
    returned) to make repeated calls allocation-free.
    """
    import torch
    lib = load_library()
    N, D, V, K, dt = _check_inputs(hidden, W, teacher_idx, teacher_logit, ignore)
    out = dict(out or {})
    dev = hidden.device
    if "loss" not in out:
        out["loss"] = torch.empty((), dtype=torch.float32, device=dev)
    if loss_per_token and "loss_per_token" not in out:
        out["loss_per_token"] = torch.empty(N, dtype=torch.float32, device=dev)
    gh_dtype = torch.float32 if grad_hidden_f32 else hidden.dtype
    if grad_hidden and "grad_hidden" not in out:
        out["grad_hidden"] = torch.empty(N, D, dtype=gh_dtype, device=dev)
    if grad_W:
        if grad_W_out is not None:
            out["grad_W"] = grad_W_out
        elif "grad_W" not in out:
            out["grad_W"] = torch.empty(V, D, dtype=torch.float32, device=dev)
    _check_tensor("loss", out["loss"], (), torch.float32, dev)
    if loss_per_token:
        _check_tensor("loss_per_token", out["loss_per_token"], (N,), torch.float32, dev)
    if grad_hidden:
        _check_tensor("grad_hidden", out["grad_hidden"], (N, D), gh_dtype, dev)
    if grad_W:
        _check_tensor("grad_W", out["grad_W"], (V, D), torch.float32, dev)
    pr = problem(N, D, V, K, chunk, tau, dt, _flags(teacher_logprobs, grad_hidden_f32))
    if workspace is None:
        workspace = alloc_workspace(N, D, V, K, chunk, tau, dt, dev)
    _check_workspace(workspace, dev)
    with torch.cuda.device(dev):
        rc = lib.kd_topk_kl_fwd_bwd(
            ctypes.byref(pr), _ptr(hidden), _ptr(W), _ptr(teacher_idx), _ptr(teacher_logit),
            _ptr(ignore), _ptr(out["loss"]), _ptr(out.get("loss_per_token") if loss_per_token else None),
            _ptr(out.get("grad_hidden") if grad_hidden else None),
            _ptr(out.get("grad_W") if grad_W else None), int(bool(accumulate_grad_W)),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_fwd_bwd")
    res = {"loss": out["loss"]}
    if loss_per_token:
        res["loss_per_token"] = out["loss_per_token"]
    if grad_hidden:
        res["grad_hidden"] = out["grad_hidden"]
    if grad_W:
        res["grad_W"] = out["grad_W"]
    return res


def fwd_bwd_noalloc(hidden, W, teacher_idx, teacher_logit, tau: float = 1.0, ignore=None,
                    chunk: int = 4096, out=None, grad_hidden: bool = True, grad_W: bool = True,
                    loss_per_token: bool = False, accumulate_grad_W: bool = False,
                    teacher_logprobs: bool = False):
    """kd_topk_kl_fwd_bwd_noalloc: kd_topk_kl_fwd_bwd with the library's own
    static per-device scratch as workspace. Pass every wanted output in `out`
    ('loss' 0-d fp32, 'loss_per_token' [N] fp32, 'grad_hidden' [N, D] in
    hidden's dtype, 'grad_W' [V, D] fp32) to make the call allocation-free;
    missing ones are allocated here. Returns the outputs as fwd_bwd does."""
    import torch
    lib = load_library()
    N, D, V, K, dt = _check_inputs(hidden, W, teacher_idx, teacher_logit, ignore)
    dev = hidden.device
    out = dict(out or {})
    want = {"loss": ((), torch.float32, True),
            "loss_per_token": ((N,), torch.float32, loss_per_token),
            "grad_hidden": ((N, D), hidden.dtype, grad_hidden),
            "grad_W": ((V, D), torch.float32, grad_W)}
    for k, (shape, dtype, on) in want.items():
        if not on:
            continue
        if k not in out:
            out[k] = torch.empty(shape, dtype=dtype, device=dev)
        _check_tensor(k, out[k], shape, dtype, dev)
    pr = problem(N, D, V, K, chunk, tau, dt, _flags(teacher_logprobs))
    with torch.cuda.device(dev):
        rc = lib.kd_topk_kl_fwd_bwd_noalloc(
            ctypes.byref(pr), _ptr(hidden), _ptr(W), _ptr(teacher_idx), _ptr(teacher_logit),
            _ptr(ignore), _ptr(out["loss"]),
            _ptr(out["loss_per_token"] if loss_per_token else None),
            _ptr(out["grad_hidden"] if grad_hidden else None),
            _ptr(out["grad_W"] if grad_W else None), int(bool(accumulate_grad_W)),
            _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_fwd_bwd_noalloc")
    return {k: out[k] for k, (_, _, on) in want.items() if on}


def fwd(hidden, W, teacher_idx, teacher_logit, tau: float = 1.0, ignore=None,
        chunk: int = 4096, loss_per_token: bool = False, workspace=None,
        teacher_logprobs: bool = False):
    """kd_topk_kl_fwd: the loss without gradient work, plus the per-token
    log-normaliser log Z the backward needs. Returns a dict with 'loss' (0-d),
    'saved_logz' [N] and, when requested, 'loss_per_token' [N]."""
    import torch
    lib = load_library()
    N, D, V, K, dt = _check_inputs(hidden, W, teacher_idx, teacher_logit, ignore)
    dev = hidden.device
    res = {"loss": torch.empty((), dtype=torch.float32, device=dev),
           "saved_logz": torch.empty(N, dtype=torch.float32, device=dev)}
    if loss_per_token:
        res["loss_per_token"] = torch.empty(N, dtype=torch.float32, device=dev)
    pr = problem(N, D, V, K, chunk, tau, dt, _flags(teacher_logprobs))
    if workspace is None:
        workspace = alloc_workspace(N, D, V, K, chunk, tau, dt, dev)
    _check_workspace(workspace, dev)
    with torch.cuda.device(dev):
        rc = lib.kd_topk_kl_fwd(
            ctypes.byref(pr), _ptr(hidden), _ptr(W), _ptr(teacher_idx), _ptr(teacher_logit),
            _ptr(ignore), _ptr(res["loss"]), _ptr(res.get("loss_per_token")), _ptr(res["saved_logz"]),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_fwd")
    return res


def bwd(hidden, W, teacher_idx, teacher_logit, saved_logz, tau: float = 1.0, ignore=None,
        chunk: int = 4096, grad_loss=None, grad_loss_per_token=None, grad_hidden: bool = True,
        grad_W: bool = True, grad_W_out=None, accumulate_grad_W: bool = False, workspace=None,
        teacher_logprobs: bool = False, grad_hidden_f32: bool = False):
    """kd_topk_kl_bwd: gradients from the saved log-normaliser. grad_loss is the
    upstream gradient of the mean loss (0-d fp32 device tensor, None = 1);
    grad_loss_per_token [N] fp32 replaces it with per-token upstream gradients.
    Returns a dict with 'grad_hidden' (hidden's dtype, or fp32 with
    grad_hidden_f32) and 'grad_W' as requested."""
    import torch
    lib = load_library()
    N, D, V, K, dt = _check_inputs(hidden, W, teacher_idx, teacher_logit, ignore)
    dev = hidden.device
    _check_tensor("saved_logz", saved_logz, (N,), torch.float32, dev)
    if grad_loss is not None and grad_loss.numel() == 1:
        _check_tensor("grad_loss", grad_loss, tuple(grad_loss.shape), torch.float32, dev)
    elif grad_loss is not None:
        raise ValueError("grad_loss must hold one value (the upstream gradient of the mean)")
    if grad_loss_per_token is not None:
        _check_tensor("grad_loss_per_token", grad_loss_per_token, (N,), torch.float32, dev)
    res = {}
    if grad_hidden:
        res["grad_hidden"] = torch.empty(N, D, device=dev,
                                         dtype=torch.float32 if grad_hidden_f32 else hidden.dtype)
    if grad_W:
        res["grad_W"] = grad_W_out if grad_W_out is not None else torch.empty(
            V, D, dtype=torch.float32, device=dev)
        _check_tensor("grad_W", res["grad_W"], (V, D), torch.float32, dev)
    pr = problem(N, D, V, K, chunk, tau, dt, _flags(teacher_logprobs, grad_hidden_f32))
    if workspace is None:
        workspace = alloc_workspace(N, D, V, K, chunk, tau, dt, dev)
    _check_workspace(workspace, dev)
    with torch.cuda.device(dev):
        rc = lib.kd_topk_kl_bwd(
            ctypes.byref(pr), _ptr(hidden), _ptr(W), _ptr(teacher_idx), _ptr(teacher_logit),
            _ptr(ignore), _ptr(saved_logz), _ptr(grad_loss), _ptr(grad_loss_per_token),
            _ptr(res.get("grad_hidden")), _ptr(res.get("grad_W")), int(bool(accumulate_grad_W)),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_bwd")
    return res


def scale_grads(grad_loss, grad_hidden=None, grad_hidden_out=None, grad_W=None,
                grad_W_out=None):
    """kd_scale_grads on the current stream: out = grad_loss * in for the fp32
    gradients grad_hidden and grad_W of the mean loss, each written to its
    output (fp32 or bf16; an fp32 output may be its input). grad_loss is the
    upstream gradient of the mean, a one-element fp32 device tensor."""
    import torch
    lib = load_library()
    pairs = (("grad_hidden", grad_hidden, grad_hidden_out), ("grad_W", grad_W, grad_W_out))
    dev = None
    for name, x, y in pairs:
        if (x is None) != (y is None):
            raise ValueError(f"{name} and its output go together")
        if x is not None:
            dev = x.device if dev is None else dev
            _check_tensor(name, x, tuple(x.shape), torch.float32, dev)
            _check_tensor(name + "_out", y, tuple(x.shape), y.dtype, dev)
    if dev is None:
        return
    if grad_loss.numel() != 1:
        raise ValueError("grad_loss must hold one value")
    _check_tensor("grad_loss", grad_loss, tuple(grad_loss.shape), torch.float32, dev)

    def code(y):
        return _dtype_code(y.dtype) if y is not None else KD_F32

    with torch.cuda.device(dev):
        rc = lib.kd_scale_grads(
            _ptr(grad_loss), _ptr(grad_hidden), code(grad_hidden_out), _ptr(grad_hidden_out),
            grad_hidden.numel() if grad_hidden is not None else 0,
            _ptr(grad_W), code(grad_W_out), _ptr(grad_W_out),
            grad_W.numel() if grad_W is not None else 0, _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_scale_grads")


def _autograd_functions():
    import torch

    class TopKKLLoss(torch.autograd.Function):
        """Mean top-K KL loss as an autograd function, Algorithm 1's schedule:
        forward runs kd_topk_kl_fwd and saves log Z; backward runs
        kd_topk_kl_bwd with the upstream gradient (logit recompute). grad_W is
        returned in W's dtype (fp32 accumulation inside one call; use
        bwd(..., accumulate_grad_W=True) to accumulate micro-batches in fp32)."""

        @staticmethod
        def forward(ctx, hidden, W, teacher_idx, teacher_logit, tau, ignore, chunk,
                    teacher_logprobs, workspace):
            res = fwd(hidden, W, teacher_idx, teacher_logit, tau=tau, ignore=ignore, chunk=chunk,
                      teacher_logprobs=teacher_logprobs, workspace=workspace)
            ctx.save_for_backward(hidden, W, teacher_idx, teacher_logit, res["saved_logz"],
                                  *([ignore] if ignore is not None else []))
            ctx.cfg = (tau, chunk, teacher_logprobs, ignore is not None)
            ctx.workspace = workspace
            return res["loss"]

        @staticmethod
        def backward(ctx, grad_out):
            tau, chunk, logprobs, has_ignore = ctx.cfg
            saved = ctx.saved_tensors
            hidden, W, idx, tl, logz = saved[:5]
            ignore = saved[5] if has_ignore else None
            g = grad_out.detach().to(torch.float32).contiguous()
            need_h, need_W = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
            res = bwd(hidden, W, idx, tl, logz, tau=tau, ignore=ignore, chunk=chunk, grad_loss=g,
                      grad_hidden=need_h, grad_W=need_W, teacher_logprobs=logprobs,
                      workspace=ctx.workspace)
            gW = res.get("grad_W")
            if gW is not None and gW.dtype != W.dtype:
                gW = gW.to(W.dtype)
            return res.get("grad_hidden"), gW, None, None, None, None, None, None, None

    class TopKKLLossFused(torch.autograd.Function):
        """Mean top-K KL loss as an autograd function, one projection per chunk:
        when a gradient is wanted, forward runs kd_topk_kl_fwd_bwd and keeps the
        gradients of the mean (both in fp32); backward has kd_scale_grads
        multiply them by the upstream gradient (exact: the loss is linear in
        it) and round them once to the inputs' dtypes. The gradients are held
        from forward to backward; backward runs once per graph."""

        @staticmethod
        def forward(ctx, hidden, W, teacher_idx, teacher_logit, tau, ignore, chunk,
                    teacher_logprobs, workspace):
            need_h, need_W = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
            ctx.grads = None
            if not (need_h or need_W):
                # the loss alone (no log Z to save): the fused call without
                # gradients, which leaves ignored tokens out
                return fwd_bwd(hidden, W, teacher_idx, teacher_logit, tau=tau, ignore=ignore,
                               chunk=chunk, grad_hidden=False, grad_W=False,
                               teacher_logprobs=teacher_logprobs, workspace=workspace)["loss"]
            out = fwd_bwd(hidden, W, teacher_idx, teacher_logit, tau=tau, ignore=ignore,
                          chunk=chunk, grad_hidden=need_h, grad_W=need_W,
                          teacher_logprobs=teacher_logprobs, workspace=workspace,
                          grad_hidden_f32=True)
            ctx.grads = [out.get("grad_hidden"), out.get("grad_W")]
            ctx.dtypes = (hidden.dtype, W.dtype)
            return out["loss"]

        @staticmethod
        def backward(ctx, grad_out):
            if ctx.grads is None:
                raise RuntimeError("topk_kl_loss(schedule='fused') supports one backward per "
                                   "graph; use schedule='recompute' to run backward again")
            gh, gW = ctx.grads
            ctx.grads = None
            h_dtype, w_dtype = ctx.dtypes
            g = grad_out.detach().to(torch.float32).contiguous()
            # both gradients are fp32 here: scaled by g in the library and
            # rounded once to the inputs' dtypes (in place when fp32)
            gh_out = None
            if gh is not None:
                gh_out = gh if h_dtype == torch.float32 else torch.empty_like(gh, dtype=h_dtype)
            gW_out = None
            if gW is not None:
                gW_out = gW if w_dtype == torch.float32 else torch.empty_like(gW, dtype=w_dtype)
            scale_grads(g, grad_hidden=gh, grad_hidden_out=gh_out, grad_W=gW, grad_W_out=gW_out)
            return gh_out, gW_out, None, None, None, None, None, None, None

    class TopKKLLossCheckpoint(torch.autograd.Function):
        """Mean top-K KL loss as an autograd function that keeps its hidden
        states in 8 bits: forward computes the loss from the exact ones and
        writes their checkpoint; backward runs kd_topk_kl_bwd_checkpoint with the
        upstream gradient."""

        @staticmethod
        def forward(ctx, hidden, W, teacher_idx, teacher_logit, tau, ignore, chunk,
                    teacher_logprobs, workspace):
            loss = fwd_bwd(hidden, W, teacher_idx, teacher_logit, tau=tau, ignore=ignore,
                           chunk=chunk, grad_hidden=False, grad_W=False,
                           teacher_logprobs=teacher_logprobs, workspace=workspace)["loss"]
            if ctx.needs_input_grad[0] or ctx.needs_input_grad[1]:
                c = checkpoint_write(hidden)
                ctx.save_for_backward(c["codes"], c["scales"], W, teacher_idx, teacher_logit,
                                      *([ignore] if ignore is not None else []))
            ctx.cfg = (tau, chunk, teacher_logprobs, ignore is not None)
            ctx.workspace = workspace
            return loss

        @staticmethod
        def backward(ctx, grad_out):
            tau, chunk, logprobs, has_ignore = ctx.cfg
            saved = ctx.saved_tensors
            codes, scales, W, idx, tl = saved[:5]
            g = grad_out.detach().to(torch.float32).contiguous()
            res = bwd_checkpoint(codes, scales, W, idx, tl, tau=tau,
                                 ignore=saved[5] if has_ignore else None, chunk=chunk, grad_loss=g,
                                 grad_hidden=ctx.needs_input_grad[0],
                                 grad_W=ctx.needs_input_grad[1], teacher_logprobs=logprobs,
                                 workspace=ctx.workspace)
            gW = res.get("grad_W")
            if gW is not None and gW.dtype != W.dtype:
                gW = gW.to(W.dtype)
            return res.get("grad_hidden"), gW, None, None, None, None, None, None, None

    return {"recompute": TopKKLLoss, "fused": TopKKLLossFused,
            "checkpoint": TopKKLLossCheckpoint}


_TOPK_KL = None


def topk_kl_loss(hidden, W, teacher_idx, teacher_logit, tau: float = 1.0, ignore=None,
                 chunk: int = 4096, teacher_logprobs: bool = False, schedule: str = "fused",
                 workspace=None, checkpoint: bool = False):
    """Differentiable mean top-K KL loss.

    schedule="fused": when hidden or W needs a gradient, the forward computes
    the loss and the gradients of the mean in one kd_topk_kl_fwd_bwd call (one
    projection per chunk) and the backward scales them by the upstream
    gradient in the library (kd_scale_grads), rounding each once to its
    input's dtype; backward runs once per graph. Cost when no backward
    follows (a loss only logged with grad mode on): the forward still does
    all the gradient work (about 3x the forward-only time) and holds the fp32
    gradients ([N, D] and [V, D]: 2.5 GiB at N = 32768, D = 4096,
    V = 131072) until the graph is freed; they are kept on the autograd
    context, so saved-tensor hooks (offloading) do not see them. Compute such
    a loss under torch.no_grad() (the loss alone, through kd_topk_kl_fwd_bwd
    without gradients), or use schedule="recompute", whose forward is
    kd_topk_kl_fwd alone and which saves only log Z.
    schedule="recompute": Algorithm 1's schedule through the split entry
    points (forward saves log Z; backward recomputes the logits).
    checkpoint=True (schedule="recompute" only): the hidden states are kept from
    forward to backward in 8 bits (checkpoint_write: 1.03 bytes an element
    instead of 2 or 4; the caller's own tensor may be freed), and the gradients
    are those of the loss at the values held (bwd_checkpoint). The loss itself is
    computed from the exact ones. The backward is the fused schedule's, which forms
    log Z with the gradient: in bf16 grad_W's contraction has the hidden rows times
    their tokens' factors, rounded to bf16 (2.9e-3 off in the 2-norm, final rounding
    included), where schedule="recompute" alone has the rows as they are (2.3e-3).
    workspace: a uint8 device tensor of at least workspace_size(...) bytes to
    reuse across calls (allocated per call when None)."""
    import torch
    global _TOPK_KL
    if schedule not in ("fused", "recompute"):
        raise ValueError("schedule must be 'fused' or 'recompute'")
    if checkpoint and schedule != "recompute":
        raise ValueError("checkpoint=True goes with schedule='recompute' (the fused schedule keeps "
                         "gradients, not hidden states)")
    if not torch.is_grad_enabled():
        # no graph will be built: the loss alone (no gradient work; ignored
        # tokens left out)
        return fwd_bwd(hidden, W, teacher_idx, teacher_logit, tau=tau, ignore=ignore,
                       chunk=chunk, grad_hidden=False, grad_W=False,
                       teacher_logprobs=teacher_logprobs, workspace=workspace)["loss"]
    if _TOPK_KL is None:
        _TOPK_KL = _autograd_functions()
    return _TOPK_KL["checkpoint" if checkpoint else schedule].apply(
        hidden, W, teacher_idx, teacher_logit, float(tau), ignore, int(chunk),
        bool(teacher_logprobs), workspace)


def check_indices(teacher_idx, V, chunk=4096, D=64, tau=1.0, dtype=KD_BF16, workspace=None):
    """True if every index is in [0, V) and no row repeats one (synchronises)."""
    import torch
    lib = load_library()
    if teacher_idx.device.type != "cuda" or teacher_idx.dtype != torch.int32 \
            or teacher_idx.dim() != 2 or not teacher_idx.is_contiguous():
        raise ValueError("teacher_idx must be a contiguous [N, K] int32 GPU tensor")
    N, K = teacher_idx.shape
    pr = problem(N, D, V, K, chunk, tau, dtype)
    if workspace is None:
        # (what the check uses of a workspace)
        workspace = torch.empty(256, dtype=torch.uint8, device=teacher_idx.device)
    _check_workspace(workspace, teacher_idx.device)
    with torch.cuda.device(teacher_idx.device):
        rc = lib.kd_topk_kl_check_indices(ctypes.byref(pr), _ptr(teacher_idx), _ptr(workspace),
                                          ctypes.c_size_t(workspace.numel()),
                                          _stream_handle(teacher_idx.device))
    if rc == 6:
        return False
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_check_indices")
    return True


def _call(name, device, *args):
    """One call of the library on device's current stream (the last argument); tensors
    are passed as they are, None as NULL. The small operators' calls take a few
    microseconds on the GPU, so the host's part counts: the device is switched to
    only where it is not the current one."""
    import torch
    fn = getattr(_lib, name)
    args = [a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]
    # (by number: half the time of the same by device)
    stream = torch.cuda.current_stream(device.index).cuda_stream
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream)
    if rc != 0:
        raise KdError(rc, name)


def _logits_rows(name, logits, dim):
    """dtype code and element stride of the rows of logits[..., V]: the last
    dimension contiguous, the rows evenly spaced."""
    if logits.device.type != "cuda":
        raise ValueError(f"{name} must be on a GPU")
    if logits.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions")
    code = _dtype_code(logits.dtype)
    V = logits.shape[-1]
    ld = V
    # (a dimension of one row may have any stride)
    if dim == 2 and logits.shape[0] > 1:
        ld = logits.stride(0)
    elif dim == 3:
        if logits.shape[1] > 1:
            ld = logits.stride(1)
        elif logits.shape[0] > 1:
            ld = logits.stride(0)
        if logits.shape[0] > 1 and logits.shape[1] > 0 \
                and logits.stride(0) != logits.shape[1] * ld:
            raise ValueError(f"the rows of {name} must be evenly spaced")
    if (V > 1 and logits.stride(-1) != 1) or ld < V:
        raise ValueError(f"the rows of {name} must be contiguous and must not overlap")
    return code, ld


def _topk_rows(logits, K, logprobs, workspace):
    """The problem and workspace of a selection, with its checks."""
    import torch
    load_library()
    code, ld = _logits_rows("logits", logits, 2)
    N, V = logits.shape
    if workspace is None:
        workspace = torch.empty(topk_workspace_size(N, V, int(K), code), dtype=torch.uint8,
                                device=logits.device)
    _check_workspace(workspace, logits.device)
    return KdRows(N, V, ld, int(K), code, KD_FLAG_TEACHER_LOGPROBS if logprobs else 0), workspace


def _out_tensors(out, want, device):
    """The outputs of `want` (name -> (shape, dtype)): from `out`, checked, or new."""
    import torch
    res = {}
    for name, (shape, dtype) in want.items():
        t = out.get(name) if out else None
        if t is None:
            t = torch.empty(shape, dtype=dtype, device=device)
        else:
            _check_tensor(name, t, shape, dtype, device)
        res[name] = t
    return res


def topk_entries(logits, K, logprobs: bool = False, out=None, workspace=None):
    """kd_topk_entries on the current stream: the K largest logits of each row
    of logits [N, V] (bf16 or fp32, rows evenly spaced), as the loss takes them.
    Returns {'teacher_idx' [N, K] int32, 'teacher_logit' [N, K] fp32}, largest
    first, of equal ones the lowest index first; log-probabilities over the
    whole vocabulary with logprobs (for teacher_logprobs=True). No gradient flows
    to logits. A row whose first value is -inf holds no target, and one with +inf
    no finite loss: pass such rows to the loss as ignored. `out` may carry the
    outputs, `workspace` a uint8 tensor of topk_workspace_size bytes."""
    import torch
    pr, workspace = _topk_rows(logits, K, logprobs, workspace)
    dev = logits.device
    res = _out_tensors(out, {"teacher_idx": ((pr.N, pr.K), torch.int32),
                             "teacher_logit": ((pr.N, pr.K), torch.float32)}, dev)
    _call("kd_topk_entries", dev, pr, logits, res["teacher_idx"], res["teacher_logit"], workspace,
          workspace.numel())
    return res


@functools.lru_cache(maxsize=256)
def topk_workspace_size(N, V, K, dtype=KD_BF16) -> int:
    """Bytes of workspace of topk_entries and teacher_cache_write."""
    n = ctypes.c_size_t(0)
    pr = KdRows(int(N), int(V), int(V), int(K), int(dtype), 0)
    rc = load_library().kd_topk_entries_workspace_size(ctypes.byref(pr), ctypes.byref(n))
    if rc != 0:
        raise KdError(rc, "kd_topk_entries_workspace_size")
    return int(n.value)


def teacher_cache_write(logits, K, logprobs: bool = False, out=None, workspace=None):
    """kd_teacher_cache_write on the current stream: the K largest logits of
    each row as a teacher cache of 4 bytes an entry. Returns {'entries' [N, K]
    int32 (index << 12 | code), 'scale' [N, 2] fp32 (top, step)}; `out` may
    carry them, e.g. as rows of a larger cache."""
    import torch
    pr, workspace = _topk_rows(logits, K, logprobs, workspace)
    dev = logits.device
    res = _out_tensors(out, {"entries": ((pr.N, pr.K), torch.int32),
                             "scale": ((pr.N, 2), torch.float32)}, dev)
    _call("kd_teacher_cache_write", dev, pr, logits, res["entries"], res["scale"], workspace,
          workspace.numel())
    return res


def teacher_cache_read(entries, scale, rows=None, out=None):
    """kd_teacher_cache_read on the current stream: cache rows [N, K] (all of
    them, or those that `rows` [M] int64 names) as the loss's arguments
    {'teacher_idx' [M, K], 'teacher_logit' [M, K], 'ignore' [M] uint8}; ignore is
    1 for a token without a target."""
    import torch
    load_library()
    if entries.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if entries.dim() != 2:
        raise ValueError("entries must be [N, K]")
    dev = entries.device
    N, K = entries.shape
    _check_tensor("entries", entries, (N, K), torch.int32, dev)
    _check_tensor("scale", scale, (N, 2), torch.float32, dev)
    M = N
    if rows is not None:
        if rows.dim() != 1:
            raise ValueError("rows must be [M]")
        M = rows.shape[0]
        _check_tensor("rows", rows, (M,), torch.int64, dev)
    res = _out_tensors(out, {"teacher_idx": ((M, K), torch.int32),
                             "teacher_logit": ((M, K), torch.float32),
                             "ignore": ((M,), torch.uint8)}, dev)
    _call("kd_teacher_cache_read", dev, N, K, entries, scale, rows, M, res["teacher_idx"],
          res["teacher_logit"], res["ignore"])
    return res


def checkpoint_write(hidden, out=None):
    """kd_checkpoint_write on the current stream: hidden [N, D] (bf16 or fp32,
    D a multiple of 32) in 8 bits, {'codes' [N, D] uint8 (e4m3), 'scales'
    [N, D / 32] uint8 (power of two, biased by 127)}."""
    import torch
    load_library()
    if hidden.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if hidden.dim() != 2 or not hidden.is_contiguous():
        raise ValueError("hidden must be a contiguous [N, D]")
    dev, code = hidden.device, _dtype_code(hidden.dtype)
    N, D = hidden.shape
    res = _out_tensors(out, {"codes": ((N, D), torch.uint8),
                             "scales": ((N, D // 32), torch.uint8)}, dev)
    _call("kd_checkpoint_write", dev, N, D, code, hidden, res["codes"], res["scales"])
    return res


def _check_checkpoint(codes, scales):
    import torch
    if codes.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if codes.dim() != 2:
        raise ValueError("codes must be [N, D]")
    N, D = codes.shape
    _check_tensor("codes", codes, (N, D), torch.uint8, codes.device)
    _check_tensor("scales", scales, (N, D // 32), torch.uint8, codes.device)
    return N, D, codes.device


def checkpoint_read(codes, scales, dtype, out=None):
    """kd_checkpoint_read on the current stream: the hidden states [N, D] that a
    checkpoint holds, in dtype (torch.bfloat16 or torch.float32)."""
    import torch
    load_library()
    N, D, dev = _check_checkpoint(codes, scales)
    code = _dtype_code(dtype)
    hidden = torch.empty(N, D, dtype=dtype, device=dev) if out is None else out
    if out is not None:
        _check_tensor("out", hidden, (N, D), dtype, dev)
    _call("kd_checkpoint_read", dev, N, D, code, codes, scales, hidden)
    return hidden


def bwd_checkpoint(codes, scales, W, teacher_idx, teacher_logit, tau: float = 1.0, ignore=None,
                   chunk: int = 4096, grad_loss=None, grad_loss_per_token=None,
                   grad_hidden: bool = True, grad_W: bool = True, grad_W_out=None,
                   accumulate_grad_W: bool = False, workspace=None,
                   teacher_logprobs: bool = False, grad_hidden_f32: bool = False):
    """kd_topk_kl_bwd_checkpoint: gradients of the loss at the hidden states that
    a checkpoint holds (checkpoint_write's codes and scales), in W's dtype. The
    other arguments as for bwd, without a saved log-normaliser. Returns a dict
    with 'grad_hidden' and 'grad_W' as requested."""
    import torch
    lib = load_library()
    N, D, dev = _check_checkpoint(codes, scales)
    _, _, V, K, dt = _check_inputs(codes, W, teacher_idx, teacher_logit, ignore, checkpoint=True)
    if grad_loss is not None and grad_loss.numel() == 1:
        _check_tensor("grad_loss", grad_loss, tuple(grad_loss.shape), torch.float32, dev)
    elif grad_loss is not None:
        raise ValueError("grad_loss must hold one value (the upstream gradient of the mean)")
    if grad_loss_per_token is not None:
        _check_tensor("grad_loss_per_token", grad_loss_per_token, (N,), torch.float32, dev)
    res = {}
    if grad_hidden:
        res["grad_hidden"] = torch.empty(N, D, device=dev,
                                         dtype=torch.float32 if grad_hidden_f32 else W.dtype)
    if grad_W:
        res["grad_W"] = grad_W_out if grad_W_out is not None else torch.empty(
            V, D, dtype=torch.float32, device=dev)
        _check_tensor("grad_W", res["grad_W"], (V, D), torch.float32, dev)
    pr = problem(N, D, V, K, chunk, tau, dt, _flags(teacher_logprobs, grad_hidden_f32))
    if workspace is None:
        workspace = alloc_workspace(N, D, V, K, chunk, tau, dt, dev)
    _check_workspace(workspace, dev)
    with torch.cuda.device(dev):
        rc = lib.kd_topk_kl_bwd_checkpoint(
            ctypes.byref(pr), _ptr(codes), _ptr(scales), _ptr(W), _ptr(teacher_idx),
            _ptr(teacher_logit), _ptr(ignore), _ptr(grad_loss), _ptr(grad_loss_per_token),
            _ptr(res.get("grad_hidden")), _ptr(res.get("grad_W")), int(bool(accumulate_grad_W)),
            _ptr(workspace), ctypes.c_size_t(workspace.numel()), _stream_handle(dev))
    if rc != 0:
        raise KdError(rc, "kd_topk_kl_bwd_checkpoint")
    return res


def verify_draft(target_logits, draft_tokens, uniform, draft_idx=None, draft_logit=None,
                 draft_logits=None, lengths=None, tau: float = 1.0, accept_prob: bool = False,
                 out=None, workspace=None):
    """kd_verify_draft on the current stream: which drafted tokens the target
    keeps, and the token behind them.

    target_logits [B, T + 1, V] (bf16 or fp32), draft_tokens [B, T] int32,
    uniform [B, T + 1] fp32 in [0, 1); the draft's distribution as draft_idx and
    draft_logit [B, T, K] (topk_entries of its logits) or as draft_logits
    [B, T, V] in the target's dtype; lengths [B] int32 or None. Returns
    {'tokens' [B, T + 1] int32 (kept, next, then -1), 'accepted' [B] int32} and,
    when requested, 'accept_prob' [B, T] fp32."""
    import torch
    load_library()
    code, ld = _logits_rows("target_logits", target_logits, 3)
    dev = target_logits.device
    B, T, V = target_logits.shape[0], target_logits.shape[1] - 1, target_logits.shape[2]
    if T < 0:
        raise ValueError("target_logits must be [B, T + 1, V]")
    _check_tensor("draft_tokens", draft_tokens, (B, T), torch.int32, dev)
    _check_tensor("uniform", uniform, (B, T + 1), torch.float32, dev)
    if (draft_idx is None) != (draft_logit is None):
        raise ValueError("draft_idx and draft_logit go together")
    if T > 0 and (draft_idx is None) == (draft_logits is None):
        raise ValueError("the draft is either draft_idx and draft_logit, or draft_logits")
    K, ld_draft = 0, V
    if draft_idx is not None:
        if draft_idx.dim() != 3 or draft_idx.shape[2] < 1:
            raise ValueError("draft_idx must be [B, T, K]")
        K = draft_idx.shape[2]
        _check_tensor("draft_idx", draft_idx, (B, T, K), torch.int32, dev)
        _check_tensor("draft_logit", draft_logit, (B, T, K), torch.float32, dev)
    elif draft_logits is not None:
        dcode, ld_draft = _logits_rows("draft_logits", draft_logits, 3)
        if dcode != code or tuple(draft_logits.shape) != (B, T, V) or draft_logits.device != dev:
            raise ValueError("draft_logits must be [B, T, V] in the target's dtype and device")
    if lengths is not None:
        _check_tensor("lengths", lengths, (B,), torch.int32, dev)
    want = {"tokens": ((B, T + 1), torch.int32), "accepted": ((B,), torch.int32)}
    if accept_prob:
        want["accept_prob"] = ((B, T), torch.float32)
    res = _out_tensors(out, want, dev)
    pr = KdDraft(B, T, V, ld, ld_draft, K, code, float(tau), 0)
    if workspace is None:
        workspace = torch.empty(verify_workspace_size(B, T, V, K, code), dtype=torch.uint8,
                                device=dev)
    _check_workspace(workspace, dev)
    _call("kd_verify_draft", dev, pr, target_logits, draft_tokens, draft_idx, draft_logit,
          draft_logits, uniform, lengths, res["tokens"], res["accepted"], res.get("accept_prob"),
          workspace, workspace.numel())
    return res


@functools.lru_cache(maxsize=256)
def verify_workspace_size(B, T, V, K, dtype=KD_BF16) -> int:
    """Bytes of workspace of verify_draft (K = 0: a dense draft)."""
    n = ctypes.c_size_t(0)
    pr = KdDraft(int(B), int(T), int(V), int(V), int(V), int(K), int(dtype), 1.0, 0)
    rc = load_library().kd_verify_draft_workspace_size(ctypes.byref(pr), ctypes.byref(n))
    if rc != 0:
        raise KdError(rc, "kd_verify_draft_workspace_size")
    return int(n.value)


def _label_problem(hidden, W, labels, z_loss, chunk, workspace, grad_hidden_f32=False):
    """The problem and workspace of a cross entropy, with its checks."""
    import torch
    load_library()
    if hidden.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if hidden.dim() != 2 or W.dim() != 2:
        raise ValueError("hidden must be [N, D] and W [V, D]")
    dev, code = hidden.device, _dtype_code(hidden.dtype)
    if W.dtype != hidden.dtype:
        raise TypeError("hidden and W must share a dtype")
    if labels.dtype != torch.int64:
        raise TypeError("labels must be torch.int64")
    N, D = hidden.shape
    _check_tensor("hidden", hidden, (N, D), hidden.dtype, dev)
    _check_tensor("W", W, (W.shape[0], D), W.dtype, dev)
    _check_tensor("labels", labels, (N,), torch.int64, dev)
    pr = KdLabelProblem(N, D, W.shape[0], int(chunk), code, float(z_loss),
                        _flags(grad_hidden_f32=grad_hidden_f32))
    if workspace is None:
        workspace = torch.empty(ce_workspace_size(N, D, W.shape[0], int(chunk), code),
                                dtype=torch.uint8, device=dev)
    _check_workspace(workspace, dev)
    return pr, workspace, dev


@functools.lru_cache(maxsize=256)
def ce_workspace_size(N, D, V, chunk=4096, dtype=KD_BF16) -> int:
    """Bytes of workspace of cross_entropy, ce_fwd_bwd, ce_fwd and ce_bwd."""
    n = ctypes.c_size_t(0)
    pr = KdLabelProblem(int(N), int(D), int(V), int(chunk), int(dtype), 0.0, 0)
    rc = load_library().kd_cross_entropy_workspace_size(ctypes.byref(pr), ctypes.byref(n))
    if rc != 0:
        raise KdError(rc, "kd_cross_entropy_workspace_size")
    return int(n.value)


def ce_fwd_bwd(hidden, W, labels, z_loss: float = 0.0, chunk: int = 4096,
               grad_hidden: bool = True, grad_W: bool = True, loss_per_token: bool = False,
               grad_W_out=None, accumulate_grad_W: bool = False, workspace=None, out=None,
               grad_hidden_f32: bool = False):
    """kd_cross_entropy_fwd_bwd on the current stream: the mean cross entropy of
    hidden W^T [N, V] against labels [N] int64 (a label outside [0, V) is ignored),
    plus z_loss (ln Z)^2 a token, and its gradients. hidden [N, D] and W [V, D] in
    bf16 or fp32. Returns and `out` as for fwd_bwd. With grad_hidden_f32 the labels' part
    of both gradients of bf16 tensors (grad_W alone too) is formed in fp32: near a
    uniform distribution they are 3e-5 off in the 2-norm at most, else 2.3e-3."""
    import torch
    pr, workspace, dev = _label_problem(hidden, W, labels, z_loss, chunk, workspace,
                                        grad_hidden_f32)
    want = {"loss": ((), torch.float32)}
    if loss_per_token:
        want["loss_per_token"] = ((pr.N,), torch.float32)
    if grad_hidden:
        want["grad_hidden"] = ((pr.N, pr.D), torch.float32 if grad_hidden_f32 else hidden.dtype)
    if grad_W:
        want["grad_W"] = ((pr.V, pr.D), torch.float32)
        if grad_W_out is not None:
            out = {**(out or {}), "grad_W": grad_W_out}
    if accumulate_grad_W and (not grad_W or out is None or out.get("grad_W") is None):
        raise ValueError("accumulate_grad_W needs the gradient to add to (grad_W_out)")
    res = _out_tensors(out, want, dev)
    _call("kd_cross_entropy_fwd_bwd", dev, pr, hidden, W, labels, res["loss"],
          res.get("loss_per_token"), res.get("grad_hidden"), res.get("grad_W"),
          int(bool(accumulate_grad_W)), workspace, workspace.numel())
    return res


def ce_fwd(hidden, W, labels, z_loss: float = 0.0, chunk: int = 4096,
           loss_per_token: bool = False, workspace=None):
    """kd_cross_entropy_fwd: the loss without gradient work. Returns a dict with
    'loss' (0-d), 'saved_logz' [N] (ln Z, for ce_bwd) and, when requested,
    'loss_per_token' [N]."""
    import torch
    pr, workspace, dev = _label_problem(hidden, W, labels, z_loss, chunk, workspace)
    want = {"loss": ((), torch.float32), "saved_logz": ((pr.N,), torch.float32)}
    if loss_per_token:
        want["loss_per_token"] = ((pr.N,), torch.float32)
    res = _out_tensors(None, want, dev)
    _call("kd_cross_entropy_fwd", dev, pr, hidden, W, labels, res["loss"],
          res.get("loss_per_token"), res["saved_logz"], workspace, workspace.numel())
    return res


def ce_bwd(hidden, W, labels, saved_logz, z_loss: float = 0.0, chunk: int = 4096, grad_loss=None,
           grad_loss_per_token=None, grad_hidden: bool = True, grad_W: bool = True,
           grad_W_out=None, accumulate_grad_W: bool = False, workspace=None,
           grad_hidden_f32: bool = False):
    """kd_cross_entropy_bwd: gradients from ce_fwd's log-normaliser; grad_loss and
    grad_loss_per_token as for bwd. Returns a dict with 'grad_hidden' and 'grad_W' as
    requested."""
    import torch
    pr, workspace, dev = _label_problem(hidden, W, labels, z_loss, chunk, workspace,
                                        grad_hidden_f32)
    _check_tensor("saved_logz", saved_logz, (pr.N,), torch.float32, dev)
    if grad_loss is not None:
        if grad_loss.numel() != 1:
            raise ValueError("grad_loss must hold one value (the upstream gradient of the mean)")
        _check_tensor("grad_loss", grad_loss, grad_loss.shape, torch.float32, dev)
    if grad_loss_per_token is not None:
        _check_tensor("grad_loss_per_token", grad_loss_per_token, (pr.N,), torch.float32, dev)
    if accumulate_grad_W and (not grad_W or grad_W_out is None):
        raise ValueError("accumulate_grad_W needs the gradient to add to (grad_W_out)")
    want = {}
    if grad_hidden:
        want["grad_hidden"] = ((pr.N, pr.D), torch.float32 if grad_hidden_f32 else hidden.dtype)
    if grad_W:
        want["grad_W"] = ((pr.V, pr.D), torch.float32)
    res = _out_tensors(None if grad_W_out is None else {"grad_W": grad_W_out}, want, dev)
    _call("kd_cross_entropy_bwd", dev, pr, hidden, W, labels, saved_logz, grad_loss,
          grad_loss_per_token, res.get("grad_hidden"), res.get("grad_W"),
          int(bool(accumulate_grad_W)), workspace, workspace.numel())
    return res


def _ce_functions():
    import torch

    class Once(torch.autograd.Function):
        """A gradient as it is, whose own derivative is an error."""

        @staticmethod
        def forward(ctx, grad):
            return grad.view_as(grad)

        @staticmethod
        def backward(ctx, grad_out):
            raise RuntimeError("cross_entropy has no second derivative")

    def once(grad):
        """What a backward returns: with create_graph, not a constant, whose derivative
        would be taken for 0."""
        if grad is None or not torch.is_grad_enabled():
            return grad
        return Once.apply(grad.detach().requires_grad_())

    class CrossEntropy(torch.autograd.Function):
        """Mean cross entropy; forward saves ln Z, backward forms the logits again."""

        @staticmethod
        def forward(ctx, hidden, W, labels, z_loss, chunk, workspace):
            res = ce_fwd(hidden, W, labels, z_loss=z_loss, chunk=chunk, workspace=workspace)
            ctx.save_for_backward(hidden, W, labels, res["saved_logz"])
            ctx.cfg = (z_loss, chunk, workspace)
            return res["loss"]

        @staticmethod
        def backward(ctx, grad_out):
            hidden, W, labels, logz = ctx.saved_tensors
            z_loss, chunk, workspace = ctx.cfg
            res = ce_bwd(hidden, W, labels, logz, z_loss=z_loss, chunk=chunk,
                         grad_loss=grad_out.detach().to(torch.float32).contiguous(),
                         grad_hidden=ctx.needs_input_grad[0], grad_W=ctx.needs_input_grad[1],
                         workspace=workspace)
            gW = res.get("grad_W")
            return (once(res.get("grad_hidden")), once(None if gW is None else gW.to(W.dtype)),
                    None, None, None, None)

    class CrossEntropyFused(torch.autograd.Function):
        """Mean cross entropy; forward forms both gradients of the mean in fp32 with one
        projection, backward scales them and rounds each once (kd_scale_grads). One
        backward per graph."""

        @staticmethod
        def forward(ctx, hidden, W, labels, z_loss, chunk, workspace):
            need_h, need_W = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
            out = ce_fwd_bwd(hidden, W, labels, z_loss=z_loss, chunk=chunk, grad_hidden=need_h,
                             grad_W=need_W, workspace=workspace, grad_hidden_f32=True)
            ctx.grads = (out.get("grad_hidden"), out.get("grad_W"))
            ctx.dtype = hidden.dtype
            return out["loss"]

        @staticmethod
        def backward(ctx, grad_out):
            if ctx.grads is None:
                raise RuntimeError("cross_entropy(schedule='fused') supports one backward per "
                                   "graph; use schedule='recompute' to run backward again")
            (gh, gW), ctx.grads = ctx.grads, None
            g = grad_out.detach()
            if g.dtype != torch.float32:
                g = g.to(torch.float32)
            oh, oW = [x if x is None or ctx.dtype == torch.float32
                      else torch.empty_like(x, dtype=ctx.dtype) for x in (gh, gW)]
            code = _dtype_code(ctx.dtype)
            _call("kd_scale_grads", (gW if gh is None else gh).device, g, gh, code, oh,
                  0 if gh is None else gh.numel(), gW, code, oW, 0 if gW is None else gW.numel())
            return once(oh), once(oW), None, None, None, None

    return {"recompute": CrossEntropy, "fused": CrossEntropyFused}


_CE = None


def cross_entropy(hidden, W, labels, z_loss: float = 0.0, chunk: int = 4096,
                  schedule: str = "fused", workspace=None):
    """Differentiable mean cross entropy of the logits hidden W^T against labels [N]
    int64, without the logits [N, V] ever being held: the mean over the tokens whose
    label is in [0, V) of ln Z - z[label] + z_loss (ln Z)^2 (0 if there are none).
    hidden [N, D] and W [V, D] in bf16 or fp32.

    schedule and workspace (ce_workspace_size bytes) as for topk_kl_loss: "fused" forms
    both gradients in the forward with one projection and allows one backward;
    "recompute" saves ln Z only. In bf16 the labels' part of the fused gradients is formed
    in fp32; every other entry of dL/dz is held in bf16, in the recomputed ones the labels'
    too: near a uniform distribution 1.7e-3 off in the 2-norm, the final rounding, and up
    to 2.2e-3. Without a gradient wanted, the loss alone is computed. There is no
    forward-mode rule and no second derivative: tensors that carry tangents are an error,
    and so is a derivative of the gradients. Capture a step into a graph with no eager loss
    of the same hidden or W alive: torch ties their gradients to the stream of the first."""
    import torch
    global _CE
    if schedule not in ("fused", "recompute"):
        raise ValueError("schedule must be 'fused' or 'recompute'")
    tangent = torch.autograd.forward_ad.unpack_dual
    if not (torch.is_grad_enabled() and (hidden.requires_grad or W.requires_grad)) \
            and tangent(hidden).tangent is None and tangent(W).tangent is None:
        return ce_fwd_bwd(hidden, W, labels, z_loss=z_loss, chunk=chunk, grad_hidden=False,
                          grad_W=False, workspace=workspace)["loss"]
    if _CE is None:
        _CE = _ce_functions()
    # (a tensor that carries a tangent is refused here)
    return _CE[schedule].apply(hidden, W, labels, float(z_loss), int(chunk), workspace)


def mx4_write(x, out=None):
    """kd_mx4_write on the current stream: x [N, D] (bf16 or fp32, D a multiple of
    32) in 4 bits, {'codes' [N, D / 2] uint8 (two e2m1 codes a byte, the even column
    low), 'scales' [N, D / 32] uint8 (power of two, biased by 127)}. No gradient
    flows (mx4_round has one)."""
    import torch
    load_library()
    if x.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if x.dim() != 2 or not x.is_contiguous():
        raise ValueError("x must be a contiguous [N, D]")
    dev, code = x.device, _dtype_code(x.dtype)
    N, D = x.shape
    res = _out_tensors(out, {"codes": ((N, D // 2), torch.uint8),
                             "scales": ((N, D // 32), torch.uint8)}, dev)
    _call("kd_mx4_write", dev, N, D, code, x, res["codes"], res["scales"])
    return res


def _check_mx4(name, codes, scales, device=None):
    """Rows and columns of a matrix in 4 bits."""
    import torch
    if codes.device.type != "cuda":
        raise ValueError("tensors must be on a GPU")
    if codes.dim() != 2:
        raise ValueError(f"{name} must be [rows, D / 2]")
    dev = codes.device if device is None else device
    N, D = codes.shape[0], 2 * codes.shape[1]
    _check_tensor(name, codes, (N, D // 2), torch.uint8, dev)
    _check_tensor(f"scales of {name}", scales, (N, D // 32), torch.uint8, dev)
    return N, D, dev


def mx4_read(codes, scales, dtype, out=None):
    """kd_mx4_read on the current stream: the matrix [N, D] that codes and scales
    stand for, in dtype (torch.bfloat16 or torch.float32; exact in both)."""
    import torch
    load_library()
    N, D, dev = _check_mx4("codes", codes, scales)
    code = _dtype_code(dtype)
    x = torch.empty(N, D, dtype=dtype, device=dev) if out is None else out
    if out is not None:
        _check_tensor("out", x, (N, D), dtype, dev)
    _call("kd_mx4_read", dev, N, D, code, codes, scales, x)
    return x


_MX4_ROUND = None


def mx4_round(W):
    """The values that W [V, D] has in 4 bits (mx4_write, mx4_read), in W's dtype, for
    training a head that will be held so: the loss takes them, and the gradient goes to
    W as it is (straight through)."""
    import torch
    global _MX4_ROUND
    if _MX4_ROUND is None:
        class Mx4Round(torch.autograd.Function):
            @staticmethod
            def forward(ctx, W):
                q = mx4_write(W)
                return mx4_read(q["codes"], q["scales"], W.dtype)

            @staticmethod
            def backward(ctx, grad_out):
                return grad_out

        _MX4_ROUND = Mx4Round
    return _MX4_ROUND.apply(W)


def mx4_logits(hidden, codes, scales, hidden_scales=None, dtype=None, out=None, workspace=None):
    """kd_mx4_logits on the current stream: the logits [N, V] of hidden rows with a
    head in 4 bits (mx4_write's codes [V, D / 2] and scales).

    hidden [N, D] in bf16 or fp32 (rows evenly spaced, 16-byte aligned), used as it
    is, or 4-bit hidden rows: codes [N, D / 2] with hidden_scales [N, D / 32]. dtype of
    the logits: torch.bfloat16 or torch.float32; hidden's by default (bf16 for 4-bit
    rows). `out` may carry them (rows evenly spaced), `workspace` a uint8 tensor of
    mx4_workspace_size bytes. No gradient flows."""
    import torch
    load_library()
    V, D, dev = _check_mx4("codes", codes, scales)
    if hidden_scales is not None:
        N, Dh, _ = _check_mx4("hidden", hidden, hidden_scales, dev)
        code, ld = KD_MX4, Dh
    else:
        code, ld = _logits_rows("hidden", hidden, 2)
        N, Dh = hidden.shape
        if hidden.device != dev:
            raise ValueError("inputs must be on one device")
    if Dh != D:
        raise ValueError(f"hidden has {Dh} columns, the head {D}")
    if out is not None:
        dtype = out.dtype if dtype is None else dtype
        ocode, ldo = _logits_rows("out", out, 2)
        if out.shape != (N, V) or out.device != dev or out.dtype != dtype:
            raise ValueError(f"out must be a {dtype} tensor of shape {(N, V)} on {dev}")
    else:
        if dtype is None:
            dtype = torch.bfloat16 if code == KD_MX4 else hidden.dtype
        ocode, ldo = _dtype_code(dtype), V
        out = torch.empty(N, V, dtype=dtype, device=dev)
    if workspace is None:
        workspace = torch.empty(mx4_workspace_size(N, D, V, code, ld), dtype=torch.uint8,
                                device=dev)
    _check_workspace(workspace, dev)
    _call("kd_mx4_logits", dev, KdMx4Head(N, D, V, ld, ldo, code, ocode, 0), hidden, hidden_scales,
          codes, scales, out, workspace, workspace.numel())
    return out


@functools.lru_cache(maxsize=256)
def mx4_workspace_size(N, D, V, dtype=KD_BF16, ld_hidden=None) -> int:
    """Bytes of workspace of mx4_logits for N hidden rows and any fewer (dtype of the
    hidden rows, KD_MX4: 4 bits; their row stride in elements where it is not D)."""
    n = ctypes.c_size_t(0)
    pr = KdMx4Head(int(N), int(D), int(V), int(ld_hidden or D), int(V), int(dtype), KD_F32, 0)
    rc = load_library().kd_mx4_logits_workspace_size(ctypes.byref(pr), ctypes.byref(n))
    if rc != 0:
        raise KdError(rc, "kd_mx4_logits_workspace_size")
    return int(n.value)


def profile_enable(on: bool = True, contractions_only: bool = False):
    """Per-kernel HIP-event timing inside the library (instrumentation): off,
    around every kernel, or only around the contraction kernels."""
    rc = load_library().kd_profile_enable(0 if not on else (2 if contractions_only else 1))
    if rc != 0:
        raise KdError(rc, "kd_profile_enable")


def profile_read() -> dict:
    """{kernel kind: {launches, total_ms, flops}} recorded since the last read."""
    arr = (KdKernelTime * 32)()
    n = load_library().kd_profile_read(arr, 32)
    if n < 0:
        raise KdError(7, "kd_profile_read")
    return {arr[i].name.decode(): dict(launches=int(arr[i].launches),
                                       total_ms=float(arr[i].total_ms),
                                       flops=float(arr[i].flops)) for i in range(n)}
