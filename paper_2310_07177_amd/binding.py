"""Thin Python binding of libosd (include/osd.h).

The functions carry the C ABI's names and only marshal arguments: torch
supplies device memory and the current stream, every computation happens in
the HIP kernels behind the C ABI.  There is no fallback: if the library or a
GPU is missing, the call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libosd.so")

OSD_OK, OSD_ERR_INVALID_ARG, OSD_ERR_UNSUPPORTED, OSD_ERR_DEVICE, OSD_ERR_WORKSPACE, OSD_ERR_SCRATCH = 0, -1, -2, -3, -4, -5
OSD_VERIFY_NOALLOC_SCRATCH_BYTES = 4 << 20
OSD_F32, OSD_BF16 = 0, 1
OSD_FKL, OSD_RKL, OSD_JSD = 0, 1, 2
OSD_MAX_K = 16
OSD_MAX_SHARDS = 64
OSD_MAX_TREE_NODES = 64
OSD_MAX_TOPK = 256
OSD_MAX_HEAD_DIM = 256
OSD_MAX_CACHE_BATCH = 4096
OSD_ROTATE_HALVES, OSD_ROTATE_PAIRS = 0, 1
# Byte sizes of the sharded verification's records (osd_shard_row_stats,
# osd_shard_mass in include/osd.h); the binding keeps them as uint8 tensors.
SHARD_ROW_STATS_BYTES = 40
SHARD_MASS_BYTES = 48
KINDS = {"fkl": OSD_FKL, "rkl": OSD_RKL, "jsd": OSD_JSD}

EXPORTS = ("osd_max_vocab", "osd_status_string", "osd_verify_workspace_bytes", "osd_verify", "osd_verify_noalloc",
           "osd_distill_workspace_bytes", "osd_distill_loss_grad", "osd_verify_distill_workspace_bytes",
           "osd_verify_distill", "osd_verify_distill_rejected", "osd_verify_tree_workspace_bytes", "osd_verify_tree",
           "osd_sample_workspace_bytes", "osd_sample", "osd_shard_verify_stats", "osd_shard_verify_mass",
           "osd_shard_verify_draw", "osd_topk", "osd_distill_topk_workspace_bytes",
           "osd_distill_topk_loss_grad", "osd_verify_topk_workspace_bytes", "osd_verify_topk",
           "osd_cache_append", "osd_tree_attention_workspace_bytes", "osd_tree_attention", "osd_cache_keep")

_lib = None
_lock = threading.Lock()


class OsdError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn} failed: {lib().osd_status_string(status).decode()}")


def lib():
    """Load libosd.so (built in-tree by paper_2310_07177_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                                   "`python -m paper_2310_07177_amd.build`")
            L = ctypes.CDLL(LIB_PATH)
            vp, i32, i64, f32, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                     ctypes.c_float, ctypes.c_size_t)
            L.osd_max_vocab.restype = i32
            L.osd_max_vocab.argtypes = [i32]
            L.osd_status_string.restype = ctypes.c_char_p
            L.osd_status_string.argtypes = [i32]
            L.osd_verify_workspace_bytes.restype = sz
            L.osd_verify_workspace_bytes.argtypes = [i32, i32]
            L.osd_verify.restype = i32
            L.osd_verify.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, f32,
                                     vp, vp, vp, vp, sz, vp]
            L.osd_verify_noalloc.restype = i32
            L.osd_verify_noalloc.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp, vp]
            L.osd_distill_workspace_bytes.restype = sz
            L.osd_distill_workspace_bytes.argtypes = [i32, i32]
            L.osd_distill_loss_grad.restype = i32
            L.osd_distill_loss_grad.argtypes = [vp, i64, vp, i64, i32, i32, i32, i32, vp, i32,
                                                f32, f32, vp, vp, vp, vp, sz, vp]
            L.osd_verify_distill_workspace_bytes.restype = sz
            L.osd_verify_distill_workspace_bytes.argtypes = [i32, i32]
            L.osd_verify_distill.restype = i32
            L.osd_verify_distill.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp,
                                             vp, i32, f32, vp, vp, vp, vp, sz, vp]
            L.osd_verify_distill_rejected.restype = i32
            L.osd_verify_distill_rejected.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp,
                                                      vp, i32, f32, vp, vp, vp, vp, sz, vp]
            L.osd_verify_tree_workspace_bytes.restype = sz
            L.osd_verify_tree_workspace_bytes.argtypes = [i32, i32]
            L.osd_verify_tree.restype = i32
            L.osd_verify_tree.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp]
            L.osd_sample.restype = i32
            L.osd_sample_workspace_bytes.restype = sz
            L.osd_sample_workspace_bytes.argtypes = [i32]
            L.osd_sample.argtypes = [vp, i64, vp, i64, i32, i32, i32, f32, f32, vp, vp, vp, sz, vp]
            L.osd_shard_verify_stats.restype = i32
            L.osd_shard_verify_stats.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, f32, vp, vp]
            L.osd_shard_verify_mass.restype = i32
            L.osd_shard_verify_mass.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, f32, vp, vp, vp]
            L.osd_shard_verify_draw.restype = i32
            L.osd_shard_verify_draw.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, f32,
                                                vp, vp, vp, vp, vp]
            L.osd_topk.restype = i32
            L.osd_topk.argtypes = [vp, i64, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp]
            L.osd_distill_topk_workspace_bytes.restype = sz
            L.osd_distill_topk_workspace_bytes.argtypes = [i32, i32]
            L.osd_distill_topk_loss_grad.restype = i32
            L.osd_distill_topk_loss_grad.argtypes = [vp, vp, vp, i64, i32, vp, i64, i32, i32, i32, i32, vp, i32, f32,
                                                     f32, vp, vp, vp, vp, sz, vp]
            L.osd_verify_topk_workspace_bytes.restype = sz
            L.osd_verify_topk_workspace_bytes.argtypes = [i32, i32]
            L.osd_verify_topk.restype = i32
            L.osd_verify_topk.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp, vp,
                                          sz, vp]
            for f in (L.osd_cache_append, L.osd_tree_attention, L.osd_cache_keep):
                f.restype = i32
                f.argtypes = [ctypes.c_char_p, vp]
            L.osd_tree_attention_workspace_bytes.restype = sz
            L.osd_tree_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
            _lib = L
    return _lib


# The host path of a short call is as long as its kernel (verification of one
# sequence on the GPU: 10 us), so what every entry point does per call is kept to
# plain integers: no argument objects, no torch.cuda.Stream built to ask for its
# handle, one lookup of module and library (verification of one sequence, K = 4,
# V = 32000, call after call: 15.2 -> 10.6 us, the kernel's own 10.3).
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return OSD_BF16
    if t.dtype == torch.float32:
        return OSD_F32
    raise TypeError(f"logits must be bfloat16 or float32, got {t.dtype}")


def _check_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("every tensor argument must live on the GPU")


def _stream_handle(device):
    return _torch()._C._cuda_getCurrentRawStream(device.index)


# Zero-initialised workspaces, one per (device, stream, kind): the kernels leave
# them zeroed, so they are reused across calls on the same stream.  A captured graph
# holds its workspace's address, so one that a larger call supersedes is kept (sizes
# are powers of two: all of a stream's superseded ones together are smaller than the
# one in use).  A graph replayed on another stream than the one it was captured on
# must not overlap calls on that one, nor other graphs captured on it.
_workspaces = {}
# Those that hold scratch as well, of which the kernels leave the counters zero.
_scratch = {}
_superseded = []
# A workspace first needed during a capture is the graph's own: its zero fill is
# recorded, not executed, so calls outside that capture cannot use it.
# key -> (capture, workspace)
_captured = {}


def _capture_id(stream):
    """The capture that `stream` (a handle) takes part in, 0 if none (as the null stream)."""
    if not stream:
        return 0
    status, capture = ctypes.c_int(0), ctypes.c_ulonglong(0)
    err = lib().hipStreamGetCaptureInfo(ctypes.c_void_p(stream), ctypes.byref(status), ctypes.byref(capture))
    return capture.value if err == 0 and status.value == 1 else 0


def workspace(kind, nbytes, device, held=None):
    held = _workspaces if held is None else held
    key = (device.index, _stream_handle(device), kind)
    ws = held.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = _new_workspace(key, nbytes, device, held)
    return ws


def _new_workspace(key, nbytes, device, workspaces):
    torch = _torch()
    capture = _capture_id(key[1])
    if capture:
        held = _captured.get(key)
        if held is not None and held[0] == capture and held[1].numel() >= nbytes:
            return held[1]
    size = 1 << (max(int(nbytes), 256) - 1).bit_length()
    ws = torch.zeros(size, dtype=torch.uint8, device=device)
    if capture:
        _captured[key] = (capture, ws)
        return ws
    with _lock:
        _captured.pop(key, None)
        if key in workspaces:
            _superseded.append(workspaces[key])
        workspaces[key] = ws
    return ws


def osd_max_vocab(dtype_code: int) -> int:
    return lib().osd_max_vocab(dtype_code)


def osd_verify(target_logits, draft_logits, draft_tokens, u_accept, u_resample, temperature,
               draft_len=None, out=None):
    """Speculative-sampling verification through the C ABI.

    target_logits [B, K+1, V], draft_logits [B, K, V] (bf16 or fp32, on the
    GPU; draft may be None for temperature 0), draft_tokens [B, K] int32,
    u_accept [B, K] / u_resample [B] float32 (None for temperature 0),
    draft_len [B] int32 or None.  Returns (accepted_len [B], out_tokens
    [B, K+1], reject_mask [B, K]) as new (or the given `out`) GPU tensors."""
    torch = _torch()
    B, K1, V = target_logits.shape
    K = K1 - 1
    _check_cuda(target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len)
    dev = target_logits.device
    for t in (target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if draft_tokens.dtype != torch.int32 or (draft_len is not None and draft_len.dtype != torch.int32):
        raise TypeError("draft_tokens and draft_len must be int32")
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, K + 1, dtype=torch.int32, device=dev),
               torch.empty(B, K, dtype=torch.uint8, device=dev))
    acc, toks, rmask = out
    L = lib()
    nbytes = L.osd_verify_workspace_bytes(B, K)
    ws = workspace("verify", nbytes, dev)
    st = L.osd_verify(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), B, K, V,
                      _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept), _ptr(u_resample),
                      float(temperature), _ptr(acc), _ptr(toks), _ptr(rmask), _ptr(ws),
                      ws.numel(), _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify", st)
    return acc, toks, rmask


def osd_verify_noalloc(target_logits, draft_logits, draft_tokens, u_accept, u_resample, temperature,
                       draft_len=None, out=None):
    """osd_verify through the allocation-free entry point: no workspace, the
    library's per-GPU scratch array instead (calls that overlap on one GPU
    race).  Arguments and results as osd_verify; the outputs must be given
    (`out`) by a caller that cannot allocate."""
    torch = _torch()
    B, K1, V = target_logits.shape
    K = K1 - 1
    _check_cuda(target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len)
    dev = target_logits.device
    for t in (target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if draft_tokens.dtype != torch.int32 or (draft_len is not None and draft_len.dtype != torch.int32):
        raise TypeError("draft_tokens and draft_len must be int32")
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, K + 1, dtype=torch.int32, device=dev),
               torch.empty(B, K, dtype=torch.uint8, device=dev))
    acc, toks, rmask = out
    st = lib().osd_verify_noalloc(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), B, K, V,
                                  _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept), _ptr(u_resample),
                                  float(temperature), _ptr(acc), _ptr(toks), _ptr(rmask), _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify_noalloc", st)
    return acc, toks, rmask


def osd_distill_loss_grad(teacher_logits, student_logits, kind, beta=0.5, tau=1.0, mask=None,
                          B=None, K=None, teacher_batch_stride=None, student_batch_stride=None,
                          grad=True, row_loss=True, out=None):
    """Masked distillation divergence and gradient through the C ABI.

    By default teacher and student are [B, K, V]; pass B, K and explicit
    batch strides (elements) to distil the first K rows of a [B, K+1, V]
    target.  Returns (loss [2] fp32 = {mean, sum}, row_loss [B, K] fp32 or
    None, grad [B, K, V] or None)."""
    torch = _torch()
    _check_cuda(teacher_logits, student_logits, mask)
    dev = student_logits.device
    V = student_logits.shape[-1]
    if B is None:
        B, K = student_logits.shape[0], student_logits.shape[1]
    if teacher_batch_stride is None:
        teacher_batch_stride = teacher_logits.stride(0)
    if student_batch_stride is None:
        student_batch_stride = student_logits.stride(0)
    if teacher_logits.dtype != student_logits.dtype:
        raise TypeError("teacher and student logits must share a dtype")
    if mask is not None and (mask.dtype != torch.uint8 or not mask.is_contiguous()):
        raise TypeError("mask must be a contiguous uint8 tensor")
    kind_code = KINDS[kind] if isinstance(kind, str) else int(kind)
    if out is None:
        out = (torch.empty(2, dtype=torch.float32, device=dev),
               torch.empty(B, K, dtype=torch.float32, device=dev) if row_loss else None,
               torch.empty(B, K, V, dtype=student_logits.dtype, device=dev) if grad else None)
    loss, rows, g = out
    L = lib()
    nbytes = L.osd_distill_workspace_bytes(B, K)
    ws = workspace("distill", nbytes, dev)
    st = L.osd_distill_loss_grad(_ptr(teacher_logits), int(teacher_batch_stride),
                                 _ptr(student_logits), int(student_batch_stride),
                                 _dtype_code(student_logits), B, K, V, _ptr(mask), kind_code,
                                 float(beta), float(tau), _ptr(loss), _ptr(rows), _ptr(g),
                                 _ptr(ws), ws.numel(), _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_distill_loss_grad", st)
    return loss, rows, g


def osd_verify_distill(target_logits, draft_logits, draft_tokens, u_accept, u_resample, temperature,
                       kind, beta=0.5, distill_mask=None, draft_len=None, grad=True, row_loss=True):
    """Verification and distillation of one step in one pass through the C
    ABI: the results of osd_verify(...) and of osd_distill_loss_grad on the
    first K target rows and the draft rows at tau = temperature.

    Returns (accepted_len [B], out_tokens [B, K+1], reject_mask [B, K],
    loss [2], row_loss [B, K] or None, grad [B, K, V] or None)."""
    torch = _torch()
    B, K1, V = target_logits.shape
    K = K1 - 1
    _check_cuda(target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len, distill_mask)
    dev = target_logits.device
    for t in (target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len, distill_mask):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if draft_tokens.dtype != torch.int32 or (draft_len is not None and draft_len.dtype != torch.int32):
        raise TypeError("draft_tokens and draft_len must be int32")
    if target_logits.dtype != draft_logits.dtype:
        raise TypeError("target and draft logits must share a dtype")
    if distill_mask is not None and distill_mask.dtype != torch.uint8:
        raise TypeError("distill_mask must be uint8")
    kind_code = KINDS[kind] if isinstance(kind, str) else int(kind)
    acc = torch.empty(B, dtype=torch.int32, device=dev)
    toks = torch.empty(B, K + 1, dtype=torch.int32, device=dev)
    rmask = torch.empty(B, K, dtype=torch.uint8, device=dev)
    loss = torch.empty(2, dtype=torch.float32, device=dev)
    rows = torch.empty(B, K, dtype=torch.float32, device=dev) if row_loss else None
    g = torch.empty(B, K, V, dtype=draft_logits.dtype, device=dev) if grad else None
    L = lib()
    ws = workspace("verify_distill", L.osd_verify_distill_workspace_bytes(B, K), dev)
    st = L.osd_verify_distill(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), B, K, V,
                              _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept), _ptr(u_resample),
                              float(temperature), _ptr(acc), _ptr(toks), _ptr(rmask), _ptr(distill_mask),
                              kind_code, float(beta), _ptr(loss), _ptr(rows), _ptr(g), _ptr(ws), ws.numel(),
                              _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify_distill", st)
    return acc, toks, rmask, loss, rows, g


def osd_verify_distill_rejected(target_logits, draft_logits, draft_tokens, u_accept, u_resample, temperature,
                                kind, beta=0.5, draft_len=None, grad=True, row_loss=True):
    """Verification and distillation of the row at each sequence's first
    rejection (the error index), in one pass through the C ABI: the results
    of osd_verify(...) and of osd_distill_loss_grad with mask = reject_mask
    at tau = temperature.  Returns what osd_verify_distill returns."""
    torch = _torch()
    B, K1, V = target_logits.shape
    K = K1 - 1
    _check_cuda(target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len)
    dev = target_logits.device
    for t in (target_logits, draft_logits, draft_tokens, u_accept, u_resample, draft_len):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if draft_tokens.dtype != torch.int32 or (draft_len is not None and draft_len.dtype != torch.int32):
        raise TypeError("draft_tokens and draft_len must be int32")
    if target_logits.dtype != draft_logits.dtype:
        raise TypeError("target and draft logits must share a dtype")
    kind_code = KINDS[kind] if isinstance(kind, str) else int(kind)
    acc = torch.empty(B, dtype=torch.int32, device=dev)
    toks = torch.empty(B, K + 1, dtype=torch.int32, device=dev)
    rmask = torch.empty(B, K, dtype=torch.uint8, device=dev)
    loss = torch.empty(2, dtype=torch.float32, device=dev)
    rows = torch.empty(B, K, dtype=torch.float32, device=dev) if row_loss else None
    g = torch.empty(B, K, V, dtype=draft_logits.dtype, device=dev) if grad else None
    L = lib()
    ws = workspace("verify_distill", L.osd_verify_distill_workspace_bytes(B, K), dev)
    st = L.osd_verify_distill_rejected(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), B, K,
                                       V, _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept), _ptr(u_resample),
                                       float(temperature), _ptr(acc), _ptr(toks), _ptr(rmask), kind_code,
                                       float(beta), _ptr(loss), _ptr(rows), _ptr(g), _ptr(ws), ws.numel(),
                                       _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify_distill_rejected", st)
    return acc, toks, rmask, loss, rows, g


def osd_verify_tree(target_logits, draft_logits, parent, node_tokens, u_accept, u_resample, temperature):
    """Multi-candidate (tree) verification through the C ABI.  target_logits,
    draft_logits [B, N, V] (draft may be None at temperature 0), parent and
    node_tokens [B, N] int32, u_accept [B, N] and u_resample [B] float32 (None
    at temperature 0).  Returns (accepted_len [B], out_tokens [B, N],
    path_nodes [B, N])."""
    torch = _torch()
    B, N, V = target_logits.shape
    _check_cuda(target_logits, draft_logits, parent, node_tokens, u_accept, u_resample)
    dev = target_logits.device
    for t in (target_logits, draft_logits, parent, node_tokens, u_accept, u_resample):
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if parent.dtype != torch.int32 or node_tokens.dtype != torch.int32:
        raise TypeError("parent and node_tokens must be int32")
    acc = torch.empty(B, dtype=torch.int32, device=dev)
    toks = torch.empty(B, N, dtype=torch.int32, device=dev)
    nodes = torch.empty(B, N, dtype=torch.int32, device=dev)
    L = lib()
    ws = workspace("verify_tree", L.osd_verify_tree_workspace_bytes(B, N), dev)
    st = L.osd_verify_tree(_ptr(target_logits), _ptr(draft_logits), _dtype_code(target_logits), B, N, V,
                           _ptr(parent), _ptr(node_tokens), _ptr(u_accept), _ptr(u_resample), float(temperature),
                           _ptr(acc), _ptr(toks), _ptr(nodes), _ptr(ws), ws.numel(), _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify_tree", st)
    return acc, toks, nodes


def osd_sample(p_logits, q_logits, temperature, beta, u=None, out=None):
    """Token sampling through the C ABI: pi = beta softmax(p/T) +
    (1 - beta) softmax(q/T) per row, inverse CDF with u (argmax at T == 0).

    p_logits, q_logits: [N, V] bf16 or fp32 GPU tensors whose rows are
    contiguous (a row stride other than V is passed through, e.g. a slice
    [:, i, :] of a [B, K+1, V] tensor); either may be None when its weight is
    0.  u: [N] float32 (None at T == 0).  Returns out_tokens [N] int32."""
    torch = _torch()
    ref = p_logits if p_logits is not None else q_logits
    if ref is None:
        raise ValueError("p_logits or q_logits is needed")
    _check_cuda(p_logits, q_logits, u)
    for t in (p_logits, q_logits):
        if t is not None and (t.dim() != 2 or t.stride(1) != 1 or t.dtype != ref.dtype or t.shape != ref.shape):
            raise ValueError("logit rows must be [N, V] views of one dtype with contiguous rows")
    if u is not None and (u.dtype != torch.float32 or not u.is_contiguous()):
        raise TypeError("u must be a contiguous float32 tensor")
    N, V = ref.shape
    if out is None:
        out = torch.empty(N, dtype=torch.int32, device=ref.device)
    stride = lambda t: 0 if t is None else (t.stride(0) if N > 1 else V)
    L = lib()
    ws = workspace("sample", L.osd_sample_workspace_bytes(N), ref.device)
    st = L.osd_sample(_ptr(p_logits), stride(p_logits), _ptr(q_logits), stride(q_logits),
                      _dtype_code(ref), N, V, float(temperature), float(beta), _ptr(u), _ptr(out),
                      _ptr(ws), ws.numel(), _stream_handle(ref.device))
    if st != OSD_OK:
        raise OsdError("osd_sample", st)
    return out


def _shard_args(target_shard, draft_shard, draft_tokens, draft_len, temperature, *more):
    torch = _torch()
    _check_cuda(target_shard, draft_shard, draft_tokens, draft_len, *more)
    for t in (target_shard, draft_shard, draft_tokens, draft_len) + more:
        if t is not None and not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
    if draft_tokens.dtype != torch.int32 or (draft_len is not None and draft_len.dtype != torch.int32):
        raise TypeError("draft_tokens and draft_len must be int32")
    if temperature != 0 and draft_shard is not None and draft_shard.dtype != target_shard.dtype:
        raise TypeError("target and draft logits must share a dtype")
    B, K1, Vs = target_shard.shape
    return B, K1 - 1, Vs


def osd_shard_verify_stats(target_shard, draft_shard, draft_tokens, temperature, v_begin, V, draft_len=None,
                           out=None):
    """Phase 1 of vocabulary-sharded verification on this rank's slice
    (target_shard [B, K+1, V_g], draft_shard [B, K, V_g], columns
    v_begin .. v_begin+V_g-1 of a V-token vocabulary).  Returns the
    osd_shard_row_stats records as a uint8 tensor [B, K+1, 40]."""
    torch = _torch()
    B, K, Vs = _shard_args(target_shard, draft_shard, draft_tokens, draft_len, temperature)
    if out is None:
        out = torch.empty(B, K + 1, SHARD_ROW_STATS_BYTES, dtype=torch.uint8, device=target_shard.device)
    st = lib().osd_shard_verify_stats(_ptr(target_shard), _ptr(draft_shard), _dtype_code(target_shard), B, K, Vs,
                                      int(v_begin), int(V), _ptr(draft_tokens), _ptr(draft_len),
                                      float(temperature), _ptr(out), _stream_handle(target_shard.device))
    if st != OSD_OK:
        raise OsdError("osd_shard_verify_stats", st)
    return out


def osd_shard_verify_mass(target_shard, draft_shard, draft_tokens, u_accept, temperature, stats_all,
                          draft_len=None, out=None):
    """Phase 2: stats_all [G, B, K+1, 40] holds the records of every rank in
    rank order (the all-gather of phase 1).  Returns this rank's
    osd_shard_mass records as a uint8 tensor [B, 48]."""
    torch = _torch()
    B, K, Vs = _shard_args(target_shard, draft_shard, draft_tokens, draft_len, temperature, u_accept, stats_all)
    G = stats_all.shape[0]
    if tuple(stats_all.shape) != (G, B, K + 1, SHARD_ROW_STATS_BYTES) or stats_all.dtype != torch.uint8:
        raise ValueError("stats_all must be a uint8 tensor [G, B, K+1, 40]")
    if out is None:
        out = torch.empty(B, SHARD_MASS_BYTES, dtype=torch.uint8, device=target_shard.device)
    st = lib().osd_shard_verify_mass(_ptr(target_shard), _ptr(draft_shard), _dtype_code(target_shard), B, K, Vs,
                                     G, _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept), float(temperature),
                                     _ptr(stats_all), _ptr(out), _stream_handle(target_shard.device))
    if st != OSD_OK:
        raise OsdError("osd_shard_verify_mass", st)
    return out


def osd_shard_verify_draw(target_shard, draft_shard, draft_tokens, u_resample, temperature, v_begin, shard,
                          mass_all, draft_len=None, out=None):
    """Phase 3: mass_all [G, B, 48] holds every rank's phase-2 records in rank
    order.  Returns (accepted_len [B], out_tokens [B, K+1], reject_mask
    [B, K]); out_tokens carries the extra token only on the rank that drew
    it (-1 on the others), so an all-reduce MAX over the ranks completes it."""
    torch = _torch()
    B, K, Vs = _shard_args(target_shard, draft_shard, draft_tokens, draft_len, temperature, u_resample, mass_all)
    G = mass_all.shape[0]
    if tuple(mass_all.shape) != (G, B, SHARD_MASS_BYTES) or mass_all.dtype != torch.uint8:
        raise ValueError("mass_all must be a uint8 tensor [G, B, 48]")
    dev = target_shard.device
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, K + 1, dtype=torch.int32, device=dev),
               torch.empty(B, K, dtype=torch.uint8, device=dev))
    acc, toks, rmask = out
    st = lib().osd_shard_verify_draw(_ptr(target_shard), _ptr(draft_shard), _dtype_code(target_shard), B, K, Vs,
                                     int(v_begin), G, int(shard), _ptr(draft_tokens), _ptr(draft_len),
                                     _ptr(u_resample), float(temperature), _ptr(mass_all), _ptr(acc), _ptr(toks),
                                     _ptr(rmask), _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_shard_verify_draw", st)
    return acc, toks, rmask


def _check_same_device(dev, *ts):
    """Every tensor given lives on the GPU `dev`."""
    for t in ts:
        if t is not None and (not t.is_cuda or t.device != dev):
            raise ValueError("every tensor argument must live on one GPU")


def _on_device(dev, fn, *args):
    """fn(*args) with `dev` as the current device (a launch goes to the current
    device's queues)."""
    torch = _torch()
    if torch._C._cuda_getDevice() == dev.index:
        return fn(*args)
    with torch.cuda.device(dev):
        return fn(*args)


def _check_out(t, shape, dtype, name):
    if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")


def osd_topk(logits, k, temperature=1.0, u=None, rest=True, tokens=None, out=None):
    """The record of each row of logits through the C ABI: its k largest
    logits with their ids, the log mass of the others relative to the first
    slot's, and a token drawn from the record.

    logits: [N, V] bf16 or fp32 GPU tensor with contiguous rows (any row
    stride, e.g. a slice [:, i, :] of a [B, K, V] tensor).  u: [N] float32
    uniforms; given, or with tokens=True (the argmax at T == 0), a token is
    drawn.  Returns (ids [N, k] int32, top [N, k] like logits, rest [N]
    float32 or None, tokens [N] int32 or None) as new (or the given `out`)
    tensors; pass rest=False at T == 0."""
    torch = _torch()
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be a [N, V] tensor with contiguous rows")
    N, V = logits.shape
    dev = logits.device
    _check_same_device(dev, logits, u)
    if u is not None:
        _check_out(u, (N,), torch.float32, "u")
    if tokens is None:
        tokens = u is not None
    k = int(k)
    if out is None:
        out = (torch.empty(N, k, dtype=torch.int32, device=dev),
               torch.empty(N, k, dtype=logits.dtype, device=dev),
               torch.empty(N, dtype=torch.float32, device=dev) if rest else None,
               torch.empty(N, dtype=torch.int32, device=dev) if tokens else None)
        ids, top, rst, toks = out
    else:
        ids, top, rst, toks = out
        _check_same_device(dev, *out)
        _check_out(ids, (N, k), torch.int32, "ids")
        _check_out(top, (N, k), logits.dtype, "top")
        _check_out(rst, (N,), torch.float32, "rest")
        _check_out(toks, (N,), torch.int32, "tokens")
    st = _on_device(dev, lib().osd_topk, _ptr(logits), logits.stride(0) if N > 1 else V, _dtype_code(logits), N, V, k,
                    float(temperature), _ptr(u), _ptr(ids), _ptr(top), _ptr(rst), _ptr(toks),
                    _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_topk", st)
    return ids, top, rst, toks


def osd_distill_topk_loss_grad(teacher_ids, teacher_top, teacher_rest, student_logits, kind, beta=0.5, tau=1.0,
                               mask=None, grad=True, row_loss=True, out=None):
    """Distillation divergence and gradient against teacher records through
    the C ABI.

    teacher_ids [B, Kt, k] int32, teacher_top [B, Kt, k] and teacher_rest
    [B, Kt] float32 or None: records as osd_topk returns them, Kt >= K (the
    first K of each sequence are distilled, so a [B, K+1] target's records
    serve as they are).  student_logits [B, K, V] with rows one after another
    (any batch stride).  Returns (loss [2] float32 = {mean, sum}, row_loss
    [B, K] float32 or None, grad [B, K, V] or None)."""
    torch = _torch()
    if student_logits.dim() != 3 or teacher_ids.dim() != 3:
        raise ValueError("student_logits must be [B, K, V], teacher_ids [B, Kt, k]")
    B, K, V = student_logits.shape
    Kt, k = teacher_ids.shape[1:]
    dev = student_logits.device
    _check_same_device(dev, student_logits, teacher_ids, teacher_top, teacher_rest, mask)
    s = student_logits
    if (V > 1 and s.stride(2) != 1) or (K > 1 and s.stride(1) != V):
        raise ValueError("the student's rows must lie one after another")
    if Kt < K or teacher_ids.shape[0] != B:
        raise ValueError("teacher records must be [B, Kt, k] with Kt >= K")
    if teacher_top.dtype != s.dtype:
        raise TypeError("teacher_top and student logits must share a dtype")
    _check_out(teacher_ids, (B, Kt, k), torch.int32, "teacher_ids")
    _check_out(teacher_top, (B, Kt, k), s.dtype, "teacher_top")
    _check_out(teacher_rest, (B, Kt), torch.float32, "teacher_rest")
    _check_out(mask, (B, K), torch.uint8, "mask")
    kind_code = KINDS[kind] if isinstance(kind, str) else int(kind)
    if out is None:
        out = (torch.empty(2, dtype=torch.float32, device=dev),
               torch.empty(B, K, dtype=torch.float32, device=dev) if row_loss else None,
               torch.empty(B, K, V, dtype=s.dtype, device=dev) if grad else None)
        loss, rows, g = out
    else:
        loss, rows, g = out
        _check_same_device(dev, *out)
        _check_out(loss, (2,), torch.float32, "loss")
        _check_out(rows, (B, K), torch.float32, "row_loss")
        _check_out(g, (B, K, V), s.dtype, "grad")
    L = lib()
    ws = workspace("distill_topk", L.osd_distill_topk_workspace_bytes(B, K), dev, _scratch)
    st = _on_device(dev, L.osd_distill_topk_loss_grad, _ptr(teacher_ids), _ptr(teacher_top), _ptr(teacher_rest), Kt, k,
                    _ptr(s), s.stride(0) if B > 1 else K * V, _dtype_code(s), B, K, V, _ptr(mask), kind_code,
                    float(beta), float(tau), _ptr(loss), _ptr(rows), _ptr(g), _ptr(ws), ws.numel(),
                    _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_distill_topk_loss_grad", st)
    return loss, rows, g


def osd_verify_topk(target_logits, draft_ids, draft_top, draft_tokens, u_accept, u_resample, temperature,
                    draft_len=None, out=None):
    """Verification of proposals drawn from the draft's records through the
    C ABI.

    target_logits [B, K+1, V]; draft_ids [B, K, k] int32 and draft_top
    [B, K, k]: the records (osd_topk at the same temperature) that
    draft_tokens [B, K] int32 were drawn from; the other arguments and the
    results as osd_verify, temperature > 0."""
    torch = _torch()
    if target_logits.dim() != 3 or draft_ids.dim() != 3:
        raise ValueError("target_logits must be [B, K+1, V], draft_ids [B, K, k]")
    B, K1, V = target_logits.shape
    K, k = K1 - 1, draft_ids.shape[2]
    dev = target_logits.device
    _check_same_device(dev, target_logits, draft_ids, draft_top, draft_tokens, u_accept, u_resample, draft_len)
    if not target_logits.is_contiguous():
        raise ValueError("tensor arguments must be contiguous")
    if draft_top.dtype != target_logits.dtype:
        raise TypeError("target logits and draft_top must share a dtype")
    _check_out(draft_ids, (B, K, k), torch.int32, "draft_ids")
    _check_out(draft_top, (B, K, k), target_logits.dtype, "draft_top")
    _check_out(draft_tokens, (B, K), torch.int32, "draft_tokens")
    _check_out(u_accept, (B, K), torch.float32, "u_accept")
    _check_out(u_resample, (B,), torch.float32, "u_resample")
    _check_out(draft_len, (B,), torch.int32, "draft_len")
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, K + 1, dtype=torch.int32, device=dev),
               torch.empty(B, K, dtype=torch.uint8, device=dev))
        acc, toks, rmask = out
    else:
        acc, toks, rmask = out
        _check_same_device(dev, *out)
        _check_out(acc, (B,), torch.int32, "accepted_len")
        _check_out(toks, (B, K + 1), torch.int32, "out_tokens")
        _check_out(rmask, (B, K), torch.uint8, "reject_mask")
    L = lib()
    ws = workspace("verify_topk", L.osd_verify_topk_workspace_bytes(B, K), dev, _scratch)
    st = _on_device(dev, L.osd_verify_topk, _ptr(target_logits), _ptr(draft_ids), _ptr(draft_top), k,
                    _dtype_code(target_logits), B, K, V, _ptr(draft_tokens), _ptr(draft_len), _ptr(u_accept),
                    _ptr(u_resample), float(temperature), _ptr(acc), _ptr(toks), _ptr(rmask), _ptr(ws), ws.numel(),
                    _stream_handle(dev))
    if st != OSD_OK:
        raise OsdError("osd_verify_topk", st)
    return acc, toks, rmask


# The structs of the calls on the paged cache (osd_append, osd_attention and osd_keep in
# include/osd.h), packed at once: an argument of a ctypes call costs 0.1 us.
_CACHE = "=5q8i"
_APPEND = struct.Struct(_CACHE + "11q4i")
_ATTENTION = struct.Struct(_CACHE + "7qif")
_KEEP = struct.Struct(_CACHE + "4q2i")


def _page_strides(t):
    """Strides of a cache, None if a page is not contiguous.  Those of axes of one
    element say nothing; they become what a contiguous tensor has."""
    shape, stride, step = t.shape, list(t.stride()), 1
    for i in range(len(shape) - 1, -1, -1):
        if shape[i] == 1:
            stride[i] = step
        elif i >= len(shape) - 3 and stride[i] != step:
            return None
        step = stride[i] * shape[i]
    return tuple(stride)


def _cache_args(k_cache, v_cache, page_table, seq_len, layers):
    """The C ABI's description of a paged cache, checked; `layers`: its leading axes."""
    torch = _torch()
    shape, stride = k_cache.shape, k_cache.stride()
    if len(shape) != 4 + layers or v_cache.shape != shape:
        raise ValueError("the caches must be two " + ("[layers, " if layers else "[")
                         + "pages, kv_heads, page_size, head_dim] tensors of one shape")
    if v_cache.dtype != k_cache.dtype:
        raise TypeError("the caches must share a dtype")
    P, H, S, D = shape[layers:]
    if v_cache.stride() != stride or stride[-3:] != (S * D, D, 1) or P == 1:
        stride = _page_strides(k_cache)
        if stride is None or _page_strides(v_cache) != stride:
            raise ValueError("a page must be contiguous, and the caches' strides the same")
    int32 = torch.int32
    at = page_table.shape
    if len(at) != 2 or page_table.dtype != int32 or not page_table.is_contiguous():
        raise ValueError("page_table must be a contiguous int32 tensor [B, pages of a sequence]")
    _check_out(seq_len, at[:1], int32, "seq_len")
    return at[0], at[1], stride[layers], P, H, S, D, _dtype_code(k_cache)


def _token_stride(t, B, N, H, D, dtype, name):
    """Elements between the tokens of a [B, N, H, D] tensor."""
    if t.shape != (B, N, H, D) or t.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {(B, N, H, D)}")
    s = t.stride()
    step = s[1] if N > 1 else s[0] if B > 1 else H * D
    if s[3] != 1 or (H > 1 and s[2] != D) or (B > 1 and s[0] != N * step):
        raise ValueError(f"{name}: a token's heads must lie one after another, tokens at one distance")
    return step


def _one_gpu(*ts):
    """The GPU that all tensors given live on (its index)."""
    at = ts[0].get_device()
    for t in ts:
        if t is not None and t.get_device() != at:
            at = -1
    if at < 0:
        raise ValueError("every tensor argument must live on one GPU")
    return at


def _cache_call(name, call, at):
    """One of the calls on the cache, on the GPU `at`, on its current stream."""
    c = _torch()._C
    fn = getattr(lib(), name)
    if c._cuda_getDevice() == at:
        st = fn(call, c._cuda_getCurrentRawStream(at))
    else:
        with _torch().cuda.device(at):
            st = fn(call, c._cuda_getCurrentRawStream(at))
    if st != OSD_OK:
        raise OsdError(name, st)


def osd_cache_append(k, v, k_cache, v_cache, page_table, seq_len, q=None, rotation=None, pairs=False, parent=None,
                     new_len=None, q_out=None):
    """New tokens' keys and values into the paged cache through the C ABI,
    rotated by their positions on the way, their queries along with them.

    k, v [B, N, kv_heads, head_dim] and q [B, N, q_heads, head_dim] or None:
    bf16 or fp32, a token's heads one after another (slices of one projection
    serve as they are).  k_cache, v_cache [pages, kv_heads, page_size,
    head_dim] like them (any distance between pages), page_table [B, T] and
    seq_len [B] int32 (context lengths; -1: no sequence).  rotation: [rows,
    rotary_dim] float32, the cosines, then the sines of a position's angles, or
    None; pairs: of elements side by side instead of the two halves.  parent
    [B, N] int32 as osd_verify_tree takes it, or None: a chain.  new_len [B]
    int32: how many of the N tokens a sequence has.  Returns the rotated
    queries (new, or `q_out`, which may be q) or None."""
    B, table_len, page_stride, P, H, S, D, code = _cache_args(k_cache, v_cache, page_table, seq_len, 0)
    at = _one_gpu(k_cache, v_cache, k, v, page_table, seq_len, q, rotation, parent, new_len, q_out)
    if k.dim() != 4 or (q is not None and q.dim() != 4):
        raise ValueError("k, v and q must be [B, N, heads, head_dim]")
    N, dt = k.shape[1], k_cache.dtype
    k_step, v_step = _token_stride(k, B, N, H, D, dt, "k"), _token_stride(v, B, N, H, D, dt, "v")
    Hq = q_step = out_step = qp = op = rows = R = rp = 0
    if q is not None:
        Hq = q.shape[2]
        q_step, qp = _token_stride(q, B, N, Hq, D, dt, "q"), q.data_ptr()
        if q_out is None:
            q_out = q.new_empty((B, N, Hq, D))
            out_step = Hq * D
        else:
            out_step = _token_stride(q_out, B, N, Hq, D, dt, "q_out")
        op = q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    if rotation is not None:
        if rotation.dim() != 2:
            raise ValueError("rotation must be [positions, rotary_dim]")
        rows, R = rotation.shape
        _check_out(rotation, (rows, R), _torch().float32, "rotation")
        rp = rotation.data_ptr()
    _check_out(parent, (B, N), _torch().int32, "parent")
    _check_out(new_len, (B,), _torch().int32, "new_len")
    _cache_call("osd_cache_append", _APPEND.pack(
        k_cache.data_ptr(), v_cache.data_ptr(), page_stride, page_table.data_ptr(), seq_len.data_ptr(), P, S, H, D,
        code, table_len, B, N, qp, q_step, op, out_step, k.data_ptr(), k_step, v.data_ptr(), v_step, _ptr(parent) or 0,
        _ptr(new_len) or 0, rp, Hq, rows, R, OSD_ROTATE_PAIRS if pairs else OSD_ROTATE_HALVES), at)
    return q_out


def osd_tree_attention(q, k_cache, v_cache, page_table, seq_len, parent=None, new_len=None, scale=None, out=None):
    """Attention of drafted tokens through the C ABI: every node of a tree (or
    chain: parent None) over the context, its ancestors and itself, all in the
    paged cache.

    q [B, N, q_heads, head_dim] (any distance between tokens), the other
    arguments as osd_cache_append; scale: 1 / sqrt(head_dim) by default.
    Returns [B, N, q_heads, head_dim] as a new (or the given `out`) tensor."""
    B, table_len, page_stride, P, H, S, D, code = _cache_args(k_cache, v_cache, page_table, seq_len, 0)
    at = _one_gpu(q, k_cache, v_cache, page_table, seq_len, parent, new_len, out)
    if q.dim() != 4:
        raise ValueError("q must be [B, N, q_heads, head_dim]")
    N, Hq = q.shape[1:3]
    step = _token_stride(q, B, N, Hq, D, k_cache.dtype, "q")
    _check_out(parent, (B, N), _torch().int32, "parent")
    _check_out(new_len, (B,), _torch().int32, "new_len")
    if out is None:
        out = q.new_empty((B, N, Hq, D))
    else:
        _check_out(out, (B, N, Hq, D), q.dtype, "out")
    ws = workspace("tree_attention", lib().osd_tree_attention_workspace_bytes(B, N, Hq, H, D), q.device, _scratch)
    _cache_call("osd_tree_attention", _ATTENTION.pack(
        k_cache.data_ptr(), v_cache.data_ptr(), page_stride, page_table.data_ptr(), seq_len.data_ptr(), P, S, H, D,
        code, table_len, B, N, q.data_ptr(), step, _ptr(parent) or 0, _ptr(new_len) or 0, out.data_ptr(),
        ws.data_ptr(), ws.numel(), Hq, D ** -0.5 if scale is None else float(scale)), at)
    return out


def osd_cache_keep(k_cache, v_cache, page_table, seq_len, path_nodes, accepted_len, out=None):
    """The accepted path of each sequence's tree moves to where its context
    ends, through the C ABI, in the caches of all layers at once.

    k_cache, v_cache [layers, pages, kv_heads, page_size, head_dim] (one
    layer: without the first axis), path_nodes [B, N] and accepted_len [B]
    int32 as osd_verify_tree returns them.  Returns the new context lengths [B]
    int32 (a new tensor, or the given `out`, no part of the arguments)."""
    if k_cache.dim() == 4:
        layers = 1
        B, table_len, page_stride, P, H, S, D, code = _cache_args(k_cache, v_cache, page_table, seq_len, 0)
        layer_stride = 0
    else:
        B, table_len, page_stride, P, H, S, D, code = _cache_args(k_cache, v_cache, page_table, seq_len, 1)
        layers = k_cache.shape[0]
        layer_stride = k_cache.stride(0) if layers > 1 else 0
    at = _one_gpu(k_cache, v_cache, page_table, seq_len, path_nodes, accepted_len, out)
    if path_nodes.dim() != 2:
        raise ValueError("path_nodes must be [B, N]")
    N = path_nodes.shape[1]
    _check_out(path_nodes, (B, N), _torch().int32, "path_nodes")
    _check_out(accepted_len, (B,), _torch().int32, "accepted_len")
    if out is None:
        out = seq_len.new_empty((B,))
    else:
        _check_out(out, (B,), _torch().int32, "out")
    _cache_call("osd_cache_keep", _KEEP.pack(
        k_cache.data_ptr(), v_cache.data_ptr(), page_stride, page_table.data_ptr(), seq_len.data_ptr(), P, S, H, D,
        code, table_len, B, N, layer_stride, path_nodes.data_ptr(), accepted_len.data_ptr(), out.data_ptr(), layers, 0),
        at)
    return out
