"""Python binding of the C-ABI library declared in ``include/paep.h``.

Argument marshalling only: tensors (PyTorch-ROCm, used for device memory and
streams and nothing else) are checked, their device pointers and the current
HIP stream are handed to the C entry points of the same names, and a non-zero
status becomes an exception.  There is no fallback: if ``libpaep.so`` has not
been built (``python -m paper_2511_10676_amd.build``), loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpaep.so")

# enums of paep.h
F32, BF16 = 0, 1
ACT = {"none": 0, "silu": 1, "gelu": 2}
PATH = {"auto": 0, "simple": 1, "decode": 2, "prefill": 3}
PATH_NAME = {v: k for k, v in PATH.items()}
PROB = {"softmax": 0, "softmax_topk": 1, "sigmoid": 2}
TILE_CFG = {0: "128x128", 1: "128x128 wide", 2: "256x256", 3: "256x128", 4: "256x256 wide", 5: "64x64",
            6: "two-pass 256x256", 7: "128-256x256"}
MAX_K, MAX_E = 32, 1024

STATUS_NAMES = ["PAEP_OK", "PAEP_ERR_NULL", "PAEP_ERR_SHAPE", "PAEP_ERR_K", "PAEP_ERR_DTYPE",
                "PAEP_ERR_ALIGN", "PAEP_ERR_WORKSPACE", "PAEP_ERR_HIP", "PAEP_ERR_UNSUPPORTED"]

STATIC_SCRATCH_BYTES = 16 << 20

EXPORTS = ["paep_predict_workspace_bytes", "paep_predict_workspace_min_bytes", "paep_predict_resolve_path", "paep_predict_plan",
           "paep_predict_kernel", "paep_predict",
           "paep_static_init", "paep_predict_static",
           "paep_predict_counted", "paep_predict_confidence", "paep_fold_batchnorm",
           "paep_group_workspace_bytes", "paep_group_by_expert", "paep_score",
           "paep_score_rows", "paep_confidence_select", "paep_activation_profile", "paep_probe_read",
           "paep_probe_mfma", "paep_status_string", "paep_version",
           "paep_attend_workspace_bytes", "paep_attend", "paep_cache_append", "paep_cache_evict",
           "paep_moe_workspace_bytes", "paep_moe_layer", "paep_moe_experts"]


class PredictDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("r", ctypes.c_int32),
                ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("L", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("path", ctypes.c_int32),
                ("prob", ctypes.c_int32),
                ("x_layer_stride", ctypes.c_int64), ("w1_layer_stride", ctypes.c_int64),
                ("w2_layer_stride", ctypes.c_int64)]


class CacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hkv", "Dk", "Dv", "page_size", "n_pages", "max_pages", "dtype")] + \
               [(n, ctypes.c_int64) for n in ("k_page_stride", "k_head_stride", "k_slot_stride",
                                              "v_page_stride", "v_head_stride", "v_slot_stride")]


# the same bytes as the two structures, in a third of the time
_CACHE_BYTES, _ATTEND_BYTES = struct.Struct("8i6q"), struct.Struct("2ifi3q")


class AttendDesc(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("max_len", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("q_seq_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64), ("mass_stride", ctypes.c_int64)]


class MoeDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "d", "f", "E", "k", "dtype", "act", "prob")]


class PaepError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        try:
            msg = lib().paep_status_string(status).decode()
        except Exception:  # pragma: no cover
            msg = ""
        super().__init__(f"{where}: {name} ({msg})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2511_10676_amd.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        dp = ctypes.POINTER(PredictDesc)
        L.paep_predict_workspace_bytes.argtypes = [dp]
        L.paep_predict_workspace_bytes.restype = sz
        L.paep_predict_workspace_min_bytes.argtypes = [dp]
        L.paep_predict_workspace_min_bytes.restype = sz
        L.paep_predict_resolve_path.argtypes = [dp]
        L.paep_predict_resolve_path.restype = ctypes.c_int
        L.paep_predict.argtypes = [dp] + [vp] * 9 + [sz, vp]
        L.paep_predict.restype = ctypes.c_int
        L.paep_predict_counted.argtypes = [dp] + [vp] * 10 + [sz, vp]
        L.paep_predict_counted.restype = ctypes.c_int
        L.paep_predict_confidence.argtypes = [dp] + [vp] * 11 + [sz, vp]
        L.paep_predict_confidence.restype = ctypes.c_int
        L.paep_predict_static.argtypes = [dp] + [vp] * 8 + [vp]
        L.paep_predict_static.restype = ctypes.c_int
        L.paep_static_init.argtypes = []
        L.paep_static_init.restype = ctypes.c_int
        L.paep_predict_plan.argtypes = [dp, i32, ctypes.POINTER(ctypes.c_int32 * 4)]
        L.paep_predict_plan.restype = ctypes.c_int
        L.paep_predict_kernel.argtypes = [dp, i32, i32, sz]
        L.paep_predict_kernel.restype = ctypes.c_char_p
        L.paep_fold_batchnorm.argtypes = [vp] * 6 + [ctypes.c_float] + [i32] * 4 + [vp] * 3
        L.paep_fold_batchnorm.restype = ctypes.c_int
        L.paep_group_workspace_bytes.argtypes = [i32] * 4
        L.paep_group_workspace_bytes.restype = sz
        L.paep_group_by_expert.argtypes = [vp] + [i32] * 4 + [vp] * 7 + [sz, vp]
        L.paep_group_by_expert.restype = ctypes.c_int
        L.paep_score.argtypes = [vp, i32, vp, i32, i32, i32, i32, vp, vp]
        L.paep_score.restype = ctypes.c_int
        L.paep_score_rows.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, vp, vp]
        L.paep_score_rows.restype = ctypes.c_int
        L.paep_confidence_select.argtypes = [vp, vp, i32, i32, i32, i32, ctypes.c_float, vp, vp, vp, vp]
        L.paep_confidence_select.restype = ctypes.c_int
        L.paep_activation_profile.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.paep_activation_profile.restype = ctypes.c_int
        L.paep_probe_read.argtypes = [vp, sz, vp, sz, vp]
        L.paep_probe_read.restype = ctypes.c_int
        L.paep_probe_mfma.argtypes = [i32, i32, vp, sz, vp, ctypes.POINTER(ctypes.c_double)]
        L.paep_probe_mfma.restype = ctypes.c_int
        i64, cp, ap, mp = ctypes.c_int64, vp, vp, ctypes.POINTER(MoeDesc)      # (cp, ap: the structure by reference, or its bytes)
        L.paep_attend_workspace_bytes.argtypes = [cp, ap, i32]
        L.paep_attend_workspace_bytes.restype = sz
        L.paep_attend.argtypes = [cp, ap] + [vp] * 10 + [sz, vp]
        L.paep_attend.restype = ctypes.c_int
        L.paep_cache_append.argtypes = [cp, i32, vp, i64, vp, i64] + [vp] * 6 + [i64, vp]
        L.paep_cache_append.restype = ctypes.c_int
        L.paep_cache_evict.argtypes = [cp, i32, i32, i32] + [vp] * 5 + [i64, vp, i32, vp, vp, i64, vp, vp]
        L.paep_cache_evict.restype = ctypes.c_int
        L.paep_moe_workspace_bytes.argtypes = [mp]
        L.paep_moe_workspace_bytes.restype = sz
        L.paep_moe_layer.argtypes = [mp] + [vp] * 11 + [sz, vp]
        L.paep_moe_layer.restype = ctypes.c_int
        L.paep_moe_experts.argtypes = [mp] + [vp] * 8 + [sz, vp]
        L.paep_moe_experts.restype = ctypes.c_int
        L.paep_status_string.argtypes = [ctypes.c_int]
        L.paep_status_string.restype = ctypes.c_char_p
        L.paep_version.restype = ctypes.c_int
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is None:
        # torch.cuda.current_stream() makes a Stream object: 3 us, as long as the shortest kernels here
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())
    return stream.cuda_stream


def _on(stream):
    """Context in which torch allocates on `stream` (its caching allocator ties a block to the stream that
    was current when it was handed out): temporaries made for a call must belong to the stream the call's
    kernels are enqueued on, or the allocator may hand them to someone else while those kernels still run."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _storage_dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported storage dtype {t.dtype}; use float32 or bfloat16")


def _need_device(*tensors):
    for t in tensors:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("every tensor must be a contiguous device tensor")


class Prepared:
    """One library call with its arguments marshalled once.  Calling the object enqueues the work on
    `stream` (default: torch's current stream) at the cost of a single foreign call -- for loops that
    repeat the same call on the same buffers (a decode step per token)."""

    __slots__ = ("_fn", "_name", "_args", "_keep", "result")

    def __init__(self, fn, name, args, keep, result):
        self._fn, self._name, self._args, self._keep, self.result = fn, name, args, keep, result

    def __call__(self, stream=None):
        st = self._fn(*self._args, _stream_ptr(stream))
        if st != 0:
            raise PaepError(st, self._name)
        return self.result


class Prediction(NamedTuple):
    idx: torch.Tensor                 # [L, T, k] int32
    probs: torch.Tensor               # [L, T, k] float32
    logits: Optional[torch.Tensor]    # [L, T, E] float32 or None
    path: str
    margin: Optional[torch.Tensor] = None   # [L, T] float32: last selected score minus the best one left out


class Plan(NamedTuple):
    path: str
    tile: str                 # prefill tile configuration ("" on the other paths)
    groups: int               # workgroups sharing one token tile (r split between them)
    chunks_per_group: int


def make_desc(T, d, r, E, k, L, dtype, act="none", path="auto",
              x_layer_stride=None, w1_layer_stride=None, w2_layer_stride=None, prob="softmax") -> PredictDesc:
    return PredictDesc(T=T, d=d, r=r, E=E, k=k, L=L, dtype=dtype, act=ACT[act], path=PATH[path], prob=PROB[prob],
                       x_layer_stride=T * d if x_layer_stride is None else x_layer_stride,
                       w1_layer_stride=r * d if w1_layer_stride is None else w1_layer_stride,
                       w2_layer_stride=E * r if w2_layer_stride is None else w2_layer_stride)


def predict_workspace_bytes(desc: PredictDesc) -> int:
    return int(lib().paep_predict_workspace_bytes(ctypes.byref(desc)))


def predict_workspace_min_bytes(desc: PredictDesc) -> int:
    return int(lib().paep_predict_workspace_min_bytes(ctypes.byref(desc)))


def resolve_path(desc: PredictDesc) -> str:
    p = int(lib().paep_predict_resolve_path(ctypes.byref(desc)))
    return PATH_NAME.get(p, "invalid")


def predict_plan(desc: PredictDesc, want_margin: bool = False) -> Plan:
    """How paep_predict will run this shape (kernel family, prefill tile configuration, r split)."""
    out = (ctypes.c_int32 * 4)()
    st = lib().paep_predict_plan(ctypes.byref(desc), int(bool(want_margin)), ctypes.byref(out))
    if st != 0:
        raise PaepError(st, "paep_predict_plan")
    path = PATH_NAME.get(out[0], "invalid")
    return Plan(path, TILE_CFG.get(out[1], "?") if path == "prefill" else "", int(out[2]), int(out[3]))


def predict_kernel(desc: PredictDesc, want_margin: bool = False, workspace_bytes: Optional[int] = None,
                   with_b1: bool = False) -> str:
    """The kernel that the call, with or without b1, runs in a workspace of that size (default: predict_workspace_bytes), in words;
    "" where it would be refused."""
    if workspace_bytes is None:
        workspace_bytes = predict_workspace_bytes(desc)
    name = lib().paep_predict_kernel(ctypes.byref(desc), int(bool(want_margin)), int(bool(with_b1)), workspace_bytes)
    return name.decode() if name else ""


def _check_predict_inputs(x, W1, W2, k, b1, b2, act, path, prob):
    """Shape and dtype checks shared by the predict calls; returns the 3-D views and the descriptor."""
    if W1.dim() == 2:
        W1 = W1.unsqueeze(0)
    if W2.dim() == 2:
        W2 = W2.unsqueeze(0)
    if x.dim() == 2:
        x = x.unsqueeze(0)
    _need_device(x, W1, W2, b1, b2)
    L, r, d = W1.shape
    L2, E, r2 = W2.shape
    Lx, T, dx = x.shape
    if L2 != L or r2 != r or dx != d or Lx not in (1, L):
        raise ValueError(f"shape mismatch: x{tuple(x.shape)} W1{tuple(W1.shape)} W2{tuple(W2.shape)}")
    dt = _storage_dtype(x)
    if _storage_dtype(W1) != dt or _storage_dtype(W2) != dt:
        raise TypeError("x, W1 and W2 must share one storage dtype")
    for b, n in ((b1, r), (b2, E)):
        if b is not None and (b.numel() != L * n or _storage_dtype(b) != dt):
            raise ValueError("bias must be [L, r] / [L, E] in the storage dtype")
    desc = make_desc(T, d, r, E, k, L, dt, act, path, x_layer_stride=(T * d if Lx == L and L > 1 else 0), prob=prob)
    if L == 1:
        desc.x_layer_stride = T * d
    return x, W1, W2, desc, (L, T, E)


def prepare_predict(x: torch.Tensor, W1: torch.Tensor, W2: torch.Tensor, k: int, *,
                    b1: Optional[torch.Tensor] = None, b2: Optional[torch.Tensor] = None,
                    act: str = "none", path: str = "auto", want_logits: bool = False,
                    out: Optional[Prediction] = None, workspace: Optional[torch.Tensor] = None,
                    counts: Optional[torch.Tensor] = None, prob: str = "softmax",
                    want_margin: bool = False) -> Prepared:
    """Check and marshal one predict call; the returned object runs it (see `predict` for the arguments)."""
    x, W1, W2, desc, (L, T, E) = _check_predict_inputs(x, W1, W2, k, b1, b2, act, path, prob)
    dev = x.device
    if out is None:
        idx = torch.empty((L, T, k), dtype=torch.int32, device=dev)
        probs = torch.empty((L, T, k), dtype=torch.float32, device=dev)
        logits = torch.empty((L, T, E), dtype=torch.float32, device=dev) if want_logits else None
        margin = torch.empty((L, T), dtype=torch.float32, device=dev) if want_margin else None
    else:
        idx, probs, logits, margin = out.idx, out.probs, out.logits, out.margin
        _need_device(idx, probs, logits, margin)
        if margin is not None and (tuple(margin.shape) != (L, T) or margin.dtype != torch.float32):
            raise ValueError("margin buffer has the wrong shape or dtype")
        if tuple(idx.shape) != (L, T, k) or tuple(probs.shape) != (L, T, k) or idx.dtype != torch.int32 \
                or probs.dtype != torch.float32:
            raise ValueError("out buffers have the wrong shape or dtype")
        if logits is not None and (tuple(logits.shape) != (L, T, E) or logits.dtype != torch.float32):
            raise ValueError("logits buffer has the wrong shape or dtype")
    need = predict_workspace_bytes(desc)
    if workspace is None and need > 0:
        try:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        except torch.OutOfMemoryError:
            # the hidden vectors of two passes, say: the call runs without them, in one kernel
            least = predict_workspace_min_bytes(desc)
            if least == need:
                raise
            if least > 0:
                workspace = torch.empty(least, dtype=torch.uint8, device=dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if counts is not None:
        _need_device(counts)
        if counts.dtype != torch.int32 or tuple(counts.shape) != (L, E):
            raise ValueError("counts must be int32 [L, E]")
    if margin is not None:
        # the family is chosen knowing that one more candidate per row is kept
        args = (ctypes.byref(desc), _ptr(x), _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2),
                _ptr(idx), _ptr(probs), _ptr(logits), _ptr(counts), _ptr(margin), _ptr(workspace), ws_bytes)
        fam = predict_plan(desc, True).path
        return Prepared(lib().paep_predict_confidence, "paep_predict_confidence", args,
                        (desc, x, W1, W2, b1, b2, workspace, counts), Prediction(idx, probs, logits, fam, margin))
    result = Prediction(idx, probs, logits, resolve_path(desc))
    if counts is not None:
        args = (ctypes.byref(desc), _ptr(x), _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2),
                _ptr(idx), _ptr(probs), _ptr(logits), _ptr(counts), _ptr(workspace), ws_bytes)
        return Prepared(lib().paep_predict_counted, "paep_predict_counted", args,
                        (desc, x, W1, W2, b1, b2, workspace, counts), result)
    args = (ctypes.byref(desc), _ptr(x), _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2),
            _ptr(idx), _ptr(probs), _ptr(logits), _ptr(workspace), ws_bytes)
    return Prepared(lib().paep_predict, "paep_predict", args, (desc, x, W1, W2, b1, b2, workspace), result)


def predict(x: torch.Tensor, W1: torch.Tensor, W2: torch.Tensor, k: int, *,
            b1: Optional[torch.Tensor] = None, b2: Optional[torch.Tensor] = None,
            act: str = "none", path: str = "auto", want_logits: bool = False,
            out: Optional[Prediction] = None, workspace: Optional[torch.Tensor] = None,
            counts: Optional[torch.Tensor] = None, prob: str = "softmax", want_margin: bool = False,
            stream=None) -> Prediction:
    """predict(x[L|1,T,d], W1[L,r,d], W2[L,E,r], k) -> idx[L,T,k], probs[L,T,k].

    2-D inputs are taken as one layer.  x with a leading dimension of 1 (or
    2-D x with 3-D weights) feeds the same tokens to every layer.  `out` and
    `workspace` let a caller reuse buffers; otherwise they are allocated here.
    `counts` (int32 [L, E]) is increased by the activation counts of this call.
    `prob` picks what probs holds ("softmax" over all E, "softmax_topk" over the k selected, "sigmoid");
    `want_margin` adds margin[L, T], the last selected score minus the best one left out.
    Buffers allocated here are allocated on `stream`, the stream the kernels run on.
    """
    with _on(stream):
        prep = prepare_predict(x, W1, W2, k, b1=b1, b2=b2, act=act, path=path, want_logits=want_logits, out=out,
                               workspace=workspace, counts=counts, prob=prob, want_margin=want_margin)
    return prep(stream)


def static_init() -> None:
    """Bind the library's built-in scratch buffer on the current device (once per device, before graph capture)."""
    st = lib().paep_static_init()
    if st != 0:
        raise PaepError(st, "paep_static_init")


def predict_static(x: torch.Tensor, W1: torch.Tensor, W2: torch.Tensor, k: int, out: Prediction, *,
                   b1: Optional[torch.Tensor] = None, b2: Optional[torch.Tensor] = None,
                   act: str = "none", path: str = "auto", prob: str = "softmax", stream=None) -> Prediction:
    """paep_predict_static: predict into caller-provided `out` buffers using the library's built-in scratch
    buffer; nothing is allocated (shapes that need more than STATIC_SCRATCH_BYTES of workspace raise)."""
    x, W1, W2, desc, (L, T, E) = _check_predict_inputs(x, W1, W2, k, b1, b2, act, path, prob)
    _need_device(out.idx, out.probs, out.logits)
    if tuple(out.idx.shape) != (L, T, k) or tuple(out.probs.shape) != (L, T, k) or out.idx.dtype != torch.int32 \
            or out.probs.dtype != torch.float32:
        raise ValueError("out buffers have the wrong shape or dtype")
    if out.logits is not None and (tuple(out.logits.shape) != (L, T, E) or out.logits.dtype != torch.float32):
        raise ValueError("logits buffer has the wrong shape or dtype")
    st = lib().paep_predict_static(ctypes.byref(desc), _ptr(x), _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2),
                                   _ptr(out.idx), _ptr(out.probs), _ptr(out.logits), _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_predict_static")
    return Prediction(out.idx, out.probs, out.logits, resolve_path(desc))


class Grouping(NamedTuple):
    counts: torch.Tensor      # [L, E] int32
    offsets: torch.Tensor     # [L, E+1] int32
    token_pos: torch.Tensor   # [L, T*k] int32
    active: torch.Tensor      # [L, E] int32
    n_active: torch.Tensor    # [L] int32
    n_invalid: torch.Tensor   # [L] int32


def group_workspace_bytes(L: int, T: int, k: int, E: int) -> int:
    return int(lib().paep_group_workspace_bytes(L, T, k, E))


def alloc_grouping(L: int, T: int, k: int, E: int, device) -> Grouping:
    # empty_like costs half of empty's argument parsing, and calls of short kernels wait for the host
    i32 = dict(dtype=torch.int32, device=device)
    counts, n_active = torch.empty((L, E), **i32), torch.empty((L,), **i32)
    return Grouping(counts, torch.empty((L, E + 1), **i32), torch.empty((L, T * k), **i32), torch.empty_like(counts),
                    n_active, torch.empty_like(n_active))


def prepare_group_by_expert(idx: torch.Tensor, E: int, *, out: Optional[Grouping] = None,
                            workspace: Optional[torch.Tensor] = None) -> Prepared:
    """Check and marshal one group_by_expert call; the returned object runs it."""
    if idx.dim() == 2:
        idx = idx.unsqueeze(0)
    _need_device(idx)
    if idx.dtype != torch.int32 or idx.dim() != 3:
        raise TypeError("idx must be int32 [L, T, k]")
    L, T, k = idx.shape
    if out is None:
        out = alloc_grouping(L, T, k, E, idx.device)
    need = group_workspace_bytes(L, T, k, E)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=idx.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    args = (_ptr(idx), L, T, k, E, _ptr(out.counts), _ptr(out.offsets), _ptr(out.token_pos), _ptr(out.active),
            _ptr(out.n_active), _ptr(out.n_invalid), _ptr(workspace), ws_bytes)
    return Prepared(lib().paep_group_by_expert, "paep_group_by_expert", args, (idx, workspace), out)


def group_by_expert(idx: torch.Tensor, E: int, *, out: Optional[Grouping] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> Grouping:
    """group_by_expert(idx[L,T,k]) -> counts[L,E], offsets[L,E+1], token lists, prefetch list."""
    with _on(stream):
        prep = prepare_group_by_expert(idx, E, out=out, workspace=workspace)
    return prep(stream)


def prepare_score(idx: torch.Tensor, ref_idx: torch.Tensor, E: int, *, k_row: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None) -> Prepared:
    """Check and marshal one score call; the returned object runs it."""
    if idx.dim() == 2:
        idx = idx.unsqueeze(0)
    if ref_idx.dim() == 2:
        ref_idx = ref_idx.unsqueeze(0)
    _need_device(idx, ref_idx)
    if idx.dtype != torch.int32 or ref_idx.dtype != torch.int32:
        raise TypeError("idx and ref_idx must be int32")
    L, T, k_pred = idx.shape
    if ref_idx.shape[0] != L or ref_idx.shape[1] != T:
        raise ValueError("idx and ref_idx must agree on [L, T]")
    k_ref = ref_idx.shape[2]
    if out is None:
        out = torch.empty((L, 4), dtype=torch.int64, device=idx.device)
    if k_row is None:
        return Prepared(lib().paep_score, "paep_score",
                        (_ptr(idx), k_pred, _ptr(ref_idx), k_ref, L, T, E, _ptr(out)), (idx, ref_idx), out)
    _need_device(k_row)
    if k_row.dtype != torch.int32 or k_row.numel() != L * T or not k_row.is_contiguous():
        raise TypeError("k_row must be contiguous int32 [L, T]")
    return Prepared(lib().paep_score_rows, "paep_score_rows",
                    (_ptr(idx), k_pred, _ptr(k_row), _ptr(ref_idx), k_ref, L, T, E, _ptr(out)),
                    (idx, ref_idx, k_row), out)


def score(idx: torch.Tensor, ref_idx: torch.Tensor, E: int, *, k_row: Optional[torch.Tensor] = None,
          out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """score(idx[L,T,k_pred], ref_idx[L,T,k_ref]) -> int64 [L,4]: n_exact, n_hit, n_cover, n_top1.
    With k_row[L,T] (int32) each row uses only its first k_row predicted ids."""
    with _on(stream):
        prep = prepare_score(idx, ref_idx, E, k_row=k_row, out=out)
    return prep(stream)


class Widened(NamedTuple):
    idx: torch.Tensor         # [L, T, k_pred] int32, -1 past each row's width
    k_row: torch.Tensor       # [L, T] int32
    n_wide: torch.Tensor      # [L] int32


def confidence_select(idx: torch.Tensor, probs: torch.Tensor, k_base: int, ratio: float, stream=None) -> Widened:
    """Keep k_base predictions on confident rows (probs[k_base-1] >= ratio * probs[k_base]), all of them elsewhere."""
    if idx.dim() == 2:
        idx, probs = idx.unsqueeze(0), probs.unsqueeze(0)
    _need_device(idx, probs)
    if idx.dtype != torch.int32 or probs.dtype != torch.float32 or idx.shape != probs.shape \
            or not idx.is_contiguous() or not probs.is_contiguous():
        raise TypeError("idx int32 and probs float32 must be contiguous and of one shape [L, T, k_pred]")
    L, T, k_pred = idx.shape
    with _on(stream):
        out = Widened(torch.empty_like(idx), torch.empty((L, T), dtype=torch.int32, device=idx.device),
                      torch.empty((L,), dtype=torch.int32, device=idx.device))
    st = lib().paep_confidence_select(_ptr(idx), _ptr(probs), L, T, k_pred, k_base, float(ratio), _ptr(out.idx),
                                      _ptr(out.k_row), _ptr(out.n_wide), _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_confidence_select")
    return out


class ActivationProfile(NamedTuple):
    order: torch.Tensor       # [L, E] int32: experts by descending count, then -1
    n_active: torch.Tensor    # [L] int32
    entropy: torch.Tensor     # [L] float64: normalised Shannon entropy of the activation distribution


def activation_profile(counts: torch.Tensor, stream=None) -> ActivationProfile:
    """activation_profile(counts[L,E]) -> popularity-ordered expert list and entropy per layer."""
    if counts.dim() == 1:
        counts = counts.unsqueeze(0)
    _need_device(counts)
    if counts.dtype != torch.int32 or not counts.is_contiguous():
        raise TypeError("counts must be contiguous int32")
    L, E = counts.shape
    with _on(stream):
        out = ActivationProfile(torch.empty_like(counts),
                                torch.empty((L,), dtype=torch.int32, device=counts.device),
                                torch.empty((L,), dtype=torch.float64, device=counts.device))
    st = lib().paep_activation_profile(_ptr(counts), L, E, _ptr(out.order), _ptr(out.n_active), _ptr(out.entropy),
                                       _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_activation_profile")
    return out


def fold_batchnorm(W1: torch.Tensor, b1: Optional[torch.Tensor], gamma: torch.Tensor, beta: torch.Tensor,
                   mean: torch.Tensor, var: torch.Tensor, eps: float = 1e-5, stream=None):
    """BatchNorm (inference form) folded into the first linear layer: returns (W1', b1') such that
    act(BN(W1 x + b1)) = act(W1' x + b1').  W1 [L, r, d] (or [r, d]), b1 [L, r] or None in the storage
    dtype; gamma, beta, mean, var [L, r] float32."""
    squeeze = W1.dim() == 2
    if squeeze:
        W1 = W1.unsqueeze(0)
    L, r, d = W1.shape
    stats = [t.reshape(L, r) for t in (gamma, beta, mean, var)]
    _need_device(W1, b1, *stats)
    if any(t.dtype != torch.float32 for t in stats):
        raise TypeError("gamma, beta, mean, var must be float32")
    dt = _storage_dtype(W1)
    if b1 is not None and (_storage_dtype(b1) != dt or b1.numel() != L * r):
        raise ValueError("b1 must be [L, r] in the storage dtype of W1")
    with _on(stream):
        W1o = torch.empty_like(W1)
        b1o = torch.empty((L, r), dtype=W1.dtype, device=W1.device)
    st = lib().paep_fold_batchnorm(_ptr(W1), _ptr(b1), *[_ptr(t) for t in stats], float(eps), L, r, d, dt,
                                   _ptr(W1o), _ptr(b1o), _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_fold_batchnorm")
    return (W1o[0], b1o[0]) if squeeze else (W1o, b1o)


# ---- a layer's decode step beside the predictor ----

def _need_int32(dev: int, name: str, t: torch.Tensor, shape) -> None:
    """A contiguous int32 tensor on device `dev` (shape None: any)."""
    if t.dtype is not torch.int32 or t.get_device() != dev or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be contiguous int32" + (f" {list(shape)}" if shape is not None else "") + " on the cache's device")


def _need_rows(dev: int, dtype, name: str, t: torch.Tensor) -> None:
    """A tensor of the cache's type and device whose last dimension is contiguous."""
    if t.dtype is not dtype or t.get_device() != dev or t.stride(-1) != 1:
        raise ValueError(f"{name} must be of the cache's type and device, its last dimension contiguous")


def _need_mass(dev: int, name: str, t: torch.Tensor, B: int, Hkv: int, least: int) -> None:
    if t.dtype is not torch.float32 or t.get_device() != dev or not t.is_contiguous() or t.dim() != 3 or t.shape[0] != B \
            or t.shape[1] != Hkv or t.shape[2] < least:
        raise ValueError(f"{name} must be contiguous float32 [{B}, {Hkv}, at least {least}] on the cache's device")


def _need_32_bits(name: str, v: int) -> None:
    """The library's integers have 32 bits, and what does not fit would be cut off on the way there."""
    if not -1 << 31 <= v < 1 << 31:
        raise ValueError(f"{name} must fit in 32 bits")


def _stride(t: torch.Tensor, dim: int) -> int:
    """Stride of a dimension; 0 where it has one entry (torch leaves any value there)."""
    return t.stride(dim) if t.shape[dim] > 1 else 0


class _Cache(NamedTuple):
    desc: bytes               # the paep_cache_desc
    dev: int
    B: int
    Hkv: int
    Dk: int
    Dv: int
    capacity: int             # positions of a page-table row, or as many as the library counts


def _cache(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor) -> _Cache:
    """The cache k_pages [n_pages, Hkv, page_size, Dk], v_pages [n_pages, Hkv, page_size, Dv] (any strides, the last
    dimension contiguous), page_table [B, max_pages]."""
    dev, dtype = k_pages.get_device(), k_pages.dtype
    if dev < 0 or not k_pages.is_cuda:
        raise ValueError("every tensor must be a device tensor")
    dt = _storage_dtype(k_pages)
    if k_pages.dim() != 4 or v_pages.dim() != 4 or k_pages.shape[:3] != v_pages.shape[:3] or page_table.dim() != 2:
        raise ValueError(f"shape mismatch: k_pages{tuple(k_pages.shape)} v_pages{tuple(v_pages.shape)} page_table{tuple(page_table.shape)}")
    n, H, ps, Dk = k_pages.shape
    (kp, kh, ks, k1), (vp, vh, vs, v1) = k_pages.stride(), v_pages.stride()
    if k1 != 1 or v1 != 1 or v_pages.dtype is not dtype or v_pages.get_device() != dev:
        raise ValueError("k_pages and v_pages must be of one type and device, their last dimensions contiguous")
    _need_int32(dev, "page_table", page_table, None)
    B, width = page_table.shape
    if n < 2:                                                # (see _stride)
        kp = vp = 0
    if H < 2:
        kh = vh = 0
    if ps < 2:
        ks = vs = 0
    Dv = v_pages.shape[3]
    return _Cache(_CACHE_BYTES.pack(B, H, Dk, Dv, ps, n, width, dt, kp, kh, ks, vp, vh, vs), dev, B, H, Dk, Dv,
                  min(width * ps, 0x7FFF0000))


class Attention(NamedTuple):
    out: torch.Tensor                       # [B, Hq, Dv], in the cache's type
    lse: Optional[torch.Tensor] = None      # [B, Hq] float32: ln of the sum of the exponentials of the scores


def prepare_attend(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                   lengths: torch.Tensor, *, scale: Optional[float] = None, starts: Optional[torch.Tensor] = None,
                   max_len: Optional[int] = None, mass: Optional[torch.Tensor] = None, want_lse: bool = False,
                   out: Optional[Attention] = None, workspace: Optional[torch.Tensor] = None) -> Prepared:
    """Check and marshal one attend call; the returned object runs it (see `attend` for the arguments)."""
    c = _cache(k_pages, v_pages, page_table)
    dev, B, dtype = c.dev, c.B, k_pages.dtype
    if q.dim() != 3 or q.shape[0] != B or q.shape[2] != c.Dk:
        raise ValueError(f"q must be [{B}, heads, {c.Dk}]")
    Hq = q.shape[1]
    _need_rows(dev, dtype, "q", q)
    _need_int32(dev, "lengths", lengths, (B,))
    if starts is not None:
        _need_int32(dev, "starts", starts, (B,))
    if max_len is None:
        max_len = c.capacity
    else:
        _need_32_bits("max_len", max_len)
    if mass is not None:
        _need_mass(dev, "mass", mass, B, c.Hkv, max_len)
    if out is None:
        out = Attention(q.new_empty((B, Hq, c.Dv)), q.new_empty((B, Hq), dtype=torch.float32) if want_lse else None)
    else:
        _need_device(out.out, out.lse)
        if tuple(out.out.shape) != (B, Hq, c.Dv) or out.out.dtype != dtype or \
                (out.lse is not None and (tuple(out.lse.shape) != (B, Hq) or out.lse.dtype != torch.float32)):
            raise ValueError("out buffers have the wrong shape or dtype")
    d = _ATTEND_BYTES.pack(Hq, max_len, c.Dk ** -0.5 if scale is None else scale, 0, _stride(q, 0), _stride(q, 1),
                           0 if mass is None else mass.shape[2])
    L = lib()
    need = L.paep_attend_workspace_bytes(c.desc, d, mass is not None)
    if workspace is None and need > 0:
        workspace = q.new_empty(need, dtype=torch.uint8)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    args = (c.desc, d, _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(page_table), _ptr(lengths),
            _ptr(starts), _ptr(out.out), _ptr(out.lse), _ptr(mass), _ptr(workspace), ws_bytes)
    return Prepared(L.paep_attend, "paep_attend", args,
                    (q, k_pages, v_pages, page_table, lengths, starts, mass, workspace), out)


def attend(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, *,
           scale: Optional[float] = None, starts: Optional[torch.Tensor] = None, max_len: Optional[int] = None,
           mass: Optional[torch.Tensor] = None, want_lse: bool = False, out: Optional[Attention] = None,
           workspace: Optional[torch.Tensor] = None, stream=None) -> Attention:
    """Attention of one new token per sequence over a paged key-value cache.

    q [B, Hq, Dk] (any strides, the last dimension contiguous; so the pools), k_pages [n_pages, Hkv, page_size, Dk],
    v_pages [n_pages, Hkv, page_size, Dv], page_table [B, max_pages] int32, lengths [B] int32 -> out [B, Hq, Dv],
    lse [B, Hq] with want_lse.  A page that holds its slots outside its heads is passed as its transposed view.
    `scale` defaults to Dk ** -0.5; `starts` [B] int32: the first position each sequence looks at; `max_len`: a bound on
    the lengths (default: what a row of the page table can hold, 2^31 - 2^16 at most) -- the work is laid out for it, so a
    tight one is faster, and with `mass` the workspace has 4 bytes for each of its positions at each query head;
    `mass` [B, Hkv, >= max_len] float32: increased by the attention weight of every position, summed over the query heads
    of its key-value head (what `cache_evict` goes by).  Sequences with nothing to look at give zeros."""
    with _on(stream):
        prep = prepare_attend(q, k_pages, v_pages, page_table, lengths, scale=scale, starts=starts, max_len=max_len, mass=mass,
                              want_lse=want_lse, out=out, workspace=workspace)
    return prep(stream)


def cache_append(k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                 positions: torch.Tensor, *, sequences: Optional[torch.Tensor] = None, mass: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """Write keys k [n, Hkv, Dk] and values v [n, Hkv, Dv] (rows any stride apart) into the cache: row i to position
    positions[i] of sequence sequences[i] (default: of sequence i).  Rows that name no place are skipped.  `mass`
    [B, Hkv, any] is set to 0 at the positions written."""
    c = _cache(k_pages, v_pages, page_table)
    dev = c.dev
    _need_rows(dev, k_pages.dtype, "k", k)
    _need_rows(dev, k_pages.dtype, "v", v)
    n = k.shape[0]
    if k.shape != (n, c.Hkv, c.Dk) or v.shape != (n, c.Hkv, c.Dv) or (c.Hkv > 1 and (k.stride(1) != c.Dk or v.stride(1) != c.Dv)):
        raise ValueError(f"k must be [n, {c.Hkv}, {c.Dk}] and v [n, {c.Hkv}, {c.Dv}], the heads of a row side by side")
    _need_int32(dev, "positions", positions, (n,))
    if sequences is not None:
        _need_int32(dev, "sequences", sequences, (n,))
    if mass is not None:
        _need_mass(dev, "mass", mass, c.B, c.Hkv, 0)
    st = lib().paep_cache_append(c.desc, n, _ptr(k), _stride(k, 0), _ptr(v), _stride(v, 0), _ptr(k_pages), _ptr(v_pages),
                                 _ptr(page_table), _ptr(sequences), _ptr(positions), _ptr(mass),
                                 0 if mass is None else mass.shape[2], _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_cache_append")


class Eviction(NamedTuple):
    lengths: torch.Tensor     # [B] int32: the lengths now
    kept: torch.Tensor        # [B, Hkv, budget] int32: the positions kept, ascending, then -1
    mass: torch.Tensor        # [B, Hkv, as before] float32: their accumulated weight, then 0


def cache_evict(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                mass: torch.Tensor, out_table: torch.Tensor, budget: int, recent: int, *, max_len: Optional[int] = None,
                out: Optional[Eviction] = None, stream=None) -> Eviction:
    """Cut every sequence down to `budget` positions: each head keeps its last `recent` ones and, of those before them, the
    ones with the largest accumulated weight `mass` [B, Hkv, >= max_len]; they are copied, in order, to the pages of
    out_table [B, out_pages] int32 of the same pools, which must be free.  Shorter sequences are copied whole."""
    c = _cache(k_pages, v_pages, page_table)
    dev, B, H = c.dev, c.B, c.Hkv
    if max_len is None:
        max_len = c.capacity
    else:
        _need_32_bits("max_len", max_len)
    _need_mass(dev, "mass", mass, B, H, max_len)
    if out_table.dim() != 2 or out_table.shape[0] != B:
        raise ValueError("out_table must be [B, out_pages]")
    _need_int32(dev, "lengths", lengths, (B,))
    _need_int32(dev, "out_table", out_table, None)
    if budget < 1:
        raise ValueError("budget must be at least 1")
    _need_32_bits("budget", budget)
    _need_32_bits("recent", recent)
    if out is None:
        with _on(stream):
            out = Eviction(torch.empty_like(lengths), lengths.new_empty((B, H, budget)), torch.empty_like(mass))
    else:
        _need_int32(dev, "out.lengths", out.lengths, (B,))
        _need_int32(dev, "out.kept", out.kept, (B, H, budget))
        _need_mass(dev, "out.mass", out.mass, B, H, min(budget, max_len))
        if B > 0 and (out.mass.data_ptr() == mass.data_ptr() or out.lengths.data_ptr() == lengths.data_ptr()):
            raise ValueError("out.mass and out.lengths must be other buffers than mass and lengths")
    st = lib().paep_cache_evict(c.desc, max_len, budget, recent, _ptr(k_pages), _ptr(v_pages), _ptr(page_table),
                                _ptr(lengths), _ptr(mass), mass.shape[2], _ptr(out_table), out_table.shape[1], _ptr(out.kept),
                                _ptr(out.mass), out.mass.shape[2], _ptr(out.lengths), _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_cache_evict")
    return out


class MoeOutput(NamedTuple):
    y: torch.Tensor           # [T, d]
    idx: torch.Tensor         # [T, k] int32
    probs: torch.Tensor       # [T, k] float32


def _prepare_moe(x, W13, W2, k, act, prob, residual, y, workspace):
    """Shape and type checks shared by the expert-layer calls; returns the descriptor, y, the workspace and its size."""
    if x.dim() != 2 or W13.dim() != 3 or W2.dim() != 3:
        raise ValueError("x must be [T, d], W13 [E, 2f, d], W2 [E, d, f]")
    T, d = x.shape
    E, _, f = W2.shape
    if tuple(W13.shape) != (E, 2 * f, d) or W2.shape[1] != d:
        raise ValueError(f"shape mismatch: x{tuple(x.shape)} W13{tuple(W13.shape)} W2{tuple(W2.shape)}")
    _need_device(x, W13, W2, residual, y)
    dt = _storage_dtype(x)
    for t in (W13, W2, residual, y):
        if t is not None and (t.dtype != x.dtype or t.device != x.device):
            raise TypeError("x, the weights, residual and y must share one storage dtype and device")
    for t in (residual, y):
        if t is not None and t.shape != x.shape:
            raise ValueError("residual and y must be [T, d]")
    _need_32_bits("k", k)
    desc = MoeDesc(T, d, f, E, k, dt, ACT[act], PROB[prob])
    if y is None:
        y = torch.empty_like(x)
    need = lib().paep_moe_workspace_bytes(ctypes.byref(desc))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    return desc, y, workspace, 0 if workspace is None else workspace.numel() * workspace.element_size()


def prepare_moe_layer(x: torch.Tensor, Wg: torch.Tensor, W13: torch.Tensor, W2: torch.Tensor, k: int, *,
                      bg: Optional[torch.Tensor] = None, act: str = "silu", prob: str = "softmax",
                      residual: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                      out: Optional[MoeOutput] = None, workspace: Optional[torch.Tensor] = None) -> Prepared:
    """Check and marshal one moe_layer call; the returned object runs it (see `moe_layer` for the arguments)."""
    desc, y, workspace, ws_bytes = _prepare_moe(x, W13, W2, k, act, prob, residual, None if out is None else out.y, workspace)
    T, E, dev = desc.T, desc.E, x.device
    _need_device(Wg, bg, counts)
    if tuple(Wg.shape) != (E, desc.d) or Wg.dtype != x.dtype or Wg.device != dev:
        raise ValueError("Wg must be [E, d] in the storage dtype and on the device of x")
    if bg is not None and (bg.numel() != E or bg.dtype != x.dtype or bg.device != dev):
        raise ValueError("bg must be [E] in the storage dtype and on the device of x")
    if counts is not None and (counts.dtype != torch.int32 or counts.numel() != E or counts.device != dev):
        raise ValueError("counts must be int32 [E]")
    if out is None:
        out = MoeOutput(y, torch.empty((T, k), dtype=torch.int32, device=dev), torch.empty((T, k), dtype=torch.float32, device=dev))
    else:
        _need_device(out.idx, out.probs)
        if tuple(out.idx.shape) != (T, k) or out.idx.dtype != torch.int32 or tuple(out.probs.shape) != (T, k) \
                or out.probs.dtype != torch.float32:
            raise ValueError("out buffers have the wrong shape or dtype")
    args = (ctypes.byref(desc), _ptr(x), _ptr(Wg), _ptr(bg), _ptr(W13), _ptr(W2), _ptr(residual), _ptr(out.y), _ptr(out.idx),
            _ptr(out.probs), _ptr(counts), _ptr(workspace), ws_bytes)
    return Prepared(lib().paep_moe_layer, "paep_moe_layer", args, (desc, x, Wg, bg, W13, W2, residual, counts, workspace), out)


def moe_layer(x: torch.Tensor, Wg: torch.Tensor, W13: torch.Tensor, W2: torch.Tensor, k: int, *,
              bg: Optional[torch.Tensor] = None, act: str = "silu", prob: str = "softmax",
              residual: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
              out: Optional[MoeOutput] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> MoeOutput:
    """A mixture-of-experts layer for up to 64 tokens: x [T, d], router Wg [E, d] (+ bg [E]), W13 [E, 2f, d] (the f gate rows,
    then the f others), W2 [E, d, f] -> y [T, d], idx [T, k], probs [T, k] with

        y = residual + sum over the k experts of  p * W2 (act(W1 x) * (W3 x)).

    `prob` says what weighs an expert, as in `predict`; `counts` (int32 [E]) is increased by the tokens per expert.
    Weights and tokens bf16 or float32, sums in float32."""
    with _on(stream):
        prep = prepare_moe_layer(x, Wg, W13, W2, k, bg=bg, act=act, prob=prob, residual=residual, counts=counts, out=out,
                                 workspace=workspace)
    return prep(stream)


def moe_experts(x: torch.Tensor, W13: torch.Tensor, W2: torch.Tensor, idx: torch.Tensor, probs: torch.Tensor, *,
                act: str = "silu", residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """`moe_layer` with a selection that is there already, idx [T, k] int32 and probs [T, k] float32 (another router's, or
    the predictor's own); ids outside [0, E) are skipped.  Returns y [T, d]."""
    if idx.dim() != 2 or idx.shape != probs.shape or idx.shape[0] != x.shape[0] or idx.dtype != torch.int32 \
            or probs.dtype != torch.float32 or idx.device != x.device or probs.device != x.device:
        raise ValueError("idx must be int32 [T, k] and probs float32 [T, k], on the device of x")
    _need_device(idx, probs)
    with _on(stream):
        desc, y, workspace, ws_bytes = _prepare_moe(x, W13, W2, idx.shape[1], act, "softmax", residual, out, workspace)
    st = lib().paep_moe_experts(ctypes.byref(desc), _ptr(x), _ptr(W13), _ptr(W2), _ptr(idx), _ptr(probs), _ptr(residual), _ptr(y),
                                _ptr(workspace), ws_bytes, _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_moe_experts")
    return y


def probe_read(src: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """One launch of the streaming-read probe over all of `src` (device ceilings, not part of the method)."""
    _need_device(src, sink)
    st = lib().paep_probe_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink),
                               sink.numel() * sink.element_size(), _stream_ptr(stream))
    if st != 0:
        raise PaepError(st, "paep_probe_read")


def probe_mfma(workgroups: int, iters: int, sink: torch.Tensor, stream=None) -> float:
    """One launch of the register-only matrix-instruction probe; returns the flops of the launch."""
    _need_device(sink)
    flops = ctypes.c_double(0.0)
    st = lib().paep_probe_mfma(workgroups, iters, _ptr(sink), sink.numel() * sink.element_size(),
                               _stream_ptr(stream), ctypes.byref(flops))
    if st != 0:
        raise PaepError(st, "paep_probe_mfma")
    return flops.value
