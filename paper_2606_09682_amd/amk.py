"""ctypes binding of libamk.so (include/amk.h): same names, argument marshalling only.

Every computation of the decode step runs in the HIP library; this module
only converts Python / torch arguments into the C structures and checks
status codes.  If the library is missing it raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Mapping, Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libamk.so")

# ---- constants (mirror include/amk.h) ---------------------------------------
AMK_ABI_VERSION = 5
AMK_OK = 0
AMK_ERR_INVALID_ARGUMENT = -1
AMK_ERR_UNSUPPORTED = -2
AMK_ERR_SCHEDULE_REJECTED = -3
AMK_ERR_OUT_OF_MEMORY = -4
AMK_ERR_DEVICE = -5
AMK_ERR_COOPERATIVE_UNSUPPORTED = -6
AMK_ERR_TIMEOUT = -7
AMK_ERR_BAD_STATE = -8
AMK_ERR_ABORTED = -9
AMK_ERR_NONFINITE = -10

AMK_WEIGHTS_BF16 = 0
AMK_WEIGHTS_W8A16 = 1
AMK_WEIGHTS_W4A16 = 2

AMK_SCHEDULE_SHORT, AMK_SCHEDULE_LONG, AMK_SCHEDULE_TINY = 0, 1, 2
AMK_ASSIGN_ROUND_ROBIN, AMK_ASSIGN_LPT = 0, 1
AMK_TINY_MAX = 8
AMK_F32, AMK_BF16, AMK_F16 = 0, 1, 2
AMK_TREE_MAX = 64
AMK_TOP_MAX = 32
AMK_OP_QKV, AMK_OP_ATTN, AMK_OP_COMBINE, AMK_OP_O, AMK_OP_GATEUP, AMK_OP_DOWN, AMK_OP_LMHEAD, AMK_OP_ARGMAX = range(1, 9)
AMK_MAX_WAITS = 4
AMK_CU_INLINE = -1
AMK_TRACE_FIELDS = 8
(AMK_TRACE_WAIT_BEGIN, AMK_TRACE_WAIT_END, AMK_TRACE_INPUT_READY, AMK_TRACE_COMPUTE_END,
 AMK_TRACE_SIGNALLED, AMK_TRACE_PUBLISHED, AMK_TRACE_CHAINED, AMK_TRACE_SATISFIED) = range(8)

(AMK_CHECK_OK, AMK_CHECK_WELL_FORMED, AMK_CHECK_CAPACITY, AMK_CHECK_WAIT_SATISFIABLE, AMK_CHECK_ALL_JOIN,
 AMK_CHECK_ACYCLIC, AMK_CHECK_QUEUE_ORDER, AMK_CHECK_RACE, AMK_CHECK_KV_ORDER, AMK_CHECK_OUTPUT,
 AMK_CHECK_INLINE) = range(11)


# ---- structures ---------------------------------------------------------------
class amk_config_t(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32), ("hidden", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("intermediate", ctypes.c_int32), ("vocab", ctypes.c_int32), ("max_seq", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float), ("tied_embeddings", ctypes.c_int32),
                ("weight_format", ctypes.c_int32), ("device", ctypes.c_int32), ("group_size", ctypes.c_int32)]


class amk_linear_t(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class amk_layer_weights_t(ctypes.Structure):
    _fields_ = [("attn_norm", ctypes.c_void_p), ("mlp_norm", ctypes.c_void_p)] + [
        (n, amk_linear_t) for n in ("q", "k", "v", "o", "gate", "up", "down")]


class amk_weights_t(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p), ("lm_head", amk_linear_t),
                ("layers", ctypes.POINTER(amk_layer_weights_t))]


class amk_tuning_t(ctypes.Structure):
    _fields_ = [("attn_splits", ctypes.c_int32), ("timeout_us", ctypes.c_int32),
                ("max_rows_per_task", ctypes.c_int32), ("trace", ctypes.c_int32), ("short_context", ctypes.c_int32),
                ("tiny_context", ctypes.c_int32), ("queue_assign", ctypes.c_int32)]


class amk_task_t(ctypes.Structure):
    _fields_ = [("op", ctypes.c_uint16), ("layer", ctypes.c_uint16), ("cu", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("begin", ctypes.c_int32), ("end", ctypes.c_int32), ("aux", ctypes.c_int16),
                ("n_wait", ctypes.c_int16), ("wait_counter", ctypes.c_int32 * AMK_MAX_WAITS),
                ("wait_count", ctypes.c_int32 * AMK_MAX_WAITS), ("signal_counter", ctypes.c_int32),
                ("chain_counter", ctypes.c_int32)]


class amk_check_report_t(ctypes.Structure):
    _fields_ = [("ok", ctypes.c_int32), ("rule", ctypes.c_int32), ("task", ctypes.c_int32), ("other", ctypes.c_int32),
                ("n_tasks", ctypes.c_int32), ("n_counters", ctypes.c_int32), ("n_edges", ctypes.c_int32),
                ("message", ctypes.c_char * 256)]


class amk_attention_t(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "out_token",
                                      "out_head")] + [
        ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("scale", ctypes.c_float)]


class AmkError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        super().__init__(f"{what}: {amk_status_string(status)} ({status})" if what else
                         f"{amk_status_string(status)} ({status})")


_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libamk.so (built in-tree by paper_2606_09682_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: run `python -m paper_2606_09682_amd.build` first")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    sig = {
        "amk_create": (ctypes.c_int, [P(amk_config_t), P(amk_weights_t), P(amk_tuning_t), P(ctypes.c_void_p)]),
        "amk_decode_step": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p]),
        "amk_create_static": (ctypes.c_int, [P(amk_config_t), P(amk_weights_t), P(amk_tuning_t),
                                             P(ctypes.c_void_p)]),
        "amk_destroy": (ctypes.c_int, [ctypes.c_void_p]),
        "amk_kv_cache_bytes": (ctypes.c_size_t, [P(amk_config_t)]),
        "amk_next_token_ptr": (ctypes.c_void_p, [ctypes.c_void_p]),
        "amk_copy_next_token": (ctypes.c_int, [ctypes.c_void_p, P(ctypes.c_int32), ctypes.c_void_p]),
        "amk_get_status": (ctypes.c_int, [ctypes.c_void_p]),
        "amk_read_probe": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p,
                                          ctypes.c_void_p]),
        "amk_reset": (ctypes.c_int, [ctypes.c_void_p]),
        "amk_set_abort": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int32]),
        "amk_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "amk_schedule_size": (ctypes.c_int, [P(amk_config_t), P(amk_tuning_t), ctypes.c_int32, ctypes.c_int32,
                                             P(ctypes.c_int32), P(ctypes.c_int32)]),
        "amk_schedule_export": (ctypes.c_int, [P(amk_config_t), P(amk_tuning_t), ctypes.c_int32, ctypes.c_int32,
                                               P(amk_task_t), ctypes.c_int32, P(ctypes.c_int32), P(ctypes.c_int32)]),
        "amk_schedule_check": (ctypes.c_int, [P(amk_config_t), P(amk_tuning_t), ctypes.c_int32, P(amk_task_t),
                                              ctypes.c_int32, ctypes.c_int32, P(amk_check_report_t)]),
        "amk_check_config": (ctypes.c_int, [P(amk_config_t), ctypes.c_int32]),
        "amk_trace_copy": (ctypes.c_int, [ctypes.c_void_p, P(ctypes.c_uint64), ctypes.c_int64, P(ctypes.c_int32),
                                          P(ctypes.c_int32)]),
    }
    i32, i64, ptr, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    sig.update({
        "amk_linear": (ctypes.c_int, [ptr, i64, i32, i32, i32, ptr, ptr, i32, i32, ptr, i64, i32, i32, ptr]),
        "amk_prompt_attention": (ctypes.c_int, [P(amk_attention_t), ptr, ptr, i32, i32, i32, ptr, size, ptr]),
        "amk_prompt_attention_workspace": (size, [i32] * 6),
        "amk_tree_attention": (ctypes.c_int, [P(amk_attention_t), i32, i32, P(ctypes.c_uint64), ptr, size, ptr]),
        "amk_tree_attention_workspace": (size, [i32] * 5),
        "amk_token_logprobs": (ctypes.c_int, [ptr, i32, i64, i32, i32, ptr, i32, ptr, ptr, ptr, ptr, ptr, size, ptr]),
        "amk_token_logprobs_workspace": (size, [i32] * 4),
        "amk_kv_keep": (ctypes.c_int, [ptr, i32, i32, i32, i32, i32, P(i32), i32, ptr]),
        "amk_extend": (ctypes.c_int, [ptr, P(i32), i32, i32, P(i32), ptr, ptr, i32, ptr, size, ptr]),
        "amk_extend_workspace": (size, [ptr, i32]),
    })
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int, what: str) -> None:
    if status != AMK_OK:
        raise AmkError(status, what)


# ---- thin wrappers with the C names -------------------------------------------------
def amk_status_string(status: int) -> str:
    return load().amk_status_string(status).decode()


def amk_kv_cache_bytes(cfg: amk_config_t) -> int:
    return int(load().amk_kv_cache_bytes(ctypes.byref(cfg)))


def amk_create(cfg: amk_config_t, weights: amk_weights_t, tuning: Optional[amk_tuning_t] = None) -> ctypes.c_void_p:
    h = ctypes.c_void_p()
    _check(load().amk_create(ctypes.byref(cfg), ctypes.byref(weights), ctypes.byref(tuning) if tuning else None,
                             ctypes.byref(h)), "amk_create")
    return h


def amk_create_static(cfg: amk_config_t, weights: amk_weights_t,
                      tuning: Optional[amk_tuning_t] = None) -> ctypes.c_void_p:
    """amk_create whose device memory is the library's static array (see amk.h)."""
    h = ctypes.c_void_p()
    _check(load().amk_create_static(ctypes.byref(cfg), ctypes.byref(weights),
                                    ctypes.byref(tuning) if tuning else None, ctypes.byref(h)), "amk_create_static")
    return h


def amk_decode_step(h, token: int, pos: int, kv_cache_ptr: int, logits_ptr: int, stream: int = 0) -> None:
    _check(load().amk_decode_step(h, token, pos, kv_cache_ptr, logits_ptr, stream or None), "amk_decode_step")


def amk_destroy(h) -> None:
    _check(load().amk_destroy(h), "amk_destroy")


def amk_next_token_ptr(h) -> int:
    return int(load().amk_next_token_ptr(h) or 0)


def amk_copy_next_token(h, stream: int = 0) -> int:
    v = ctypes.c_int32(-1)
    _check(load().amk_copy_next_token(h, ctypes.byref(v), stream or None), "amk_copy_next_token")
    return int(v.value)


def amk_get_status(h) -> int:
    return int(load().amk_get_status(h))


def amk_read_probe(buf_ptr: int, nbytes: int, blocks: int, sink_ptr: int, stream: int) -> None:
    """Enqueue one streaming read of nbytes at device address buf_ptr (see amk.h)."""
    _check(load().amk_read_probe(buf_ptr, nbytes, blocks, sink_ptr, stream), "amk_read_probe")


def amk_reset(h) -> None:
    _check(load().amk_reset(h), "amk_reset")


def amk_set_abort(h, value: int) -> None:
    _check(load().amk_set_abort(h, int(value)), "amk_set_abort")


def amk_trace_copy(h, n_tasks: int):
    """(variant, per-task timestamps) of the last step: a list of
    AMK_TRACE_FIELDS-tuples in the order of that variant's export."""
    buf = (ctypes.c_uint64 * (n_tasks * AMK_TRACE_FIELDS))()
    n, v = ctypes.c_int32(), ctypes.c_int32()
    _check(load().amk_trace_copy(h, buf, len(buf), ctypes.byref(n), ctypes.byref(v)), "amk_trace_copy")
    return v.value, [tuple(buf[i * AMK_TRACE_FIELDS:(i + 1) * AMK_TRACE_FIELDS]) for i in range(n.value)]


def amk_check_config(cfg: amk_config_t, n_cu: int) -> int:
    return int(load().amk_check_config(ctypes.byref(cfg), n_cu))


def amk_schedule_export(cfg: amk_config_t, n_cu: int, tuning: Optional[amk_tuning_t] = None,
                        variant: int = AMK_SCHEDULE_LONG):
    """Returns (tasks array, n_counters) of the lowering of cfg onto n_cu queues."""
    lib = load()
    nt, nc = ctypes.c_int32(), ctypes.c_int32()
    tp = ctypes.byref(tuning) if tuning else None
    _check(lib.amk_schedule_size(ctypes.byref(cfg), tp, n_cu, variant, ctypes.byref(nt), ctypes.byref(nc)),
           "amk_schedule_size")
    arr = (amk_task_t * nt.value)()
    _check(lib.amk_schedule_export(ctypes.byref(cfg), tp, n_cu, variant, arr, nt.value, ctypes.byref(nt),
                                   ctypes.byref(nc)), "amk_schedule_export")
    return arr, nc.value


def amk_schedule_check(cfg: amk_config_t, n_cu: int, tasks, n_counters: int,
                       tuning: Optional[amk_tuning_t] = None) -> amk_check_report_t:
    rep = amk_check_report_t()
    _check(load().amk_schedule_check(ctypes.byref(cfg), ctypes.byref(tuning) if tuning else None, n_cu, tasks,
                                     len(tasks), n_counters, ctypes.byref(rep)), "amk_schedule_check")
    return rep


# ---- operators for several tokens over torch device tensors ---------------------------
# Each call runs on the tensors' device and torch's current stream there, on which its
# outputs and workspaces are allocated too; nothing synchronises.  The library sees
# bare pointers, so types, shapes, devices and strides are checked here.  Small calls
# take the GPU a few microseconds, so what runs on every call is kept short: a stream
# is read as its raw handle, and messages are made only for a refusal.  They serve
# inference: results have no gradients, whether or not an operand requires them, and
# autograd does not see what is written to `out` or a cache.
_SCORE_CHUNK = 2048  # tokens whose logits Decoder.score holds at once: what amk_extend takes through the model at once
_FORMATS = {"bf16": AMK_WEIGHTS_BF16, "w8a16": AMK_WEIGHTS_W8A16, "w4a16": AMK_WEIGHTS_W4A16}
_torch = None


def _load_torch():
    """torch (imported on first use), with the types and functions the calls use."""
    global _torch, _BF16, _WEIGHT, _SCALE, _OUT, _LOGITS
    import torch
    _BF16 = (torch.bfloat16, torch.int16)  # int16: bf16 bits
    _WEIGHT = (_BF16, (torch.int8,), (torch.uint8,))
    _SCALE = ((), (torch.float32,), (torch.float16,))
    _OUT = {torch.float32: AMK_F32, torch.bfloat16: AMK_BF16}
    _LOGITS = {torch.float32: AMK_F32, torch.bfloat16: AMK_BF16, torch.float16: AMK_F16}
    _torch = torch
    return torch


def _refuse(t, what: str, index: int, dtypes, dim: int):
    if t.get_device() != index:
        raise ValueError(f"{what} is on {t.device}, expected cuda:{index}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what} has type {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    raise ValueError(f"{what} has {t.dim()} dimensions, expected {dim}")


def _call(index: int, fn, *args) -> None:
    """fn(*args, stream) with device `index` current; raises on an error status."""
    torch = _torch
    if torch.cuda.current_device() == index:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status != AMK_OK:
        raise AmkError(status, fn.__name__)


def _int32(value: int, what: str) -> None:
    """Refuses what the library's int32 arguments would silently cut."""
    if not -1 << 31 <= value < 1 << 31:
        raise ValueError(f"{what} = {value} does not fit 32 bits")


def _past_int32(*sizes: int):
    raise ValueError(f"a size of {max(sizes)} does not fit 32 bits")


def _device_index(t, what: str) -> int:
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{what} must be a device tensor")
    return index


def _workspace(nbytes: int, index: int):
    return _torch.empty(nbytes, dtype=_torch.uint8, device=_torch.device("cuda", index))


def linear(x, w, scale=None, weight_format: str = "bf16", group_size: int = 0, out=None, out_dtype=None,
           accumulate: bool = False):
    """x W^T for n tokens (amk_linear; no gradients): x bf16 [n, in] with contiguous rows; w and
    scale a projection as Decoder takes it ([out, in] bf16 or int16 bits; int8 with
    fp32 scale [out]; packed uint8 [out, in / 2] with fp16 scale [out, in / group]).
    Returns [n, out] of out_dtype (fp32, the default, or bf16), or writes it to `out`
    (contiguous rows) and returns that; accumulate adds to `out`."""
    torch = _torch or _load_torch()
    fmt = _FORMATS.get(weight_format)
    if fmt is None:
        raise ValueError(f"unknown weight format {weight_format}")
    index = _device_index(x, "x")
    if x.dtype not in _BF16 or x.dim() != 2:
        _refuse(x, "x", index, _BF16, 2)
    if w.get_device() != index or w.dtype not in _WEIGHT[fmt] or w.dim() != 2:
        _refuse(w, "w", index, _WEIGHT[fmt], 2)
    n, width = x.shape
    rows, stored = w.shape
    if (n | width | rows) >> 31:
        _past_int32(n, width, rows)
    _int32(group_size, "group_size")
    if n and x.stride(1) != 1:
        raise ValueError("x must have contiguous rows")
    if (stored * 2 if fmt == AMK_WEIGHTS_W4A16 else stored) != width or not w.is_contiguous():
        raise ValueError(f"w must be contiguous rows of {width} columns")
    scale_ptr = None
    if fmt != AMK_WEIGHTS_BF16:
        if scale is None:
            raise ValueError(f"{weight_format} weights need a scale")
        w4 = fmt == AMK_WEIGHTS_W4A16
        if scale.get_device() != index or scale.dtype not in _SCALE[fmt] or scale.dim() != 1 + w4:
            _refuse(scale, "scale", index, _SCALE[fmt], 1 + w4)
        if scale.numel() != (rows * (width // (group_size or 128)) if w4 else rows) or not scale.is_contiguous():
            raise ValueError("scale must be contiguous, one value per row (and group of columns)")
        scale_ptr = scale.data_ptr()
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out_dtype = out_dtype or torch.float32
        if out_dtype not in _OUT:
            raise ValueError("out_dtype must be float32 or bfloat16")
        out = torch.empty((n, rows), dtype=out_dtype, device=x.device)
        y_stride = rows
    else:
        allowed = tuple(_OUT) if out_dtype is None else (out_dtype,)
        if out.get_device() != index or out.dtype not in allowed or out.dtype not in _OUT or out.dim() != 2:
            _refuse(out, "out", index, tuple(_OUT), 2)
        if tuple(out.shape) != (n, rows) or (out.numel() and out.stride(1) != 1):
            raise ValueError(f"out must be [{n}, {rows}] with contiguous rows")
        y_stride = out.stride(0) if n > 1 else rows
    _call(index, load().amk_linear, x.data_ptr(), x.stride(0) if n > 1 else (width + 7) // 8 * 8, n, width, rows,
          w.data_ptr(), scale_ptr, fmt, group_size, out.data_ptr(), y_stride, _OUT[out.dtype], int(accumulate))
    return out


def _strides(t, name: str):
    """(token, head) strides of [tokens, heads, head_dim]; a dimension of one element is
    not stepped over, so any stride will do for it."""
    (tokens, heads, d), (token, head, one) = t.shape, t.stride()
    if one != 1 and d > 1 and t.numel():
        raise ValueError(f"{name} must have contiguous heads")
    return token if tokens > 1 else 8, head if heads > 1 else 8


def _attention(q, k, v, scale, out):
    """(amk_attention_t, out, device index) of operands [tokens, heads, head_dim] after checking them."""
    torch = _torch or _load_torch()
    index = _device_index(q, "q")
    if q.dtype not in _BF16 or q.dim() != 3:
        _refuse(q, "q", index, _BF16, 3)
    if k.get_device() != index or k.dtype not in _BF16 or k.dim() != 3:
        _refuse(k, "k", index, _BF16, 3)
    if v.get_device() != index or v.dtype not in _BF16 or v.dim() != 3:
        _refuse(v, "v", index, _BF16, 3)
    tokens, heads, d = q.shape
    rows, kv_heads, _ = k.shape
    if (tokens | heads | d | rows | kv_heads) >> 31:
        _past_int32(tokens, heads, d, rows, kv_heads)
    if k.shape != v.shape or k.shape[2] != d:
        raise ValueError("k and v must be [rows, kv heads, head_dim] with q's head_dim")
    if out is None:
        out = torch.empty((tokens, heads, d), dtype=q.dtype, device=q.device)
    else:
        if out.get_device() != index or out.dtype not in _BF16 or out.dim() != 3:
            _refuse(out, "out", index, _BF16, 3)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    a = amk_attention_t(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), *_strides(q, "q"), *_strides(k, "k"),
                        *_strides(v, "v"), *_strides(out, "out"), heads, kv_heads, d,
                        d ** -0.5 if scale is None else scale)
    return a, out, index


def prompt_attention(q, k, v, cu_q=None, cu_k=None, scale: Optional[float] = None, out=None):
    """Causal attention over whole prompts (amk_prompt_attention; no gradients): q bf16
    [tokens, heads, head_dim], k and v [rows, kv heads, head_dim], any strides with contiguous
    heads (a cache layer kv[l, 0] is taken as kv[l, 0].transpose(0, 1)).  cu_q and
    cu_k: int32 device tensors [sequences + 1] of offsets, or both None for one
    sequence.  Rows of `out` outside every sequence are not written; without `out` they
    hold whatever the memory did."""
    a, out, index = _attention(q, k, v, scale, out)
    seqs, pq, pk = 1, None, None
    if (cu_q is None) != (cu_k is None):
        raise ValueError("cu_q and cu_k come together")
    if cu_q is not None:
        for t, what in ((cu_q, "cu_q"), (cu_k, "cu_k")):
            if t.get_device() != index or t.dtype != _torch.int32 or t.dim() != 1:
                _refuse(t, what, index, (_torch.int32,), 1)
            if not t.is_contiguous() or t.numel() != cu_q.numel() or t.numel() < 1:
                raise ValueError("cu_q and cu_k must be contiguous and of one length")
        seqs, pq, pk = cu_q.numel() - 1, cu_q.data_ptr(), cu_k.data_ptr()
        _int32(seqs, "the number of sequences")
    lib = load()
    tokens, rows = q.shape[0], k.shape[0]
    need = lib.amk_prompt_attention_workspace(a.n_heads, a.n_kv_heads, a.head_dim, seqs, tokens, rows)
    ws = _workspace(need, index) if need else None
    _call(index, lib.amk_prompt_attention, a, pq, pk, seqs, tokens, rows, ws.data_ptr() if need else None, need)
    return out


def tree_masks(parents):
    """The masks of a drafted tree: token i sees its ancestors and itself
    (parents[i] in [-1, i), -1 for a token that follows the context)."""
    masks = []
    for i, p in enumerate(parents):
        if not -1 <= p < i:
            raise ValueError(f"parents[{i}] = {p} is not in [-1, {i})")
        masks.append(1 << i | (masks[p] if p >= 0 else 0))
    return masks


def tree_attention(q, k, v, pos: int, masks, scale: Optional[float] = None, out=None):
    """Attention of n drafted tokens over a cache (amk_tree_attention; no gradients): q
    bf16 [n, heads, head_dim]; k and v [rows, kv heads, head_dim] as in prompt_attention, with
    at least pos + n rows; masks: n whole numbers, bit j of masks[i] set where token
    i sees row pos + j (tree_masks gives a tree's)."""
    a, out, index = _attention(q, k, v, scale, out)
    n = q.shape[0]
    if len(masks) != n:
        raise ValueError(f"{len(masks)} masks for {n} tokens")
    if n > AMK_TREE_MAX:
        raise ValueError(f"a tree has at most {AMK_TREE_MAX} tokens, not {n}")
    if pos < 0 or k.shape[0] < pos + n:
        raise ValueError(f"k and v have {k.shape[0]} rows, tokens at {pos} need {pos + n}")
    lib = load()
    need = lib.amk_tree_attention_workspace(a.n_heads, a.n_kv_heads, a.head_dim, n, pos)
    ws = _workspace(need, index) if need else None
    _call(index, lib.amk_tree_attention, a, n, pos, (ctypes.c_uint64 * n)(*masks), ws.data_ptr() if need else None, need)
    return out


def token_logprobs(logits, tokens=None, top: int = 0):
    """(logprob, entropy, top_ids, top_logprobs) of rows of logits (amk_token_logprobs; no
    gradients): logits fp32, bf16 or fp16 [n, vocab] with contiguous rows; tokens int32 [n], or
    None (logprob is then None); the `top` most probable tokens of each row."""
    torch = _torch or _load_torch()
    index = _device_index(logits, "logits")
    kind = _LOGITS.get(logits.dtype)
    if kind is None or logits.dim() != 2:
        _refuse(logits, "logits", index, tuple(_LOGITS), 2)
    n, vocab = logits.shape
    if (n | vocab) >> 31:
        _past_int32(n, vocab)
    if n and vocab > 1 and logits.stride(1) != 1:
        raise ValueError("logits must have contiguous rows")
    if not 0 <= top <= AMK_TOP_MAX:
        raise ValueError(f"top must be in [0, {AMK_TOP_MAX}]")
    lib = load()
    need = lib.amk_token_logprobs_workspace(kind, n, vocab, top)
    device = logits.device
    logprob = token_ptr = logprob_ptr = None
    if tokens is not None:
        if tokens.get_device() != index or tokens.dtype != torch.int32 or tokens.dim() != 1:
            _refuse(tokens, "tokens", index, (torch.int32,), 1)
        if tokens.numel() != n or not tokens.is_contiguous():
            raise ValueError(f"tokens must be {n} contiguous values")
        logprob = torch.empty(n, dtype=torch.float32, device=device)
        token_ptr, logprob_ptr = tokens.data_ptr(), logprob.data_ptr()
    entropy = torch.empty(n, dtype=torch.float32, device=device)
    ids = torch.empty((n, top), dtype=torch.int32, device=device)
    values = torch.empty((n, top), dtype=torch.float32, device=device)
    ws = _workspace(need, index) if need else None
    _call(index, lib.amk_token_logprobs, logits.data_ptr(), kind, logits.stride(0) if n > 1 else vocab, n, vocab,
          token_ptr, top, logprob_ptr, entropy.data_ptr(), ids.data_ptr() if top else None,
          values.data_ptr() if top else None, ws.data_ptr() if need else None, need)
    return logprob, entropy, ids, values


def kv_keep(kv, pos: int, rows) -> None:
    """Move cache rows pos + rows[i] to pos + i in every layer and head (amk_kv_keep):
    kv a contiguous 2-byte tensor [layers, 2, kv heads, max_seq, head_dim], rows
    strictly ascending whole numbers."""
    if _torch is None:
        _load_torch()
    index = _device_index(kv, "kv")
    if kv.dim() != 5 or kv.shape[1] != 2 or kv.element_size() != 2 or not kv.is_contiguous():
        raise ValueError("kv must be a contiguous bf16 tensor [layers, 2, kv heads, max_seq, head_dim]")
    layers, _, heads, cap, d = kv.shape
    n = len(rows)
    _int32(pos, "pos")
    if (layers | heads | cap | d) >> 31:
        _past_int32(layers, heads, cap, d)
    if n:
        _int32(min(rows), "a row"), _int32(max(rows), "a row")
    _call(index, load().amk_kv_keep, kv.data_ptr(), layers, heads, cap, d, pos, (ctypes.c_int32 * n)(*rows), n)


# ---- convenience: a decoder over torch device tensors ---------------------------------
def make_config(hidden: int, n_layers: int, n_heads: int, n_kv_heads: int, head_dim: int, intermediate: int,
                vocab: int, max_seq: int, rope_theta: float, rms_eps: float = 1e-5, tied_embeddings: bool = False,
                weight_format: str = "bf16", device: int = -1, group_size: int = 0) -> amk_config_t:
    fmt = {"bf16": AMK_WEIGHTS_BF16, "w8a16": AMK_WEIGHTS_W8A16, "w4a16": AMK_WEIGHTS_W4A16}[weight_format]
    return amk_config_t(AMK_ABI_VERSION, hidden, n_layers, n_heads, n_kv_heads, head_dim, intermediate, vocab,
                        max_seq, rope_theta, rms_eps, int(tied_embeddings), fmt, device, group_size)


_PROJ = (("q", "wq"), ("k", "wk"), ("v", "wv"), ("o", "wo"), ("gate", "wg"), ("up", "wu"), ("down", "wd"))


def expected_sizes(cfg: amk_config_t) -> Dict[str, int]:
    """Bytes every weight tensor must have for cfg.  The library receives bare
    pointers and reads these extents; a smaller tensor would be read past its
    end on the device, so the binding checks them before amk_create."""
    H, I, V = cfg.hidden, cfg.intermediate, cfg.vocab
    qd, kd = cfg.n_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim
    shapes = {"wq": (qd, H), "wk": (kd, H), "wv": (kd, H), "wo": (H, qd), "wg": (I, H), "wu": (I, H), "wd": (H, I)}
    group = cfg.group_size or 128

    def lin(out, inp):
        if cfg.weight_format == AMK_WEIGHTS_W8A16:
            return out * inp, 4 * out
        if cfg.weight_format == AMK_WEIGHTS_W4A16:
            return out * inp // 2, 2 * out * (inp // group)
        return 2 * out * inp, 0

    sizes = {"embed": 2 * V * H, "final_norm": 2 * H}
    names = [(f"layers.{l}.{n}", shapes[n]) for l in range(cfg.n_layers) for n in shapes]
    if not cfg.tied_embeddings:
        names.append(("lm_head", (V, H)))
    for l in range(cfg.n_layers):
        sizes[f"layers.{l}.attn_norm"] = sizes[f"layers.{l}.mlp_norm"] = 2 * H
    for name, (out, inp) in names:
        w, sc = lin(out, inp)
        sizes[name] = w
        if sc:
            sizes[name + ".scale"] = sc
    return sizes


def check_sizes(cfg: amk_config_t, tensors: Mapping[str, "object"]) -> None:
    """Raise ValueError unless every tensor amk_create will read is present with
    exactly the bytes cfg implies (device and layout are checked at create)."""
    for name, nbytes in expected_sizes(cfg).items():
        if name not in tensors:
            raise ValueError(f"missing tensor {name}")
        t = tensors[name]
        have = t.numel() * t.element_size()
        if have != nbytes:
            raise ValueError(f"{name} has {have} bytes, the config needs {nbytes}")


class Decoder:
    """One handle over weights that live in torch device tensors.

    ``tensors`` maps names to contiguous device tensors: 'embed' [V,H],
    'final_norm' [H], 'lm_head' [V,H] (untied), and per layer l
    'layers.{l}.attn_norm', 'layers.{l}.mlp_norm' (bf16 [H]) and the
    projections 'layers.{l}.w{q,k,v,o,g,u,d}' [out,in] -- bf16 (any 2-byte
    dtype holding bf16 bits) or, for W8A16, int8 with an fp32 scale tensor
    under the same name + '.scale', or, for W4A16, packed uint8 [out, in/2]
    with an fp16 [out, in/group] scale tensor under name + '.scale'.  The
    tensors are borrowed: they must
    outlive the decoder, which keeps references to them.  ``static=True``
    creates the handle with amk_create_static (no device allocation)."""

    def __init__(self, cfg: amk_config_t, tensors: Mapping[str, "object"], tuning: Optional[amk_tuning_t] = None,
                 static: bool = False):
        self.cfg = cfg
        check_sizes(cfg, tensors)
        self._keep: Dict[str, object] = dict(tensors)
        quant = cfg.weight_format in (AMK_WEIGHTS_W8A16, AMK_WEIGHTS_W4A16)
        fmt_name = "W8A16" if cfg.weight_format == AMK_WEIGHTS_W8A16 else "W4A16"
        scale_size = 4 if cfg.weight_format == AMK_WEIGHTS_W8A16 else 2

        def ptr(name):
            t = tensors[name]
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous device tensor")
            return t.data_ptr()

        def lin(name, quantized):
            if quantized:
                if tensors[name].element_size() != 1:
                    raise ValueError(f"{name} must be 1-byte elements under {fmt_name}")
                if tensors[name + ".scale"].element_size() != scale_size:
                    raise ValueError(f"{name}.scale must have {scale_size}-byte elements under {fmt_name}")
                return amk_linear_t(ptr(name), ptr(name + ".scale"))
            if tensors[name].element_size() != 2:
                raise ValueError(f"{name} must hold bf16 values")
            return amk_linear_t(ptr(name), None)

        L = cfg.n_layers
        self._layers = (amk_layer_weights_t * L)()
        for l in range(L):
            p = f"layers.{l}."
            lw = self._layers[l]
            lw.attn_norm = ptr(p + "attn_norm")
            lw.mlp_norm = ptr(p + "mlp_norm")
            for field, name in _PROJ:
                setattr(lw, field, lin(p + name, quant))
        lm = amk_linear_t(None, None) if cfg.tied_embeddings else lin("lm_head", quant)
        self._weights = amk_weights_t(ptr("embed"), ptr("final_norm"), lm, self._layers)
        import torch
        # the device amk_create resolved (-1 = the current device at creation)
        self._dev = cfg.device if cfg.device >= 0 else torch.cuda.current_device()
        self.handle = (amk_create_static if static else amk_create)(cfg, self._weights, tuning)

    def kv_cache_bytes(self) -> int:
        return amk_kv_cache_bytes(self.cfg)

    def step(self, token: int, pos: int, kv_cache, logits, stream: Optional[int] = None) -> None:
        """Enqueue one decode step; kv_cache / logits are contiguous device
        tensors of at least amk_kv_cache_bytes and 4 * vocab bytes."""
        if not hasattr(self, "_need"):
            self._need = (amk_kv_cache_bytes(self.cfg), 4 * self.cfg.vocab)
        dev = self._dev
        for t, need, what in ((kv_cache, self._need[0], "kv_cache"), (logits, self._need[1], "logits")):
            if not t.is_cuda or t.device.index != dev:
                raise ValueError(f"{what} must be a tensor on cuda:{dev}, the decoder's device")
            if not t.is_contiguous() or t.numel() * t.element_size() < need:
                raise ValueError(f"{what} must be contiguous with at least {need} bytes")
        if stream is None:
            import torch
            stream = torch.cuda.current_stream().cuda_stream
        amk_decode_step(self.handle, token, pos, kv_cache.data_ptr(), logits.data_ptr(), stream)

    def extend(self, tokens, pos: int, kv_cache, n_logits: Optional[int] = None, parents=None):
        """Run several tokens through the model behind the `pos` positions in the cache
        (amk_extend): a prompt or part of one, or, with `parents` (at most AMK_TREE_MAX
        tokens, parents[i] in [-1, i)), a drafted tree.  Appends their K and V rows at
        pos .. pos + n - 1 and returns the logits of the last n_logits tokens (default
        all) as fp32 [n_logits, vocab], on torch's current stream."""
        import torch
        n = len(tokens)
        n_logits = n if n_logits is None else n_logits
        if not 0 <= n_logits <= n:
            raise ValueError(f"n_logits must be in [0, {n}]")
        if parents is not None and len(parents) != n:
            raise ValueError(f"{len(parents)} parents for {n} tokens")
        _int32(pos, "pos")
        for given, what in ((tokens, "a token"), (parents or (), "a parent")):
            if len(given):
                _int32(min(given), what), _int32(max(given), what)
        _load_torch()
        device = torch.device("cuda", self._dev)
        need = amk_kv_cache_bytes(self.cfg)
        if not kv_cache.is_cuda or kv_cache.device != device:
            raise ValueError(f"kv_cache must be a tensor on {device}, the decoder's device")
        if not kv_cache.is_contiguous() or kv_cache.numel() * kv_cache.element_size() < need:
            raise ValueError(f"kv_cache must be contiguous with at least {need} bytes")
        logits = torch.empty(n_logits, self.cfg.vocab, dtype=torch.float32, device=device)
        if n == 0:
            return logits
        lib = load()
        ws = _workspace(lib.amk_extend_workspace(self.handle, n), self._dev)
        ids = (ctypes.c_int32 * n)(*tokens)
        par = None if parents is None else (ctypes.c_int32 * n)(*parents)
        _call(self._dev, lib.amk_extend, self.handle, ids, n, pos, par, kv_cache.data_ptr(),
              logits.data_ptr() if n_logits else None, n_logits, ws.data_ptr(), ws.numel())
        return logits

    def score(self, tokens, pos: int, kv_cache, top: int = 0):
        """Score a text behind the `pos` positions in the cache: (logprob, entropy,
        top_ids, top_logprobs) of tokens[1:], each given those before it
        (token_logprobs over extend's logits).  Appends the rows of all its tokens.  The
        tokens are copied to the device, which waits for what its stream has queued: not for
        graphs."""
        import torch
        if len(tokens) < 2:
            raise ValueError("a text to score has at least two tokens")
        # a long text is taken in pieces: nothing runs before all of it is found good
        if not 0 <= top <= min(AMK_TOP_MAX, self.cfg.vocab):
            raise ValueError(f"top must be in [0, {min(AMK_TOP_MAX, self.cfg.vocab)}]")
        least, most = min(tokens), max(tokens)
        _int32(least, "a token"), _int32(most, "a token")
        if least < 0 or most >= self.cfg.vocab:
            raise AmkError(AMK_ERR_INVALID_ARGUMENT, "amk_extend")
        if pos + len(tokens) > self.cfg.max_seq:
            raise ValueError(f"{len(tokens)} tokens at {pos} exceed the cache's {self.cfg.max_seq} positions")
        parts = []
        for at in range(0, len(tokens), _SCORE_CHUNK):
            piece = tokens[at:at + _SCORE_CHUNK]
            given = torch.tensor(list(tokens[at + 1:at + 1 + len(piece)]), dtype=torch.int32, device=kv_cache.device)
            # the last token's logits predict what follows the text: not needed
            logits = self.extend(piece, pos + at, kv_cache)[:len(given)]
            parts.append(token_logprobs(logits, given, top))
        return parts[0] if len(parts) == 1 else tuple(torch.cat(p) for p in zip(*parts))

    def keep(self, pos: int, rows, kv_cache) -> None:
        """After extend with a drafted tree at `pos`: make the accepted tokens' rows
        (ascending indices into the tree) follow each other from pos on (amk_kv_keep)."""
        c = self.cfg
        shape = (c.n_layers, 2, c.n_kv_heads, c.max_seq, c.head_dim)
        count = c.n_layers * 2 * c.n_kv_heads * c.max_seq * c.head_dim
        if kv_cache.element_size() != 2 or not kv_cache.is_contiguous() or kv_cache.numel() < count:
            raise ValueError(f"kv_cache must be contiguous 2-byte elements, at least {count}")
        if not kv_cache.is_cuda or kv_cache.device.index != self._dev:
            raise ValueError(f"kv_cache must be a tensor on cuda:{self._dev}, the decoder's device")
        kv_keep(kv_cache.view(-1)[:count].view(shape), pos, rows)

    def next_token(self, stream: Optional[int] = None) -> int:
        if stream is None:
            import torch
            stream = torch.cuda.current_stream().cuda_stream
        return amk_copy_next_token(self.handle, stream)

    def status(self) -> int:
        return amk_get_status(self.handle)

    def reset(self) -> None:
        amk_reset(self.handle)

    def set_abort(self, value: int) -> None:
        amk_set_abort(self.handle, value)

    def close(self) -> None:
        if getattr(self, "handle", None):
            amk_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
