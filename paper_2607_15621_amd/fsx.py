"""Thin Python binding of libfsx (include/fsx.h): argument marshalling only.

Every step of the expert tick runs in the HIP library; this module only turns
torch tensors / numpy arrays into the raw pointers and sizes the C ABI takes,
and turns non-zero status codes into exceptions.  If the library has not been
built, loading it raises -- there is no fallback.
"""

from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfsx.so")

F32, BF16, FP8_E4M3 = 0, 1, 2
APPEND_RING, APPEND_ERROR = 0, 1
CACHE_HEAD_MAJOR, CACHE_TOKEN_MAJOR, CACHE_SHARED = 0, 1, 2
FLAG_GENERIC, FLAG_MULTI_LAUNCH, FLAG_TRACE = 1, 2, 4
HEAD_MEAN_LINEAR, HEAD_QUERY_MLP = 0, 1
PROMPT_AUTO, PROMPT_CHUNKS, PROMPT_TILES, PROMPT_TURNS = 0, 1, 2, 3
MAX_BATCH = 64
STATUS = {0: "FSX_OK", 1: "FSX_E_INVALID", 2: "FSX_E_UNSUPPORTED", 3: "FSX_E_CAPACITY", 4: "FSX_E_OOM",
          5: "FSX_E_HIP"}
SYMBOLS = ("fsx_expert_create", "fsx_expert_forward", "fsx_cache_append_rows", "fsx_expert_status",
           "fsx_expert_trace", "fsx_expert_destroy", "fsx_last_error", "fsx_expert_info", "fsx_version",
           "fsx_probe_hbm_read", "fsx_expert_forward_noalloc", "fsx_cache_append_rows_quantize",
           "fsx_loop_create", "fsx_loop_tick", "fsx_loop_append", "fsx_loop_sync", "fsx_loop_destroy",
           "fsx_loop_last_error", "fsx_backbone_create", "fsx_backbone_append", "fsx_backbone_info",
           "fsx_backbone_destroy", "fsx_prompt_attention", "fsx_prompt_attention_workspace", "fsx_cache_replace_rows",
           "fsx_cache_read_rows", "fsx_backbone_rebuild")


class FsxError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class ExpertCfg(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("n_expert_tokens", ctypes.c_int32),
                ("n_out", ctypes.c_int32), ("max_batch", ctypes.c_int32), ("max_frame_tokens", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rope_base", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("flags", ctypes.c_int32), ("tick_timeout_us", ctypes.c_int32), ("head_kind", ctypes.c_int32),
                ("head_hidden", ctypes.c_int32)]


class HeadWeights(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("b", ctypes.c_void_p), ("w2", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "attn_norm", "ffn_norm")]


class BackboneCfg(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("max_new_rows", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rope_base", ctypes.c_float),
                ("rms_eps", ctypes.c_float), ("max_prompt_rows", ctypes.c_int32)]


class LoopTickInfo(ctypes.Structure):
    _fields_ = [("tick", ctypes.c_int64), ("published", ctypes.c_int32), ("staleness", ctypes.c_int32),
                ("start", ctypes.c_int64 * MAX_BATCH), ("len", ctypes.c_int64 * MAX_BATCH),
                ("pos", ctypes.c_int64 * MAX_BATCH)]


class PromptDesc(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("q_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("kernel", ctypes.c_int32)] + \
               [(n, ctypes.c_int64) for n in ("q_rows", "k_rows", "q_row", "q_head", "k_row", "k_head", "v_row", "v_head",
                                              "out_row", "out_head")]


class CacheDescC(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("capacity", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("start", ctypes.POINTER(ctypes.c_int64)), ("len", ctypes.POINTER(ctypes.c_int64)),
                ("pos", ctypes.POINTER(ctypes.c_int64))]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libfsx.so (built by ``paper_2607_15621_amd.build``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_15621_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.fsx_expert_create.argtypes = [ctypes.POINTER(ExpertCfg), ctypes.POINTER(LayerWeights), vp,
                                        ctypes.POINTER(HeadWeights), vp, ctypes.POINTER(vp)]
        L.fsx_expert_forward.argtypes = [vp, ctypes.POINTER(CacheDescC), vp, i32, i32, vp, vp, vp]
        L.fsx_cache_append_rows.argtypes = [ctypes.POINTER(CacheDescC), vp, vp, i32, i32, vp]
        L.fsx_expert_status.argtypes = [vp, vp]
        L.fsx_expert_trace.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64), i64, ctypes.POINTER(i32),
                                       ctypes.POINTER(i32), vp]
        L.fsx_expert_destroy.argtypes = [vp]
        L.fsx_expert_destroy.restype = None
        L.fsx_last_error.restype = ctypes.c_char_p
        L.fsx_expert_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.fsx_version.restype = ctypes.c_char_p
        L.fsx_probe_hbm_read.argtypes = [vp, i64, i32, vp, vp]
        L.fsx_expert_forward_noalloc.argtypes = [vp, ctypes.POINTER(CacheDescC), vp, i32, i32, vp, vp, vp]
        L.fsx_expert_forward_noalloc.restype = ctypes.c_int
        L.fsx_cache_append_rows_quantize.argtypes = [ctypes.POINTER(CacheDescC), vp, vp, i32, i32, i32, vp]
        L.fsx_loop_create.argtypes = [vp, ctypes.POINTER(CacheDescC), i32, i32, vp, vp, ctypes.POINTER(vp)]
        L.fsx_loop_tick.argtypes = [vp, vp, i32, i32, vp, vp, ctypes.POINTER(LoopTickInfo)]
        L.fsx_loop_append.argtypes = [vp, vp, vp, i32, i32]
        L.fsx_loop_sync.argtypes = [vp, ctypes.POINTER(CacheDescC)]
        L.fsx_loop_destroy.argtypes = [vp]
        L.fsx_loop_destroy.restype = None
        L.fsx_loop_last_error.restype = ctypes.c_char_p
        for n in ("fsx_cache_append_rows_quantize", "fsx_loop_create", "fsx_loop_tick", "fsx_loop_append",
                  "fsx_loop_sync"):
            getattr(L, n).restype = ctypes.c_int
        L.fsx_backbone_create.argtypes = [ctypes.POINTER(BackboneCfg), ctypes.POINTER(LayerWeights), vp,
                                          ctypes.POINTER(vp)]
        L.fsx_backbone_append.argtypes = [vp, ctypes.POINTER(CacheDescC), vp, i32, i32, vp, i32, vp]
        L.fsx_backbone_rebuild.argtypes = [vp, ctypes.POINTER(CacheDescC), vp, ctypes.POINTER(i64), vp, ctypes.c_float, i32, vp]
        L.fsx_backbone_info.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.fsx_backbone_destroy.argtypes = [vp]
        L.fsx_backbone_destroy.restype = None
        for n in ("fsx_backbone_create", "fsx_backbone_append", "fsx_backbone_info", "fsx_backbone_rebuild"):
            getattr(L, n).restype = ctypes.c_int
        P64 = ctypes.POINTER(i64)
        L.fsx_prompt_attention.argtypes = [ctypes.POINTER(PromptDesc), vp, vp, vp, vp, vp, i32, P64, P64, P64, P64, vp, i64,
                                           vp]
        L.fsx_prompt_attention_workspace.argtypes = [ctypes.POINTER(PromptDesc), i32, P64, P64, P64]
        L.fsx_cache_replace_rows.argtypes = [ctypes.POINTER(CacheDescC), i32, i32, vp, vp, i32, i64, P64, P64,
                                             ctypes.c_float, i32, vp]
        L.fsx_cache_read_rows.argtypes = [ctypes.POINTER(CacheDescC), i32, i32, P64, vp, vp, i32, i64, P64, P64, vp]
        for n in ("fsx_prompt_attention", "fsx_prompt_attention_workspace", "fsx_cache_replace_rows",
                  "fsx_cache_read_rows", "fsx_backbone_rebuild"):
            getattr(L, n).restype = ctypes.c_int
        for n in ("fsx_expert_create", "fsx_expert_forward", "fsx_cache_append_rows", "fsx_expert_info",
                  "fsx_expert_status", "fsx_expert_trace", "fsx_probe_hbm_read"):
            getattr(L, n).restype = ctypes.c_int
        _lib = L
    return _lib


def last_error() -> str:
    return lib().fsx_last_error().decode()


def version() -> str:
    return lib().fsx_version().decode()


def _check(code: int):
    if code != 0:
        raise FsxError(code, last_error())


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    return int(t.data_ptr())


def _stream(stream) -> int:
    if stream is None:
        import torch

        return int(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


def make_cfg(n_layers, d_model, n_heads, head_dim, d_ffn, n_expert_tokens=10, n_out=10, max_batch=1,
             max_frame_tokens=0, dtype=BF16, rope_base=10000.0, rms_eps=1e-6, flags=0,
             tick_timeout_us=0, head_kind=HEAD_MEAN_LINEAR, head_hidden=0) -> ExpertCfg:
    return ExpertCfg(n_layers, d_model, n_heads, head_dim, d_ffn, n_expert_tokens, n_out, max_batch,
                     max_frame_tokens, dtype, rope_base, rms_eps, flags, tick_timeout_us, head_kind, head_hidden)


class Expert:
    """Handle returned by fsx_expert_create; fsx_expert_destroy runs on close()."""

    def __init__(self, handle: int, cfg: ExpertCfg):
        self.handle = handle
        self.cfg = cfg

    def close(self):
        if self.handle:
            lib().fsx_expert_destroy(ctypes.c_void_p(self.handle))
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def expert_create(cfg: ExpertCfg, layers: Sequence[dict], final_norm, head, stream=None) -> Expert:
    """fsx_expert_create.  layers: per layer a dict of device tensors (wq, wk, wv, wo, w_gate, w_up,
    w_down, attn_norm, ffn_norm) in nn.Linear layout.  head: the mean-pool head's weight [n_out][d], or a dict
    w1, b1, w2, b2 of device tensors for the query head."""
    arr = (LayerWeights * len(layers))()
    for i, lw in enumerate(layers):
        arr[i] = LayerWeights(*[_ptr(lw[n]) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down",
                                                        "attn_norm", "ffn_norm")])
    if isinstance(head, dict):
        hw = HeadWeights(_ptr(head["w1"]), _ptr(head["b1"]), _ptr(head["w2"]), _ptr(head["b2"]))
    else:
        hw = HeadWeights(_ptr(head), None, None, None)
    out = ctypes.c_void_p(0)
    _check(lib().fsx_expert_create(ctypes.byref(cfg), arr if len(layers) else None, _ptr(final_norm),
                                   ctypes.byref(hw), _stream(stream), ctypes.byref(out)))
    return Expert(out.value, cfg)


def expert_info(ex: Expert):
    path, wb, wsb = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int64()
    _check(lib().fsx_expert_info(ctypes.c_void_p(ex.handle), ctypes.byref(path), ctypes.byref(wb),
                                 ctypes.byref(wsb)))
    return {"path": path.value, "weight_bytes": wb.value, "workspace_bytes": wsb.value}


class CacheDesc:
    """fsx_cache_desc: device K/V tensors, [batch][n_layers][H][capacity][Dh] (layout CACHE_HEAD_MAJOR) or
    [batch][n_layers][capacity][H][Dh] (CACHE_TOKEN_MAJOR), plus host ring state.

    start / len / pos are numpy int64 arrays that the C side reads, and updates in place on append.
    """

    def __init__(self, k, v, dtype: int, n_layers: int, n_heads: int, head_dim: int, capacity: int,
                 lengths, positions=None, starts=None, k_scale=None, v_scale=None, layout: int = CACHE_HEAD_MAJOR):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        batch = len(lengths)
        self.len = np.ascontiguousarray(np.asarray(lengths, dtype=np.int64))
        self.pos = np.ascontiguousarray(np.asarray(lengths if positions is None else positions, dtype=np.int64))
        self.start = np.ascontiguousarray(np.zeros(batch, np.int64) if starts is None else
                                          np.asarray(starts, dtype=np.int64))
        P = ctypes.POINTER(ctypes.c_int64)
        self.layout = layout
        self.c = CacheDescC(dtype, batch, n_layers, n_heads, head_dim, layout, capacity, _ptr(k), _ptr(v),
                            _ptr(k_scale), _ptr(v_scale), self.start.ctypes.data_as(P),
                            self.len.ctypes.data_as(P), self.pos.ctypes.data_as(P))


def expert_forward(ex: Expert, cache: CacheDesc, tokens, batch: int, n_frame_tokens: int, waypoints,
                   hidden=None, stream=None):
    """fsx_expert_forward: one tick for `batch` agents (enqueued on `stream`)."""
    _check(lib().fsx_expert_forward(ctypes.c_void_p(ex.handle), ctypes.byref(cache.c), _ptr(tokens), batch,
                                    n_frame_tokens, _ptr(waypoints), _ptr(hidden), _stream(stream)))


def expert_forward_noalloc(ex: Expert, cache: CacheDesc, tokens, batch: int, n_frame_tokens: int, waypoints,
                           hidden=None, stream=None):
    """fsx_expert_forward_noalloc: the same tick, its workspace in the library's static device array."""
    _check(lib().fsx_expert_forward_noalloc(ctypes.c_void_p(ex.handle), ctypes.byref(cache.c), _ptr(tokens), batch,
                                            n_frame_tokens, _ptr(waypoints), _ptr(hidden), _stream(stream)))


def expert_status(ex: Expert, stream=None):
    """fsx_expert_status: synchronise the stream; raise if a tick of this handle timed out."""
    _check(lib().fsx_expert_status(ctypes.c_void_p(ex.handle), _stream(stream)))


def expert_trace(ex: Expert, n_wg_max: int = 1024, stream=None) -> np.ndarray:
    """fsx_expert_trace: [n_wg][n_events] real-time stamps (100 MHz) of the last tick."""
    n_layers = ex.cfg.n_layers
    cap = n_wg_max * (2 + 16 * n_layers + 1)
    buf = np.zeros(cap, np.uint64)
    nw, ne = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().fsx_expert_trace(ctypes.c_void_p(ex.handle), buf.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)),
                                  cap, ctypes.byref(nw), ctypes.byref(ne), _stream(stream)))
    return buf[: nw.value * ne.value].reshape(nw.value, ne.value)


def cache_append_rows(cache: CacheDesc, k_rows, v_rows, n_rows: int, policy: int = APPEND_RING, stream=None):
    """fsx_cache_append_rows: enqueue the row copy; host ring state is updated on return."""
    _check(lib().fsx_cache_append_rows(ctypes.byref(cache.c), _ptr(k_rows), _ptr(v_rows), n_rows, policy,
                                       _stream(stream)))


def probe_hbm_read(buf, nbytes: int, mode: int, sink, stream=None):
    """fsx_probe_hbm_read: enqueue one read-only pass over nbytes of buf (measurement helper)."""
    _check(lib().fsx_probe_hbm_read(_ptr(buf), nbytes, mode, _ptr(sink), _stream(stream)))


def cache_append_rows_quantize(cache: CacheDesc, k_rows, v_rows, rows_dtype: int, n_rows: int,
                               policy: int = APPEND_RING, stream=None):
    """fsx_cache_append_rows_quantize: bf16 / fp32 rows encoded into an fp8 cache with its scales."""
    _check(lib().fsx_cache_append_rows_quantize(ctypes.byref(cache.c), _ptr(k_rows), _ptr(v_rows), rows_dtype,
                                                n_rows, policy, _stream(stream)))


class PackedRows:
    """Rows of several sequences (or agents) in one tensor: sequence i in rows start[i] .. start[i] + len[i] - 1; without
    starts, one after the other."""

    def __init__(self, lengths, starts=None):
        self.len = np.array(lengths, dtype=np.int64).reshape(-1)
        self.start = (np.cumsum(self.len) - self.len if starts is None else
                      np.array(starts, dtype=np.int64).reshape(-1))
        if len(self.start) != len(self.len):
            raise ValueError("as many starts as lengths")
        P = ctypes.POINTER(ctypes.c_int64)
        self.n, self.c_start, self.c_len = len(self.len), self.start.ctypes.data_as(P), self.len.ctypes.data_as(P)


_dtypes = {}


def _dtype_of(t) -> int:
    code = _dtypes.get(t.dtype)
    if code is None:
        import torch

        _dtypes.update({torch.float32: F32, torch.bfloat16: BF16})
        code = _dtypes.get(t.dtype)
        if code is None:
            raise ValueError(f"tensors of dtype {t.dtype} are not taken here: float32 or bfloat16")
    return code


def _stream_on(stream, *tensors) -> int:
    """The stream's handle, for a call on these tensors (some may be None).  The library's kernels run on the current device: a
    tensor of another one, or of the host, is refused."""
    device = None
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at < 0 or (device is not None and at != device):
                raise ValueError("tensors must be on the current device")
            device = at
    if device is None:
        return _stream(stream)
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
        current = stream.device_index
    else:
        current = torch.cuda.current_device()
    if current != device:
        raise ValueError("tensors must be on the current device")
    return _stream(stream)


def _prompt_desc(q, k, v, out, scale: float, kernel: int) -> PromptDesc:
    """Tensors [rows][heads][head_dim], their last dimension dense."""
    sq, sk, so, tq, tk, tv, to = q.shape, k.shape, out.shape, q.stride(), k.stride(), v.stride(), out.stride()
    if len(sq) != 3 or len(sk) != 3 or sk != v.shape or sq != so or sq[2] != sk[2]:
        raise ValueError("q and out must be [rows][heads][head_dim], k and v too, with as many channels")
    if not tq[2] == tk[2] == tv[2] == to[2] == 1:
        raise ValueError("q, k, v and out must have a dense last dimension")
    if _dtype_of(k) != BF16 or _dtype_of(v) != BF16:
        raise ValueError("k and v must be bfloat16")
    return PromptDesc(sq[1], sk[1], sq[2], _dtype_of(q), _dtype_of(out), scale, kernel, sq[0], sk[0], tq[0], tq[1], tk[0], tk[1],
                      tv[0], tv[1], to[0], to[1])


def prompt_attention(q, k, v, out, q_rows: PackedRows, k_rows: Optional[PackedRows] = None, scale: float = 0.0, lse=None,
                     workspace=None, stream=None, kernel: int = PROMPT_AUTO):
    """fsx_prompt_attention: causal attention of packed sequences.  q, out [rows][n_heads][head_dim], k, v
    [rows][n_kv_heads][head_dim] (any row and head strides); lse [rows][n_heads] float32, dense, or None; workspace a dense
    device tensor of prompt_attention_workspace bytes, or None (keys are then not split over workgroups)."""
    if lse is not None and (_dtype_of(lse) != F32 or tuple(lse.shape) != tuple(q.shape[:2]) or not lse.is_contiguous()):
        raise ValueError("lse must be a dense float32 [rows][n_heads]")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be a dense tensor")
    if k_rows is not None and k_rows.n != q_rows.n:
        raise ValueError("as many sequences of keys as of queries")
    d = _prompt_desc(q, k, v, out, scale, kernel)
    _check(lib().fsx_prompt_attention(ctypes.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), q_rows.n,
                                      q_rows.c_start, q_rows.c_len, k_rows.c_start if k_rows is not None else None,
                                      k_rows.c_len if k_rows is not None else None, _ptr(workspace),
                                      workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                      _stream_on(stream, q, k, v, out, lse, workspace)))


def prompt_attention_workspace(q, k, q_rows: PackedRows, k_rows: Optional[PackedRows] = None, kernel: int = PROMPT_AUTO) -> int:
    """fsx_prompt_attention_workspace: bytes of the workspace that the call can use (0: none)."""
    if k_rows is not None and k_rows.n != q_rows.n:
        raise ValueError("as many sequences of keys as of queries")
    d, need = _prompt_desc(q, k, k, q, 0.0, kernel), ctypes.c_int64()
    _check(lib().fsx_prompt_attention_workspace(ctypes.byref(d), q_rows.n, q_rows.c_len,
                                                k_rows.c_len if k_rows is not None else None, ctypes.byref(need)))
    return need.value


def _row_tensors(cache: CacheDesc, n_layers: int, k_rows, v_rows, rows: PackedRows):
    """Dtype and total rows of packed rows [n_layers][total_rows][H][Dh] (either tensor may be None)."""
    if rows.n != cache.c.batch:
        raise ValueError("rows of every agent of the cache")
    some = k_rows if k_rows is not None else v_rows
    if some is None:
        return BF16, int((rows.start + rows.len).max(initial=0))
    shape = some.shape
    if len(shape) != 4 or shape[0] != n_layers or shape[2] != cache.c.n_heads or shape[3] != cache.c.head_dim or \
            not some.is_contiguous() or \
            (v_rows is not None and (v_rows.shape != shape or v_rows.dtype != some.dtype or not v_rows.is_contiguous())):
        raise ValueError("packed rows must be dense [n_layers][rows][n_heads][head_dim] tensors of one dtype")
    return _dtype_of(some), shape[1]


def cache_replace_rows(cache: CacheDesc, layer: int, n_layers: int, k_rows, v_rows, rows: PackedRows, headroom: float = 1.0,
                       policy: int = APPEND_RING, stream=None):
    """fsx_cache_replace_rows: the rows of every agent with rows.len > 0, in layers layer .. layer + n_layers - 1, become
    packed rows [n_layers][total][H][Dh]; an fp8 cache's scales are found from them."""
    dtype, total = _row_tensors(cache, n_layers, k_rows, v_rows, rows)
    _check(lib().fsx_cache_replace_rows(ctypes.byref(cache.c), layer, n_layers, _ptr(k_rows), _ptr(v_rows), dtype, total,
                                        rows.c_start, rows.c_len, headroom, policy, _stream_on(stream, k_rows, v_rows)))


def cache_read_rows(cache: CacheDesc, layer: int, n_layers: int, k_rows, v_rows, rows: PackedRows, first=None, stream=None):
    """fsx_cache_read_rows: cached rows first[b] .. first[b] + rows.len[b] - 1 (0: the oldest valid row) into packed rows
    [n_layers][total][H][Dh], decoded; k_rows or v_rows may be None."""
    dtype, total = _row_tensors(cache, n_layers, k_rows, v_rows, rows)
    if first is not None:
        first = np.array(first, dtype=np.int64).reshape(-1)
        if len(first) != rows.n:
            raise ValueError("a first row of every agent of the cache")
    _check(lib().fsx_cache_read_rows(ctypes.byref(cache.c), layer, n_layers,
                                     first.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)) if first is not None else None,
                                     _ptr(k_rows), _ptr(v_rows), dtype, total, rows.c_start, rows.c_len,
                                     _stream_on(stream, k_rows, v_rows)))


class Loop:
    """fsx_loop: the asynchronous deployment loop (expert every tick, appends on a second stream)."""

    def __init__(self, ex: Expert, cache: CacheDesc, append_every: int, expert_stream, append_stream,
                 policy: int = APPEND_RING):
        self.ex, self.cache = ex, cache  # the loop reads their device buffers
        out = ctypes.c_void_p(0)
        self._check(lib().fsx_loop_create(ctypes.c_void_p(ex.handle), ctypes.byref(cache.c), append_every, policy,
                                          _stream(expert_stream), _stream(append_stream), ctypes.byref(out)))
        self.handle = out.value

    @staticmethod
    def _check(code):
        if code != 0:
            raise FsxError(code, lib().fsx_loop_last_error().decode())

    def tick(self, tokens, batch: int, n_frame_tokens: int, waypoints, hidden=None) -> dict:
        info = LoopTickInfo()
        self._check(lib().fsx_loop_tick(ctypes.c_void_p(self.handle), _ptr(tokens), batch, n_frame_tokens,
                                        _ptr(waypoints), _ptr(hidden), ctypes.byref(info)))
        return {"tick": info.tick, "published": info.published, "staleness": info.staleness,
                "start": list(info.start[:batch]), "len": list(info.len[:batch]), "pos": list(info.pos[:batch])}

    def append(self, k_rows, v_rows, rows_dtype: int, n_rows: int):
        self._check(lib().fsx_loop_append(ctypes.c_void_p(self.handle), _ptr(k_rows), _ptr(v_rows), rows_dtype,
                                          n_rows))

    def sync(self, cache_out: Optional[CacheDesc] = None):
        self._check(lib().fsx_loop_sync(ctypes.c_void_p(self.handle),
                                        ctypes.byref(cache_out.c) if cache_out is not None else None))

    def close(self):
        if self.handle:
            lib().fsx_loop_destroy(ctypes.c_void_p(self.handle))
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Backbone:
    """fsx_backbone: the backbone's incremental forward that produces the appended cache rows."""

    def __init__(self, cfg: BackboneCfg, layers: Sequence[dict], stream=None):
        arr = (LayerWeights * len(layers))()
        for i, lw in enumerate(layers):
            arr[i] = LayerWeights(*[_ptr(lw[n]) for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down",
                                                            "attn_norm", "ffn_norm")])
        out = ctypes.c_void_p(0)
        _check(lib().fsx_backbone_create(ctypes.byref(cfg), arr, _stream(stream), ctypes.byref(out)))
        self.handle, self.cfg = out.value, cfg

    def append(self, cache: CacheDesc, tokens, batch: int, n_rows: int, hidden=None, policy: int = APPEND_RING,
               stream=None):
        _check(lib().fsx_backbone_append(ctypes.c_void_p(self.handle), ctypes.byref(cache.c), _ptr(tokens), batch,
                                         n_rows, _ptr(hidden), policy, _stream(stream)))

    def rebuild(self, cache: CacheDesc, tokens, lengths, hidden=None, headroom: float = 1.0, policy: int = APPEND_RING,
                stream=None):
        """fsx_backbone_rebuild: whole prompts, tokens [sum of lengths][d] bfloat16 (rows behind them are not read), replace the
        rows of the agents with lengths > 0; hidden [n_layers][sum of lengths][d] float32, or None.  Both dense."""
        n = PackedRows(lengths)
        if n.n != cache.c.batch:
            raise ValueError("a length of every agent of the cache")
        rows, d = int(n.len.sum()), self.cfg.d_model
        if tokens is not None and (tokens.dim() != 2 or tokens.shape[0] < rows or tokens.shape[1] != d or
                                   _dtype_of(tokens) != BF16 or not tokens.is_contiguous()):
            raise ValueError("tokens must be a dense bfloat16 [sum of lengths][d_model]")
        if hidden is not None and (tuple(hidden.shape) != (self.cfg.n_layers, rows, d) or _dtype_of(hidden) != F32 or
                                   not hidden.is_contiguous()):
            raise ValueError("hidden must be a dense float32 [n_layers][sum of lengths][d_model]")
        _check(lib().fsx_backbone_rebuild(ctypes.c_void_p(self.handle), ctypes.byref(cache.c), _ptr(tokens), n.c_len,
                                          _ptr(hidden), headroom, policy, _stream_on(stream, tokens, hidden)))

    def info(self):
        wb, wsb = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().fsx_backbone_info(ctypes.c_void_p(self.handle), ctypes.byref(wb), ctypes.byref(wsb)))
        return {"weight_bytes": wb.value, "workspace_bytes": wsb.value}

    def close(self):
        if self.handle:
            lib().fsx_backbone_destroy(ctypes.c_void_p(self.handle))
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
