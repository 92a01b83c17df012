"""Python binding of libc2kv.so, the C2KV compose-and-attend path on MI355X.

Argument marshalling only: torch tensors supply device memory and the current
HIP stream; every step of the path runs in the library's HIP kernels.  Names
follow the C ABI in include/c2kv.h (c2kv_compose, c2kv_attend,
c2kv_compose_attend, ...).  There is no fallback: if the library is missing,
importing the binding raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# C2KV_LIBRARY selects another build of the same library (e.g. one with extra flags)
LIB_PATH = os.environ.get("C2KV_LIBRARY") or os.path.join(_PKG, "libc2kv.so")

C2KV_OK, C2KV_E_INVAL, C2KV_E_UNSUPPORTED, C2KV_E_WORKSPACE, C2KV_E_HIP, C2KV_E_NOMEM, \
    C2KV_E_STATE = 0, -1, -2, -3, -4, -5, -6
C2KV_F32, C2KV_BF16, C2KV_I8 = 0, 1, 2
C2KV_KEYS_ROPE_AT_ORIG, C2KV_KEYS_PRE_ROPE = 0, 1
C2KV_POOL_FULL, C2KV_POOL_COMPRESSED = 0, 1
_DTYPE_CODE = {"f32": C2KV_F32, "bf16": C2KV_BF16, "i8": C2KV_I8}

EXPORTED = [
    "c2kv_plan_create", "c2kv_plan_destroy", "c2kv_plan_get_info", "c2kv_plan_get_requests",
    "c2kv_plan_get_slots", "c2kv_plan_get_block_table", "c2kv_plan_upload", "c2kv_compose",
    "c2kv_attend", "c2kv_compose_attend", "c2kv_timing_enable", "c2kv_timing_reset",
    "c2kv_timing_read", "c2kv_last_error", "c2kv_version", "c2kv_host_alloc",
    "c2kv_host_free", "c2kv_load", "c2kv_sif_plan_create", "c2kv_compose_attend_static",
    "c2kv_cache_write", "c2kv_cache_read", "c2kv_cache_attend_workspace", "c2kv_cache_attend",
    "c2kv_pool_write",
]
STATIC_SCRATCH_BYTES = 32 << 20   # C2KV_STATIC_SCRATCH_BYTES


class C2KVError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"c2kv status {status}: {msg}")
        self.status = status


class AttnCfg(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("act_dtype", ctypes.c_int32),
                ("rope_base", ctypes.c_double), ("softmax_scale", ctypes.c_float)]


class ComposeDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("req_seg_off", ctypes.c_void_p), ("seg_row0", ctypes.c_void_p),
                ("seg_span", ctypes.c_void_p), ("seg_orig_pos0", ctypes.c_void_p),
                ("seg_new_pos0", ctypes.c_void_p), ("seg_kept_off", ctypes.c_void_p),
                ("kept_idx", ctypes.c_void_p), ("key_encoding", ctypes.c_int32),
                ("pool_layout", ctypes.c_int32)]


class PlanOpts(ctypes.Structure):
    _fields_ = [("page_size", ctypes.c_int32), ("kv_splits", ctypes.c_int32),
                ("rows_per_block", ctypes.c_int32), ("num_cus", ctypes.c_int32),
                ("merge_mode", ctypes.c_int32)]


class PoolDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_rows", ctypes.c_int64)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class ChunksDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
                ("tok_off", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("max_pages", ctypes.c_int32),
                ("max_chunk", ctypes.c_int32), ("max_kv", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("suffix_len", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("total_slots", ctypes.c_int64), ("max_src_row", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_size_t), ("rows_per_block", ctypes.c_int32),
                ("n_work_items", ctypes.c_int32), ("n_merge_groups", ctypes.c_int32),
                ("max_splits", ctypes.c_int32)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python paper_2607_17715_amd/build.py`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    P = ctypes.POINTER
    sig = {
        "c2kv_plan_create": [P(AttnCfg), P(ComposeDesc), i32, P(PlanOpts), P(vp)],
        "c2kv_plan_destroy": [vp],
        "c2kv_plan_get_info": [vp, P(PlanInfo)],
        "c2kv_plan_get_requests": [vp, vp, vp],
        "c2kv_plan_get_slots": [vp, vp, vp, vp],
        "c2kv_plan_get_block_table": [vp, vp],
        "c2kv_plan_upload": [vp, vp, sz, vp],
        "c2kv_compose": [vp, P(PoolDesc), vp, vp, vp, vp, vp, vp],
        "c2kv_attend": [vp, vp, vp, vp, vp, vp, vp, vp, vp],
        "c2kv_compose_attend": [vp, P(PoolDesc), vp, vp, vp, vp, vp, vp],
        "c2kv_compose_attend_static": [vp, P(PoolDesc), vp, vp, vp, vp, vp, vp],
        "c2kv_timing_enable": [i32],
        "c2kv_timing_reset": [],
        "c2kv_timing_read": [ctypes.c_char_p, P(ctypes.c_double), P(i64)],
        "c2kv_last_error": [],
        "c2kv_version": [],
        "c2kv_host_alloc": [sz, P(vp), P(vp)],
        "c2kv_host_free": [vp],
        "c2kv_load": [vp, P(PoolDesc), P(PoolDesc), vp],
        "c2kv_sif_plan_create": [P(AttnCfg), i32, i32, i32, i32, P(PlanOpts), P(vp)],
        "c2kv_cache_write": [P(AttnCfg), P(CacheDesc), P(ChunksDesc), vp, i64, vp, i64, vp, vp],
        "c2kv_cache_read": [P(AttnCfg), P(CacheDesc), P(ChunksDesc), vp, vp, vp, vp],
        "c2kv_cache_attend_workspace": [P(AttnCfg), P(CacheDesc), P(ChunksDesc), P(sz)],
        "c2kv_cache_attend": [P(AttnCfg), P(CacheDesc), P(ChunksDesc), vp, i64, vp, vp, vp, vp,
                              sz, vp],
        "c2kv_pool_write": [P(AttnCfg), P(PoolDesc), i32, vp, vp, i64, vp, i64, vp, vp],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = None if name == "c2kv_plan_destroy" else (
            ctypes.c_char_p if name in ("c2kv_last_error", "c2kv_version") else ctypes.c_int)
    return lib


_lib = _load()


def lib() -> ctypes.CDLL:
    return _lib


def _check(status: int):
    if status != C2KV_OK:
        raise C2KVError(status, _lib.c2kv_last_error().decode(errors="replace"))


def version() -> str:
    return _lib.c2kv_version().decode()


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data


def _dev_ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class Plan:
    """Host plan of one batch of compositions (c2kv_plan_create), shared by every layer."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, act_dtype: str,
                 rope_base: float, req_seg_off, seg_row0, seg_span, seg_orig_pos0,
                 seg_kept_off, kept_idx, suffix_len: int, seg_new_pos0=None,
                 softmax_scale: float = 0.0, page_size: int = 0, kv_splits: int = 0,
                 rows_per_block: int = 0, num_cus: int = 0, merge_mode: int = 0,
                 keys_pre_rope: bool = False, pool_compressed: bool = False):
        self._arrays = dict(
            req_seg_off=np.ascontiguousarray(req_seg_off, np.int32),
            seg_row0=np.ascontiguousarray(seg_row0, np.int64),
            seg_span=np.ascontiguousarray(seg_span, np.int32),
            seg_orig_pos0=np.ascontiguousarray(seg_orig_pos0, np.int32),
            seg_kept_off=np.ascontiguousarray(seg_kept_off, np.int32),
            kept_idx=np.ascontiguousarray(kept_idx, np.int32),
            seg_new_pos0=None if seg_new_pos0 is None else np.ascontiguousarray(seg_new_pos0, np.int32),
        )
        a = self._arrays
        self.cfg = AttnCfg(n_q_heads, n_kv_heads, head_dim, _DTYPE_CODE[act_dtype],
                           float(rope_base), float(softmax_scale))
        self.act_dtype = act_dtype
        desc = ComposeDesc(len(a["req_seg_off"]) - 1, len(a["seg_row0"]),
                           _np_ptr(a["req_seg_off"]), _np_ptr(a["seg_row0"]),
                           _np_ptr(a["seg_span"]), _np_ptr(a["seg_orig_pos0"]),
                           _np_ptr(a["seg_new_pos0"]), _np_ptr(a["seg_kept_off"]),
                           _np_ptr(a["kept_idx"]), C2KV_KEYS_PRE_ROPE if keys_pre_rope
                           else C2KV_KEYS_ROPE_AT_ORIG,
                           C2KV_POOL_COMPRESSED if pool_compressed else C2KV_POOL_FULL)
        opts = PlanOpts(page_size, kv_splits, rows_per_block, num_cus, merge_mode)
        h = ctypes.c_void_p()
        _check(_lib.c2kv_plan_create(ctypes.byref(self.cfg), ctypes.byref(desc),
                                     int(suffix_len), ctypes.byref(opts), ctypes.byref(h)))
        self._h = h
        self.suffix_len = int(suffix_len)
        self.workspace = None
        inf = PlanInfo()
        _check(_lib.c2kv_plan_get_info(self._h, ctypes.byref(inf)))
        self.info = inf.as_dict()

    @classmethod
    def sif(cls, n_q_heads: int, n_kv_heads: int, head_dim: int, act_dtype: str,
            rope_base: float, batch: int, n_tokens: int, block: int, sink: int,
            softmax_scale: float = 0.0, page_size: int = 0, kv_splits: int = 0,
            rows_per_block: int = 0, num_cus: int = 0, merge_mode: int = 0) -> "Plan":
        """Plan of extraction-time SIF attention (c2kv_sif_plan_create); run it with
        c2kv_attend(plan, None, None, q, k, v, out, lse)."""
        self = cls.__new__(cls)
        self._arrays = {}
        self.cfg = AttnCfg(n_q_heads, n_kv_heads, head_dim, _DTYPE_CODE[act_dtype],
                           float(rope_base), float(softmax_scale))
        self.act_dtype = act_dtype
        opts = PlanOpts(page_size, kv_splits, rows_per_block, num_cus, merge_mode)
        h = ctypes.c_void_p()
        _check(_lib.c2kv_sif_plan_create(ctypes.byref(self.cfg), int(batch), int(n_tokens),
                                         int(block), int(sink), ctypes.byref(opts),
                                         ctypes.byref(h)))
        self._h = h
        self.workspace = None
        inf = PlanInfo()
        _check(_lib.c2kv_plan_get_info(self._h, ctypes.byref(inf)))
        self.info = inf.as_dict()
        self.suffix_len = self.info["suffix_len"]
        return self

    @classmethod
    def for_sif(cls, w, **opts) -> "Plan":
        return cls.sif(w.n_q_heads, w.n_kv_heads, w.head_dim, w.act_dtype, w.rope_base,
                       w.batch, w.n_tokens, w.block, w.sink, **opts)

    @classmethod
    def for_workload(cls, w, **opts) -> "Plan":
        return cls(w.n_q_heads, w.n_kv_heads, w.head_dim, w.act_dtype, w.rope_base,
                   w.req_seg_off, w.seg_row0, w.seg_span, w.seg_orig_pos0, w.seg_kept_off,
                   w.kept_idx, w.suffix_len, seg_new_pos0=w.seg_new_pos0,
                   keys_pre_rope=getattr(w, "keys_pre_rope", False),
                   pool_compressed=getattr(w, "pool_compressed", False), **opts)

    def __del__(self):
        h = getattr(self, "_h", None)
        lib_ = _lib
        if h is not None and h.value and lib_ is not None:   # None at interpreter teardown
            lib_.c2kv_plan_destroy(h)
            self._h = None

    @property
    def handle(self):
        return self._h

    # ---- host copies of the layout --------------------------------------------
    def requests(self):
        B = self.info["batch"]
        n = np.zeros(B, np.int32)
        e = np.zeros(B, np.int32)
        _check(_lib.c2kv_plan_get_requests(self._h, _np_ptr(n), _np_ptr(e)))
        return n, e

    def slots(self):
        T = self.info["total_slots"]
        src = np.zeros(max(T, 1), np.int64)
        pos = np.zeros(max(T, 1), np.int32)
        dl = np.zeros(max(T, 1), np.int32)
        _check(_lib.c2kv_plan_get_slots(self._h, _np_ptr(src), _np_ptr(pos), _np_ptr(dl)))
        return src[:T], pos[:T], dl[:T]

    def block_table(self):
        bt = np.zeros((self.info["batch"], self.info["max_pages"]), np.int32)
        _check(_lib.c2kv_plan_get_block_table(self._h, _np_ptr(bt)))
        return bt

    # ---- device ---------------------------------------------------------------
    def upload(self, workspace=None, stream=None):
        """Bind the plan to a device workspace (allocated here if not given)."""
        import torch
        nbytes = int(self.info["workspace_bytes"])
        if workspace is None:
            workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
            off = (-workspace.data_ptr()) % 256
            workspace = workspace[off:off + nbytes]
        _check(_lib.c2kv_plan_upload(self._h, ctypes.c_void_p(workspace.data_ptr()),
                                     workspace.numel(), _stream(stream)))
        self.workspace = workspace
        return self


def _check_scales(code: int, shape, float32, *scales):
    """Scales of a pool of rows `shape`, tensors or arrays.  (Of other than int8 pools the library
    reads none.)"""
    for s in scales:
        if code == C2KV_I8 and s is not None and (s.dtype != float32 or
                                                  tuple(s.shape) != tuple(shape[:2])):
            raise ValueError(f"pool scales must be float32 {list(shape[:2])}, got {s.dtype} "
                             f"{list(s.shape)}")


def pool_desc(k, v, k_scale=None, v_scale=None) -> PoolDesc:
    """A pool of rows k and v [n_rows][H_kv][D], for int8 with float32 scales [n_rows][H_kv],
    all on one device.  The descriptor keeps the tensors that it points to."""
    import torch
    code = {torch.float32: C2KV_F32, torch.bfloat16: C2KV_BF16, torch.int8: C2KV_I8}[k.dtype]
    if v.dtype != k.dtype or v.shape != k.shape:
        raise ValueError("pool K and V must have the same dtype and shape")
    tensors = (k, v, k_scale, v_scale)
    _check_scales(code, k.shape, torch.float32, k_scale, v_scale)
    _one_device(*tensors)
    desc = PoolDesc(code, *(_dev_ptr(t) for t in tensors), int(k.shape[0]))
    desc.tensors, desc.row_shape, desc.dev = tensors, tuple(k.shape[1:]), k.get_device()
    return desc


def page_shapes(plan: Plan):
    """Shapes of k_pages and v_pages (v_pages holds each page transposed)."""
    i, c = plan.info, plan.cfg
    return ((i["n_pages"], c.n_kv_heads, i["page_size"], c.head_dim),
            (i["n_pages"], c.n_kv_heads, c.head_dim, i["page_size"]))


def c2kv_compose(plan: Plan, pool: PoolDesc, k_pages, v_pages, slot_src_row=None,
                 slot_pos=None, block_table=None, stream=None):
    _check(_lib.c2kv_compose(plan.handle, ctypes.byref(pool), _dev_ptr(k_pages),
                             _dev_ptr(v_pages), _dev_ptr(slot_src_row), _dev_ptr(slot_pos),
                             _dev_ptr(block_table), _stream(stream)))


def c2kv_attend(plan: Plan, k_pages, v_pages, q, k_suf, v_suf, out, lse=None, stream=None):
    _check(_lib.c2kv_attend(plan.handle, _dev_ptr(k_pages), _dev_ptr(v_pages), _dev_ptr(q),
                            _dev_ptr(k_suf), _dev_ptr(v_suf), _dev_ptr(out), _dev_ptr(lse),
                            _stream(stream)))


def c2kv_compose_attend(plan: Plan, pool: PoolDesc, q, k_suf, v_suf, out, lse=None,
                        stream=None):
    _check(_lib.c2kv_compose_attend(plan.handle, ctypes.byref(pool), _dev_ptr(q),
                                    _dev_ptr(k_suf), _dev_ptr(v_suf), _dev_ptr(out),
                                    _dev_ptr(lse), _stream(stream)))


def c2kv_compose_attend_static(plan: Plan, pool: PoolDesc, q, k_suf, v_suf, out, lse=None,
                               stream=None):
    """c2kv_compose_attend with the tables and partials in the library's static
    device array (no workspace, no upload needed)."""
    _check(_lib.c2kv_compose_attend_static(plan.handle, ctypes.byref(pool), _dev_ptr(q),
                                           _dev_ptr(k_suf), _dev_ptr(v_suf), _dev_ptr(out),
                                           _dev_ptr(lse), _stream(stream)))


def c2kv_load(plan: Plan, src: PoolDesc, dst: PoolDesc, stream=None):
    _check(_lib.c2kv_load(plan.handle, ctypes.byref(src), ctypes.byref(dst), _stream(stream)))


# ---- the growing cache ---------------------------------------------------------

def attn_cfg(n_q_heads: int, n_kv_heads: int, head_dim: int, act_dtype: str, rope_base: float,
             softmax_scale: float = 0.0) -> AttnCfg:
    """Attention shape of the cache calls and c2kv_pool_write (a plan makes its own)."""
    return AttnCfg(n_q_heads, n_kv_heads, head_dim, _DTYPE_CODE[act_dtype], float(rope_base),
                   float(softmax_scale))


class Cache:
    """A paged cache of one layer (c2kv_cache): k [n_pages][H_kv][page_size][D],
    v [n_pages][H_kv][D][page_size], for int8 with scales [n_pages][H_kv][page_size]."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        import torch
        code = {torch.float32: C2KV_F32, torch.bfloat16: C2KV_BF16, torch.int8: C2KV_I8}[k.dtype]
        n_pages, heads, page, d = k.shape
        if v.dtype != k.dtype or tuple(v.shape) != (n_pages, heads, d, page):
            raise ValueError("v must have k's dtype and each page transposed")
        for s in (k_scale, v_scale):
            if s is not None and (s.dtype != torch.float32 or
                                  tuple(s.shape) != (n_pages, heads, page)):
                raise ValueError("scales must be float32 [n_pages][H_kv][page_size]")
        self.tensors = (k, v, k_scale, v_scale)
        self.device = _one_device(*self.tensors)
        self.dev, self.heads, self.head_dim = self.device.index, heads, d
        self.desc = CacheDesc(code, *(_dev_ptr(t) for t in self.tensors), n_pages, page)
        self.ref = ctypes.byref(self.desc)


class Chunks:
    """The chunk of each request of a batch (c2kv_chunks): tok_off [B+1], kv_len [B] and
    block_table [B][max_pages], int32 on the device, read when the kernels run; n_tokens
    rows in the tensors of a call; max_chunk and max_kv bound the lengths (0: unknown) and choose
    kernels, and so the rounding of an attention's queries, but not what is answered."""

    def __init__(self, tok_off, kv_len, block_table, n_tokens: int, max_chunk: int = 0,
                 max_kv: int = 0):
        import torch
        batch, max_pages = block_table.shape
        if any(t.dtype != torch.int32 for t in (tok_off, kv_len, block_table)):
            raise ValueError("tok_off, kv_len and block_table must be int32")
        if tuple(tok_off.shape) != (batch + 1,) or tuple(kv_len.shape) != (batch,):
            raise ValueError("tok_off must have B + 1 entries and kv_len B")
        self.tensors = (tok_off, kv_len, block_table)
        self.device = _one_device(*self.tensors)
        self.dev, self.n_tokens = self.device.index, int(n_tokens)
        self.desc = ChunksDesc(batch, self.n_tokens, *(_dev_ptr(t) for t in self.tensors),
                               max_pages, int(max_chunk), int(max_kv))
        self.ref = ctypes.byref(self.desc)


def _one_device(*tensors):
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1:
        raise ValueError(f"tensors on different devices: {sorted(map(str, devices))}")
    return devices.pop()


# A call of a decode step is a few microseconds of GPU work, so the checks below look at each
# tensor once and take the stream as a number (torch's Stream object costs 2.6 us a call).
_T = None


def _torch():
    global _T
    if _T is None:
        import torch
        _T = torch
    return _T


def _run(fn, dev: int, stream, *args):
    """fn(*args, stream) with `dev`, the device that the tensors are on, as the current one:
    its stream and kernels are of that device, whatever the program's current device is."""
    t = _torch()
    if t._C._cuda_getDevice() != dev:
        with t.cuda.device(dev):
            return _run(fn, dev, stream, *args)
    if stream is None:
        s = t._C._cuda_getCurrentRawStream(dev)
    elif stream.device_index != dev:
        raise ValueError(f"a stream of device {stream.device_index}, tensors on {dev}")
    else:
        s = stream.cuda_stream
    status = fn(*args, s)
    if status != C2KV_OK:
        _check(status)


def _act(cfg: AttnCfg):
    return _torch().float32 if cfg.act_dtype == C2KV_F32 else _torch().bfloat16


def _rows(t, cfg: AttnCfg, heads: int, n: int, dev: int, what: str):
    """Pointer and token stride of rows [n][heads][D]: tokens may lie apart, a token is dense."""
    shape, d = t.shape, cfg.head_dim
    if len(shape) != 3 or shape[0] < n or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{what} must be [{n}][{heads}][{d}], got {list(shape)}")
    if t.dtype is not _act(cfg) or t.get_device() != dev:
        raise ValueError(f"{what} must have the act dtype and lie on device {dev}, "
                         f"got {t.dtype} on {t.device}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != d and heads > 1):
        raise ValueError(f"the heads of {what} must be dense")
    if shape[0] > 1 and s0 < heads * d:        # (the library takes a stride of 0 as dense)
        raise ValueError(f"the tokens of {what} overlap (stride {s0})")
    return t.data_ptr(), s0 if shape[0] > 1 else 0


def _dense(t, cfg: AttnCfg, heads: int, n: int, dev: int, what: str):
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return _rows(t, cfg, heads, n, dev, what)[0]


def _index(t, dtype, n: int, dev: int, what: str):
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] < n or t.get_device() != dev \
            or not t.is_contiguous():
        raise ValueError(f"{what} must be {dtype} [{n}], contiguous, on device {dev}")
    return t.data_ptr()


def _of(cfg: AttnCfg, cache: Cache, chunks: Chunks):
    if cache.heads != cfg.n_kv_heads or cache.head_dim != cfg.head_dim:
        raise ValueError(f"the cache has {cache.heads} heads of {cache.head_dim}, the shape "
                         f"{cfg.n_kv_heads} of {cfg.head_dim}")
    if cache.dev != chunks.dev:
        raise ValueError(f"cache on {cache.device}, chunks on {chunks.device}")
    return cache.dev, chunks.n_tokens


def c2kv_cache_write(cfg: AttnCfg, cache: Cache, chunks: Chunks, k, v, pos=None, stream=None):
    """Put the chunks' tokens into the cache; pos [n_tokens] int32: k is turned to these
    positions (None: written as it is)."""
    dev, n = _of(cfg, cache, chunks)
    kp, ks = _rows(k, cfg, cfg.n_kv_heads, n, dev, "k")
    vp, vs = _rows(v, cfg, cfg.n_kv_heads, n, dev, "v")
    pos = _index(pos, _T.int32, n, dev, "pos")
    _run(_lib.c2kv_cache_write, dev, stream, ctypes.byref(cfg), cache.ref, chunks.ref, kp, ks, vp,
         vs, pos)


def c2kv_cache_read(cfg: AttnCfg, cache: Cache, chunks: Chunks, k, v, turn=None, stream=None):
    """The chunks' tokens as rows k and v [n_tokens][H_kv][D]; turn [n_tokens] int32 turns
    key i by turn[i] positions."""
    dev, n = _of(cfg, cache, chunks)
    kp = _dense(k, cfg, cfg.n_kv_heads, n, dev, "k")
    vp = _dense(v, cfg, cfg.n_kv_heads, n, dev, "v")
    turn = _index(turn, _T.int32, n, dev, "turn")
    _run(_lib.c2kv_cache_read, dev, stream, ctypes.byref(cfg), cache.ref, chunks.ref, turn, kp, vp)


def cache_attend_workspace(cfg: AttnCfg, cache: Cache, chunks: Chunks):
    """A workspace for c2kv_cache_attend calls of this shape that are ordered."""
    nbytes = ctypes.c_size_t()
    _check(_lib.c2kv_cache_attend_workspace(ctypes.byref(cfg), cache.ref, chunks.ref,
                                            ctypes.byref(nbytes)))
    raw = _torch().empty(nbytes.value + 256, dtype=_T.uint8, device=cache.device)
    off = (-raw.data_ptr()) % 256
    return raw[off:off + nbytes.value]


def c2kv_cache_attend(cfg: AttnCfg, cache: Cache, chunks: Chunks, q, out, pos=None, lse=None,
                      workspace=None, stream=None):
    """Causal attention of the chunks' queries over their requests' caches; pos [n_tokens]
    int32 turns q (None: as it is); lse [n_tokens][H_q] float32; workspace: from
    cache_attend_workspace (allocated for the call, on the current stream, if not given)."""
    dev, n = _of(cfg, cache, chunks)
    qp, qs = _rows(q, cfg, cfg.n_q_heads, n, dev, "q")
    op = _dense(out, cfg, cfg.n_q_heads, n, dev, "out")
    pos = _index(pos, _T.int32, n, dev, "pos")
    if lse is not None:
        if lse.dtype is not _T.float32 or lse.get_device() != dev or lse.dim() != 2 or \
                lse.shape[0] < n or lse.shape[1] != cfg.n_q_heads or not lse.is_contiguous():
            raise ValueError(f"lse must be float32 [{n}][{cfg.n_q_heads}], contiguous, on "
                             f"device {dev}")
        lse = lse.data_ptr()
    if workspace is None:
        if stream is not None:
            raise ValueError("a call on another stream needs a workspace of its own")
        workspace = cache_attend_workspace(cfg, cache, chunks)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and lie on device {dev}")
    _run(_lib.c2kv_cache_attend, dev, stream, ctypes.byref(cfg), cache.ref, chunks.ref, qp, qs,
         pos, op, lse, workspace.data_ptr(), workspace.nbytes)


def c2kv_pool_write(cfg: AttnCfg, pool: PoolDesc, row, k, v, pos=None, stream=None):
    """Store the rows k and v [n][H_kv][D] in pool rows row [n] int64, quantised as they are
    written where the pool is int8; pos [n] int32 encodes k at these positions."""
    n, dev = row.shape[0], row.get_device()
    if dev < 0:
        raise ValueError("expected a device tensor")
    rows = _index(row, _torch().int64, n, dev, "row")
    if getattr(pool, "row_shape", None) not in (None, (cfg.n_kv_heads, cfg.head_dim)):
        raise ValueError(f"the pool's rows are {pool.row_shape}, the shape has "
                         f"{(cfg.n_kv_heads, cfg.head_dim)}")
    if getattr(pool, "dev", dev) != dev:
        raise ValueError(f"pool on device {pool.dev}, rows on {dev}")
    kp, ks = _rows(k, cfg, cfg.n_kv_heads, n, dev, "k")
    vp, vs = _rows(v, cfg, cfg.n_kv_heads, n, dev, "v")
    pos = _index(pos, _T.int32, n, dev, "pos")
    _run(_lib.c2kv_pool_write, dev, stream, ctypes.byref(cfg), ctypes.byref(pool), n, rows, kp, ks,
         vp, vs, pos)


class HostPool:
    """A pool in page-locked host memory from c2kv_host_alloc, filled from numpy
    storage arrays (bf16 as uint16 bit patterns).  `desc` points kernels at it
    for reads in place over the host link; it is also a c2kv_load source."""

    def __init__(self, pool_k: np.ndarray, pool_v: np.ndarray, dtype: str,
                 k_scale: Optional[np.ndarray] = None, v_scale: Optional[np.ndarray] = None):
        self._host = []
        code = {"f32": C2KV_F32, "bf16": C2KV_BF16, "i8": C2KV_I8}[dtype]
        if pool_k.shape != pool_v.shape:
            raise ValueError("pool K and V must have the same shape")
        size = {"f32": 4, "bf16": 2, "i8": 1}[dtype]
        if pool_k.itemsize != size or pool_v.itemsize != size:
            raise ValueError(f"{dtype} storage has {size} bytes an element")
        _check_scales(code, pool_k.shape, np.float32, k_scale, v_scale)
        self.nbytes = 0
        ptrs = [self._put(a) for a in (pool_k, pool_v, k_scale, v_scale)]
        self.desc = PoolDesc(code, ptrs[0], ptrs[1], ptrs[2], ptrs[3], int(pool_k.shape[0]))
        self.desc.row_shape = tuple(pool_k.shape[1:])

    def _put(self, a: Optional[np.ndarray]):
        if a is None:
            return None
        a = np.ascontiguousarray(a)
        host, dev = ctypes.c_void_p(), ctypes.c_void_p()
        _check(_lib.c2kv_host_alloc(max(a.nbytes, 1), ctypes.byref(host), ctypes.byref(dev)))
        self._host.append(host)
        ctypes.memmove(host, a.ctypes.data, a.nbytes)
        self.nbytes += a.nbytes
        return dev.value

    def close(self):
        lib_ = _lib
        while self._host and lib_ is not None:
            lib_.c2kv_host_free(self._host.pop())

    def __del__(self):
        self.close()


def timing_enable(on: bool = True):
    _check(_lib.c2kv_timing_enable(1 if on else 0))


def timing_reset():
    _check(_lib.c2kv_timing_reset())


def timing_read(name: str):
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check(_lib.c2kv_timing_read(name.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


# ---- tensor helpers (host <-> device marshalling) ------------------------------

def to_device(a: np.ndarray, dtype: str):
    """numpy storage array -> device tensor ('bf16' arrays are uint16 bit patterns)."""
    import torch
    if dtype == "bf16":
        t = torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16)
    elif dtype == "f32":
        t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    elif dtype == "i8":
        t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.int8))
    else:
        raise ValueError(dtype)
    return t.to("cuda")


def to_numpy_f64(t) -> np.ndarray:
    import torch
    return t.detach().to(torch.float64).cpu().numpy()
