"""ParisKV decode-step KV retrieval for AMD MI355X (gfx950).

Python binding of ``libpariskv.so`` (declared in ``include/pariskv.h``).  It
only marshals arguments: torch tensors provide device memory and streams,
every step of the path runs in the library's HIP kernels, and a missing
library raises instead of falling back to anything.

Method: ParisKV (arXiv 2602.07721), Alg. 1 -- encode keys into centroid ids,
4-bit codes and weights; per decode step rank clusters, score collisions,
select top-beta candidates, rerank them with the RSQ-IP estimator, keep the
top-k; then attend over the fetched K/V rows only.
"""

import ctypes
import os
from dataclasses import dataclass

import numpy as np

__all__ = [
    "PariskvError", "Config", "Budget", "Index", "Window", "lib", "encode", "append", "append_rows",
    "retrieve", "retrieve_workspace_size", "workspace_layout", "sparse_attend", "retrieve_attend",
    "retrieve_attend_noalloc", "NOALLOC_SCRATCH_BYTES",
    "window_regions", "window_attend", "retrieve_window_attend", "tiered_attend", "retrieve_tiered_attend",
    "offload_rows", "window_slot", "group_attend", "QuantCache", "quantize_rows", "dequantize_rows",
    "quant_attend", "quant_tiered_attend", "tree_attend", "quant_tree_attend", "tree_workspace_size",
    "sink_window_attend", "sink_window_workspace_size", "MAX_TREE",
    "PagedCache", "PagePlan", "plan_pages", "rotate_rows", "paged_attend", "paged_workspace_size", "quantizer_table", "rotation_signs",
    "profile_enable", "profile_reset", "profile_read", "stream_copy", "stream_read",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpariskv.so")
# pariskv_abi_version() of the library this binding marshals for (struct layouts, entry points)
ABI_VERSION = 4

OK, ERR_INVALID, ERR_CAPACITY, ERR_WORKSPACE, ERR_HIP, ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
HEAD_DIM, SUBSPACES, CENTROIDS, REC_BYTES = 128, 16, 256, 128
MAX_ATTEND_ROWS = 4096
MAX_TREE = 64
# Ablation variants (Sec. "Ablation Studies"): Config.flags, Budget.flags.
NO_ROTATION, NO_ALPHA_CORRECTION = 1, 2
BINARY_COLLISIONS = 1
# Diagnostic Budget.flags bit: every selection threshold from the exact recount.
EXACT_RECOUNT = 2
# Budget.flags bit for retrieve_attend: GQA-group de-duplication of the K/V fetch.
GROUP_FETCH = 4


class PariskvError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"pariskv error {code}: {message}")
        self.code = code


class _Config(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("n_subspaces", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("q_per_kv", ctypes.c_int32),
                ("capacity", ctypes.c_int64), ("rot_signs", ctypes.POINTER(ctypes.c_int8)),
                ("flags", ctypes.c_uint32)]


class _Index(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("rec", ctypes.c_void_p), ("counts", ctypes.c_void_p)]


class _Budget(ctypes.Structure):
    _fields_ = [("n_cand", ctypes.c_int64), ("n_collide", ctypes.c_int64), ("top_k", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class _Window(ctypes.Structure):
    _fields_ = [("sink_len", ctypes.c_int64), ("retr_begin", ctypes.c_int64),
                ("dense_begin", ctypes.c_int64), ("dense_end", ctypes.c_int64)]


class _QuantCache(ctypes.Structure):
    _fields_ = [("rec", ctypes.c_void_p), ("capacity", ctypes.c_int64), ("k_bits", ctypes.c_int32),
                ("v_bits", ctypes.c_int32), ("host_mapped", ctypes.c_int32)]


class _Pages(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32)]


class _PageStep(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_width", ctypes.c_int64), ("free_pages", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("n_free", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("batch", ctypes.c_int32), ("t", ctypes.c_int64),
                ("new_lens", ctypes.c_void_p), ("new_free", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("granted", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p)]


class _Layout(ctypes.Structure):
    _fields_ = [(name, ctypes.c_size_t) for name in
                ("total", "zq", "lut", "score8", "chunk_sfx", "chunk_base", "thresh", "cand",
                 "cand_score", "stats", "surv", "group_rows", "group_part")] + \
               [(name, ctypes.c_int64) for name in ("n_pad", "n_chunks", "chunk_keys", "c_eff")] + \
               [(name, ctypes.c_int32) for name in ("quads", "topk_parts", "group_splits")]


_lib = None
_torch_module = None


def _torch():
    """torch, imported at the first call that takes tensors."""
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def lib():
    """The loaded library; raises ImportError when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2602_07721_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, VP, I32, I64, SZ = ctypes.POINTER, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.pariskv_encode.argtypes = [P(_Config), P(_Index), VP, I64, I32, VP]
        L.pariskv_append.argtypes = [P(_Config), P(_Index), VP, I64, I64, I32, VP]
        L.pariskv_append_rows.argtypes = [P(_Config), P(_Index), VP, I64, I64, I64, I64, I32, VP]
        L.pariskv_window_regions.argtypes = [I64, I64, I64, I64, I64, P(_Window), P(I64)]
        L.pariskv_window_attend.argtypes = [P(_Config), VP, VP, VP, I32, I64, VP, I32, P(_Window), I32,
                                            ctypes.c_float, VP, VP]
        L.pariskv_retrieve_window_attend.argtypes = [P(_Config), P(_Index), VP, I64, I32, P(_Budget), VP,
                                                     VP, VP, VP, I32, I64, P(_Window), ctypes.c_float, VP,
                                                     VP, SZ, VP]
        L.pariskv_retrieve_workspace.argtypes = [P(_Config), I32, I64, P(_Budget)]
        L.pariskv_retrieve_workspace.restype = SZ
        L.pariskv_workspace_layout.argtypes = [P(_Config), I32, I64, P(_Budget), P(_Layout)]
        L.pariskv_retrieve.argtypes = [P(_Config), P(_Index), VP, I64, I32, P(_Budget), VP, VP, VP,
                                       SZ, VP]
        L.pariskv_retrieve_attend_noalloc.argtypes = [P(_Config), P(_Index), VP, I64, I32, P(_Budget), VP, VP,
                                                      VP, VP, I32, I64, ctypes.c_float, VP, VP]
        L.pariskv_sparse_attend.argtypes = [P(_Config), VP, VP, VP, I32, I64, VP, I32, I32,
                                            ctypes.c_float, VP, VP]
        L.pariskv_retrieve_attend.argtypes = [P(_Config), P(_Index), VP, I64, I32, P(_Budget), VP, VP,
                                              VP, VP, I32, I64, ctypes.c_float, VP, VP, SZ, VP]
        L.pariskv_tiered_attend.argtypes = [P(_Config), VP, VP, VP, I64, VP, VP, I32, I64, VP, I32, P(_Window),
                                            I32, ctypes.c_float, VP, VP]
        L.pariskv_retrieve_tiered_attend.argtypes = [P(_Config), P(_Index), VP, I64, I32, P(_Budget), VP, VP,
                                                     VP, VP, I64, VP, VP, I32, I64, P(_Window),
                                                     ctypes.c_float, VP, VP, SZ, VP]
        L.pariskv_group_attend.argtypes = [P(_Config), VP, VP, VP, I32, I64, VP, I32, I32, ctypes.c_float, VP,
                                           VP, VP]
        L.pariskv_offload_rows.argtypes = [VP, VP, I64, I64, VP, VP, I64, I64, I64, I32, I32, VP]
        F = ctypes.c_float
        L.pariskv_quant_record_bytes.argtypes = [I32, I32]
        L.pariskv_quant_record_bytes.restype = SZ
        L.pariskv_quantize_rows.argtypes = [P(_Config), P(_QuantCache), VP, VP, I64, I64, I64, VP, I64, I32, VP]
        L.pariskv_dequantize_rows.argtypes = [P(_Config), P(_QuantCache), I64, VP, I64, VP, VP, I64, I64, I32, VP]
        L.pariskv_quant_attend.argtypes = [P(_Config), VP, P(_QuantCache), VP, I32, I32, F, VP, VP]
        L.pariskv_quant_tiered_attend.argtypes = [P(_Config), VP, VP, VP, I64, P(_QuantCache), VP, I32, P(_Window),
                                                  I32, F, VP, VP]
        L.pariskv_tree_workspace.argtypes = [P(_Config), I32, I64, I32]
        L.pariskv_tree_workspace.restype = SZ
        L.pariskv_tree_attend.argtypes = [P(_Config), VP, VP, VP, I64, VP, VP, VP, I64, VP, I32, I32, F, VP, VP, SZ,
                                          VP]
        L.pariskv_quant_tree_attend.argtypes = [P(_Config), VP, P(_QuantCache), VP, VP, VP, I64, VP, I32, I32, F, VP,
                                                VP, SZ, VP]
        L.pariskv_sink_window_workspace.argtypes = [P(_Config), I32, I64, I64, I64, I64]
        L.pariskv_sink_window_workspace.restype = SZ
        L.pariskv_sink_window_attend.argtypes = [P(_Config), VP, VP, VP, I64, I64, VP, I64, VP, I64, I64, I32, F, VP,
                                                 VP, SZ, VP]
        L.pariskv_plan_pages.argtypes = [P(_PageStep), VP]
        L.pariskv_rotate_rows.argtypes = [P(_Config), P(_Pages), VP, I64, VP, I64, VP, I64, I64, VP, VP, VP, I32, I32, VP,
                                          VP, F, VP, VP]
        L.pariskv_paged_workspace.argtypes = [P(_Config), I32, I64, I64]
        L.pariskv_paged_workspace.restype = SZ
        L.pariskv_paged_attend.argtypes = [P(_Config), VP, I64, P(_Pages), VP, I64, VP, VP, VP, I64, I64, I32, F, F, VP,
                                           VP, VP, SZ, VP]
        L.pariskv_stream_copy.argtypes = [VP, VP, SZ, VP]
        L.pariskv_stream_read.argtypes = [VP, SZ, ctypes.c_uint32, VP, VP]
        L.pariskv_quantizer_table.argtypes = [I32, P(ctypes.c_double), P(ctypes.c_double)]
        L.pariskv_rotation_signs.argtypes = [ctypes.c_uint64, I32, P(ctypes.c_int8)]
        L.pariskv_profile_enable.argtypes = [I32]
        L.pariskv_profile_read.argtypes = [I32, P(ctypes.c_char_p), P(I64), P(ctypes.c_double)]
        L.pariskv_strerror.restype = ctypes.c_char_p
        L.pariskv_strerror.argtypes = [ctypes.c_int]
        L.pariskv_last_error.restype = ctypes.c_char_p
        L.pariskv_abi_version.restype = I32
        if L.pariskv_abi_version() != ABI_VERSION:
            raise ImportError(f"{LIB_PATH} has ABI version {L.pariskv_abi_version()}, this binding expects "
                              f"{ABI_VERSION}: rebuild the library")
        _lib = L
    return _lib


def _check(rc):
    if rc != OK:
        msg = lib().pariskv_last_error().decode()
        raise PariskvError(rc, msg or lib().pariskv_strerror(rc).decode())
    return rc


@dataclass
class Config:
    """Layer shape, rotation signs and index variant flags (see ``pariskv_config``)."""
    n_kv_heads: int
    q_per_kv: int
    capacity: int
    rot_signs: np.ndarray
    head_dim: int = HEAD_DIM
    n_subspaces: int = SUBSPACES
    flags: int = 0

    def __post_init__(self):
        self._signs = np.ascontiguousarray(np.asarray(self.rot_signs, dtype=np.int8))
        self._c = _Config(self.head_dim, self.n_subspaces, self.n_kv_heads, self.q_per_kv,
                          self.capacity, self._signs.ctypes.data_as(ctypes.POINTER(ctypes.c_int8)),
                          self.flags)

    @property
    def n_q_heads(self):
        return self.n_kv_heads * self.q_per_kv

    def c(self):
        return ctypes.byref(self._c)


@dataclass
class Budget:
    """C = n_cand, C_rho = n_collide, k = top_k, flags (see ``pariskv_budget``)."""
    n_cand: int
    n_collide: int
    top_k: int
    flags: int = 0

    def c(self):
        self._c = _Budget(self.n_cand, self.n_collide, self.top_k, self.flags)
        return ctypes.byref(self._c)


def _ptr(t, name, device=True):
    if t is None:
        return None
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if device and not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    if torch.cuda.is_initialized():
        # torch.cuda.current_stream().cuda_stream without the Stream object (3 us of a small call),
        # by names that another torch may not have.
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return torch.cuda.current_stream().cuda_stream


def _arg(t, name, dtype, shape, dev=None, optional=False):
    """Pointer of a tensor argument after checking its dtype and its shape (None entries are
    free; the sizes the library derives from shapes must be consistent).  The kernels trust
    these, so a mismatch is refused here rather than read past the end of an allocation.
    A tensor that must live on the GPU and does not is appended to the list `dev`, refused by
    _require_device once every argument of the call has passed these checks."""
    if isinstance(t, _torch().Tensor) and t.dtype == dtype and t.shape == shape:
        # The whole shape given and equal: the ordinary case, in one comparison.
        if dev is not None and not t.is_cuda:
            dev.append((t, name))
        if t.is_contiguous():
            return t.data_ptr()
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != len(shape) or any(w is not None and int(d) != int(w) for d, w in zip(t.shape, shape)):
        want = "[" + ", ".join("*" if w is None else str(w) for w in shape) + "]"
        raise ValueError(f"{name} must have shape {want}, got {list(t.shape)}")
    if dev is not None and not t.is_cuda:
        dev.append((t, name))
    return _ptr(t, name, False)


def _require_device(dev):
    for _, name in dev:
        raise ValueError(f"{name} must be a GPU tensor")


def _rows(t):
    """The third dimension of a [batch][Hkv][rows][D] tensor (None, which is any, for what is not one)."""
    return t.shape[2] if isinstance(t, _torch().Tensor) and t.dim() == 4 else None


def _kv_args(cfg, batch, K, V, kv_host_mapped, dev, names=("K", "V")):
    """Pointers of a K/V cache pair [batch][Hkv][capacity][D] float16 (pinned host memory when
    kv_host_mapped) and its capacity."""
    half = _torch().float16
    if kv_host_mapped:
        dev = None
    kp = _arg(K, names[0], half, (batch, cfg.n_kv_heads, _rows(K), HEAD_DIM), dev)
    cap = K.shape[2]
    vp = _arg(V, names[1], half, (batch, cfg.n_kv_heads, cap, HEAD_DIM), dev)
    if kv_host_mapped:
        for t, nm in ((K, names[0]), (V, names[1])):
            if t.is_cuda or not t.is_pinned():
                raise ValueError(f"{nm} must be pinned host memory when kv_host_mapped")
    return kp, vp, cap


def _q_arg(cfg, q, dev):
    torch = _torch()
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [batch][Hq][D] tensor")
    batch = q.shape[0]
    return _arg(q, "q", torch.float16, (batch, cfg.n_q_heads, HEAD_DIM), dev), batch


def _out_arg(cfg, out, batch, device, dev):
    torch = _torch()
    if out is None:
        out = torch.empty((batch, cfg.n_q_heads, HEAD_DIM), dtype=torch.float32, device=device)
    return out, _arg(out, "out", torch.float32, (batch, cfg.n_q_heads, HEAD_DIM), dev)


def _idx_arg(cfg, idx, batch, dev, name="idx"):
    torch = _torch()
    if not isinstance(idx, torch.Tensor) or idx.dim() != 3:
        raise ValueError(f"{name} must be a [batch][Hq][k] int32 tensor")
    k = int(idx.shape[-1])
    return _arg(idx, name, torch.int32, (batch, cfg.n_q_heads, k), dev), k


def _retrieve_outs(cfg, budget, batch, out_idx, out_score, workspace, n, device, dev):
    """Allocate what the caller left out and check the rest: (out_idx, out_score, workspace, ptrs)."""
    torch = _torch()
    if out_idx is None:
        out_idx = torch.empty((batch, cfg.n_q_heads, budget.top_k), dtype=torch.int32, device=device)
    if workspace is None:
        workspace = torch.empty(max(256, retrieve_workspace_size(cfg, batch, n, budget)),
                                dtype=torch.uint8, device=device)
    rows = (batch, cfg.n_q_heads, budget.top_k)
    ptrs = (_arg(out_idx, "out_idx", torch.int32, rows, dev),
            _arg(out_score, "out_score", torch.float32, rows, dev, optional=True),
            _arg(workspace, "workspace", torch.uint8,
                 workspace.shape if isinstance(workspace, torch.Tensor) and workspace.dim() == 1 else (None,), dev))
    return out_idx, out_score, workspace, ptrs


class Index:
    """Device arrays of the per-key metadata (see ``pariskv_index``)."""

    def __init__(self, ids, rec, counts):
        self.ids, self.rec, self.counts = ids, rec, counts

    @classmethod
    def empty(cls, cfg, batch, device="cuda"):
        import torch
        ids = torch.empty((batch, cfg.n_kv_heads, cfg.capacity, SUBSPACES), dtype=torch.uint8, device=device)
        rec = torch.empty((batch, cfg.n_kv_heads, cfg.capacity, REC_BYTES), dtype=torch.uint8, device=device)
        counts = torch.zeros((batch, cfg.n_kv_heads, SUBSPACES, CENTROIDS), dtype=torch.int32, device=device)
        return cls(ids, rec, counts)

    @property
    def batch(self):
        return int(self.ids.shape[0])

    def c(self, cfg=None, batch=None, dev=None):
        if cfg is not None:
            torch = _torch()
            b = self.batch if batch is None else batch
            cap = cfg.capacity
            own = dev is None
            dev = [] if own else dev
            ptrs = (_arg(self.ids, "index.ids", torch.uint8, (b, cfg.n_kv_heads, cap, SUBSPACES), dev),
                    _arg(self.rec, "index.rec", torch.uint8, (b, cfg.n_kv_heads, cap, REC_BYTES), dev),
                    _arg(self.counts, "index.counts", torch.int32, (b, cfg.n_kv_heads, SUBSPACES, CENTROIDS), dev))
            if own:
                _require_device(dev)
        else:
            ptrs = (_ptr(self.ids, "ids"), _ptr(self.rec, "rec"), _ptr(self.counts, "counts"))
        self._c = _Index(*ptrs)
        return ctypes.byref(self._c)


def _keys_arg(cfg, keys, dev, name="keys"):
    torch = _torch()
    if not isinstance(keys, torch.Tensor) or keys.dim() != 4:
        raise ValueError(f"{name} must be a [batch][Hkv][n][D] float16 tensor")
    b = keys.shape[0]
    return _arg(keys, name, torch.float16, (b, cfg.n_kv_heads, keys.shape[2], HEAD_DIM), dev), b


def encode(cfg, index, keys, stream=None):
    """Prefill: encode keys [batch][Hkv][n][D] float16 into rows [0, n); resets counts."""
    dev = []
    kp, b = _keys_arg(cfg, keys, dev)
    ic = index.c(cfg, b, dev)
    _require_device(dev)
    _check(lib().pariskv_encode(cfg.c(), ic, kp, int(keys.shape[2]), b, _stream(stream)))


def append(cfg, index, keys, n_cur, stream=None):
    """Streaming update: encode keys [batch][Hkv][t][D] into rows [n_cur, n_cur + t)."""
    dev = []
    kp, b = _keys_arg(cfg, keys, dev)
    ic = index.c(cfg, b, dev)
    _require_device(dev)
    _check(lib().pariskv_append(cfg.c(), ic, kp, int(n_cur), int(keys.shape[2]), b, _stream(stream)))


def append_rows(cfg, index, K, row_begin, t, n_cur, stream=None):
    """Streaming update from the key cache K [batch][Hkv][kv_capacity][D]: encode cache rows
    [row_begin, row_begin + t) into index rows [n_cur, n_cur + t)."""
    dev = []
    kp, b = _keys_arg(cfg, K, dev, "K")
    ic = index.c(cfg, b, dev)
    _require_device(dev)
    _check(lib().pariskv_append_rows(cfg.c(), ic, kp, int(K.shape[2]), int(row_begin), int(n_cur), int(t), b,
                                     _stream(stream)))


@dataclass
class Window:
    """Rows attended besides the retrieved keys (see ``pariskv_window``): Sink rows
    [0, sink_len), retrieved index row i at cache row retr_begin + i, Local + Update Buffer
    rows [dense_begin, dense_end)."""
    sink_len: int = 0
    retr_begin: int = 0
    dense_begin: int = 0
    dense_end: int = 0

    @property
    def dense_rows(self):
        return self.sink_len + self.dense_end - self.dense_begin

    def c(self):
        self._c = _Window(self.sink_len, self.retr_begin, self.dense_begin, self.dense_end)
        return ctypes.byref(self._c)


def window_regions(P, t, sink=128, local=512, m=256):
    """(Window, n_retrieval) after a prompt of P tokens and t decode steps, buffer updates
    every m steps (Sec. "Buffer Update"); see ``pariskv_window_regions``."""
    w = _Window()
    n = ctypes.c_int64()
    _check(lib().pariskv_window_regions(int(P), int(t), int(sink), int(local), int(m), ctypes.byref(w),
                                        ctypes.byref(n)))
    return Window(w.sink_len, w.retr_begin, w.dense_begin, w.dense_end), int(n.value)


def retrieve_workspace_size(cfg, batch, n, budget):
    return int(lib().pariskv_retrieve_workspace(cfg.c(), batch, n, budget.c()))


def workspace_layout(cfg, batch, n, budget):
    L = _Layout()
    _check(lib().pariskv_workspace_layout(cfg.c(), batch, n, budget.c(), ctypes.byref(L)))
    return {name: getattr(L, name) for name, _ in _Layout._fields_}


def retrieve(cfg, index, q, n, budget, out_idx=None, out_score=None, workspace=None, stream=None):
    """Alg. 1 decode for all query heads; returns (idx, score, workspace) tensors."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    out_idx, out_score, workspace, (ip, sp, wp) = _retrieve_outs(cfg, budget, batch, out_idx, out_score,
                                                                 workspace, n, q.device, dev)
    ic = index.c(cfg, batch, dev)
    _require_device(dev)
    _check(lib().pariskv_retrieve(cfg.c(), ic, qp, int(n), batch, budget.c(), ip, sp, wp,
                                  workspace.numel(), _stream(stream)))
    return out_idx, out_score, workspace


def retrieve_attend(cfg, index, q, n, budget, K, V, scale, out_idx=None, out_score=None, out=None,
                    workspace=None, kv_host_mapped=False, stream=None):
    """retrieve + sparse_attend in one call (the attention runs inside the final top-k kernel);
    returns (idx, score, out, workspace)."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    out_idx, out_score, workspace, (ip, sp, wp) = _retrieve_outs(cfg, budget, batch, out_idx, out_score,
                                                                 workspace, n, q.device, dev)
    ic = index.c(cfg, batch, dev)
    _require_device(dev)
    _check(lib().pariskv_retrieve_attend(cfg.c(), ic, qp, int(n), batch, budget.c(), ip, sp,
                                         kp, vp, int(bool(kv_host_mapped)), cap, float(scale), op, wp,
                                         workspace.numel(), _stream(stream)))
    return out_idx, out_score, out, workspace


NOALLOC_SCRATCH_BYTES = 64 << 20


def retrieve_attend_noalloc(cfg, index, q, n, budget, K, V, scale, out_idx, out, out_score=None,
                            kv_host_mapped=False, stream=None):
    """pariskv_retrieve_attend_noalloc: retrieve_attend with the intermediates in the library's
    static per-device scratch array (NOALLOC_SCRATCH_BYTES), for callers that cannot allocate.
    Allocates nothing, so out_idx [batch][Hq][k] int32 and out [batch][Hq][D] float32 must be
    given.  Calls that overlap on one device race on the shared array."""
    torch = _torch()
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    rows = (batch, cfg.n_q_heads, budget.top_k)
    ip = _arg(out_idx, "out_idx", torch.int32, rows, dev)
    sp = _arg(out_score, "out_score", torch.float32, rows, dev, optional=True)
    op = _arg(out, "out", torch.float32, (batch, cfg.n_q_heads, HEAD_DIM), dev)
    ic = index.c(cfg, batch, dev)
    _require_device(dev)
    _check(lib().pariskv_retrieve_attend_noalloc(cfg.c(), ic, qp, int(n), batch, budget.c(), ip, sp,
                                                 kp, vp, int(bool(kv_host_mapped)), cap, float(scale), op,
                                                 _stream(stream)))
    return out_idx, out_score, out


def sparse_attend(cfg, q, K, V, idx, scale, out=None, kv_host_mapped=False, stream=None):
    """Attention over idx only; K, V [batch][Hkv][kv_capacity][D] float16 (device or pinned host)."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    _require_device(dev)
    _check(lib().pariskv_sparse_attend(cfg.c(), qp, kp, vp, int(bool(kv_host_mapped)), cap, xp, k, batch,
                                       float(scale), op, _stream(stream)))
    return out


def window_attend(cfg, q, K, V, idx, win, scale, out=None, kv_host_mapped=False, stream=None):
    """Attention over Sink + retrieved (retr_begin + idx) + Local/Buffer rows of ``win``."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    _require_device(dev)
    _check(lib().pariskv_window_attend(cfg.c(), qp, kp, vp, int(bool(kv_host_mapped)), cap, xp, k, win.c(),
                                       batch, float(scale), op, _stream(stream)))
    return out


def retrieve_window_attend(cfg, index, q, n, budget, K, V, win, scale, out_idx=None, out_score=None,
                           out=None, workspace=None, kv_host_mapped=False, stream=None):
    """retrieve over the Retrieval region + window_attend in one call; returns
    (idx, score, out, workspace)."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    out_idx, out_score, workspace, (ip, sp, wp) = _retrieve_outs(cfg, budget, batch, out_idx, out_score,
                                                                 workspace, n, q.device, dev)
    ic = index.c(cfg, batch, dev)
    _require_device(dev)
    _check(lib().pariskv_retrieve_window_attend(
        cfg.c(), ic, qp, int(n), batch, budget.c(), ip, sp, kp, vp, int(bool(kv_host_mapped)),
        cap, win.c(), float(scale), op, wp, workspace.numel(), _stream(stream)))
    return out_idx, out_score, out, workspace


def group_attend(cfg, q, K, V, idx, scale, out=None, union_rows=None, kv_host_mapped=False, stream=None):
    """sparse_attend with each distinct K/V row fetched once per KV head (quads of query heads
    attend over the union of their ascending lists); union_rows: optional int32 tensor
    [batch][Hkv][ceil(G/4)] that receives the number of rows fetched."""
    torch = _torch()
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    up = _arg(union_rows, "union_rows", torch.int32, (batch, cfg.n_kv_heads, (cfg.q_per_kv + 3) // 4), dev,
              optional=True)
    _require_device(dev)
    _check(lib().pariskv_group_attend(cfg.c(), qp, kp, vp, int(bool(kv_host_mapped)), cap, xp, k, batch,
                                      float(scale), op, up, _stream(stream)))
    return out


def window_slot(r, sink_len, win_capacity):
    """Slot of cache row r in a window cache (see ``pariskv_tiered_attend``)."""
    return r if r < sink_len else sink_len + (r - sink_len) % (win_capacity - sink_len)


def tiered_attend(cfg, q, K_win, V_win, K, V, idx, win, scale, out=None, kv_host_mapped=False, stream=None):
    """window_attend with Sink + Local/Buffer rows read from the GPU window cache K_win/V_win
    [batch][Hkv][win_capacity][D] and the retrieved rows from K/V (pinned host memory when
    kv_host_mapped)."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kwp, vwp, wcap = _kv_args(cfg, batch, K_win, V_win, False, dev, ("K_win", "V_win"))
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    _require_device(dev)
    _check(lib().pariskv_tiered_attend(cfg.c(), qp, kwp, vwp, wcap, kp, vp, int(bool(kv_host_mapped)), cap,
                                       xp, k, win.c(), batch, float(scale), op, _stream(stream)))
    return out


def retrieve_tiered_attend(cfg, index, q, n, budget, K_win, V_win, K, V, win, scale, out_idx=None,
                           out_score=None, out=None, workspace=None, kv_host_mapped=False, stream=None):
    """retrieve over the Retrieval region + tiered_attend in one call; returns (idx, score, out, ws)."""
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kwp, vwp, wcap = _kv_args(cfg, batch, K_win, V_win, False, dev, ("K_win", "V_win"))
    kp, vp, cap = _kv_args(cfg, batch, K, V, kv_host_mapped, dev)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    out_idx, out_score, workspace, (ip, sp, wp) = _retrieve_outs(cfg, budget, batch, out_idx, out_score,
                                                                 workspace, n, q.device, dev)
    ic = index.c(cfg, batch, dev)
    _require_device(dev)
    _check(lib().pariskv_retrieve_tiered_attend(
        cfg.c(), ic, qp, int(n), batch, budget.c(), ip, sp, kwp, vwp, wcap, kp, vp,
        int(bool(kv_host_mapped)), cap, win.c(), float(scale), op, wp, workspace.numel(), _stream(stream)))
    return out_idx, out_score, out, workspace


def offload_rows(K_src, V_src, src_row, K_dst, V_dst, dst_row, t, stream=None):
    """Copy rows [src_row, src_row + t) of every (sequence, KV head) of K_src/V_src to rows
    [dst_row, dst_row + t) of K_dst/V_dst (device or pinned host tensors [b][Hkv][cap][D])."""
    torch = _torch()
    named = ((K_src, "K_src"), (V_src, "V_src"), (K_dst, "K_dst"), (V_dst, "V_dst"))
    for x, nm in named:
        if not isinstance(x, torch.Tensor) or x.dim() != 4:
            raise ValueError(f"{nm} must be a [batch][Hkv][capacity][D] float16 tensor")
    b, hkv = int(K_src.shape[0]), int(K_src.shape[1])
    src_cap, dst_cap = int(K_src.shape[2]), int(K_dst.shape[2])
    ps = [_arg(x, nm, torch.float16, (b, hkv, c, HEAD_DIM))
          for x, nm, c in ((K_src, "K_src", src_cap), (V_src, "V_src", src_cap),
                           (K_dst, "K_dst", dst_cap), (V_dst, "V_dst", dst_cap))]
    for x, nm in named:
        if not x.is_cuda and not x.is_pinned():
            raise ValueError(f"{nm} must be device or pinned host memory")
    _check(lib().pariskv_offload_rows(ps[0], ps[1], src_cap, int(src_row), ps[2], ps[3], dst_cap, int(dst_row),
                                      int(t), b, hkv, _stream(stream)))


# ---- quantised K/V cache, several new tokens at a time


def _require_here(stream, *tensors):
    """The library launches on the current device: every GPU tensor and the stream must be there."""
    here = _torch().cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here and t.is_cuda:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{here}")
    if stream is not None and stream.device.index != here:
        raise ValueError(f"stream on {stream.device}, but the current device is cuda:{here}")


def _new(shape, dtype, device, stream):
    """A tensor the call writes on `stream`, owned by that stream: its memory is not reused before the work there."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class QuantCache:
    """K/V rows in 8- or 4-bit codes (see ``pariskv_quant_cache``): rec uint8 [batch][Hkv][capacity][record bytes]
    on the GPU, or in pinned host memory with host_mapped."""

    def __init__(self, rec, k_bits=8, v_bits=8, host_mapped=False):
        self.rec, self.host_mapped = rec, bool(host_mapped)
        self.k_bits, self.v_bits = int(k_bits), int(v_bits)
        self._bytes = self.record_bytes(k_bits, v_bits)

    @staticmethod
    def record_bytes(k_bits, v_bits):
        n = int(lib().pariskv_quant_record_bytes(int(k_bits), int(v_bits)))
        if n == 0:
            raise ValueError(f"k_bits and v_bits must each be 8 or 4, got {k_bits} and {v_bits}")
        return n

    @classmethod
    def empty(cls, cfg, batch, capacity, k_bits=8, v_bits=8, device="cuda", host_mapped=False):
        torch = _torch()
        shape = (batch, cfg.n_kv_heads, capacity, cls.record_bytes(k_bits, v_bits))
        rec = (torch.empty(shape, dtype=torch.uint8, pin_memory=True) if host_mapped else
               torch.empty(shape, dtype=torch.uint8, device=device))
        return cls(rec, k_bits, v_bits, host_mapped)

    @property
    def capacity(self):
        return int(self.rec.shape[2])

    def c(self, cfg, batch, dev):
        rec, host = self.rec, self.host_mapped
        ptr = _arg(rec, "cache.rec", _torch().uint8, (batch, cfg.n_kv_heads, _rows(rec), self._bytes),
                   None if host else dev)
        if host and (rec.is_cuda or not rec.is_pinned()):
            raise ValueError("cache.rec must be pinned host memory when host_mapped")
        self._c = _QuantCache(ptr, rec.shape[2], self.k_bits, self.v_bits, host)
        return ctypes.byref(self._c)


def _cache_arg(cfg, cache, batch, dev):
    if not isinstance(cache, QuantCache):
        raise TypeError("cache must be a QuantCache")
    return cache.c(cfg, batch, dev)


def _row_arg(row, batch, dev):
    """(row, pointer or None, tensor or None) of a first row: a number, or an int32 GPU tensor [batch]."""
    torch = _torch()
    if isinstance(row, torch.Tensor):
        return 0, _arg(row, "row", torch.int32, (batch,), dev), row
    return int(row), None, None


def _quant_rows(cfg, cache, K, V, row, dev):
    half = _torch().float16
    if not isinstance(K, _torch().Tensor) or K.dim() != 4:
        raise ValueError("K must be a [batch][Hkv][capacity][D] float16 tensor")
    batch = int(K.shape[0])
    kp = _arg(K, "K", half, (batch, cfg.n_kv_heads, K.shape[2], HEAD_DIM), dev)
    vp = _arg(V, "V", half, (batch, cfg.n_kv_heads, K.shape[2], HEAD_DIM), dev)
    cp = _cache_arg(cfg, cache, batch, dev)
    return batch, kp, vp, cp, _row_arg(row, batch, dev)


def quantize_rows(cfg, cache, K, V, src_row, row, t, stream=None):
    """Write rows [src_row, src_row + t) of K, V [batch][Hkv][capacity][D] float16 into the quantised cache from row
    `row` on: a number, or an int32 GPU tensor [batch] with each sequence's (rows outside the cache are skipped)."""
    dev = []
    batch, kp, vp, cp, (r, rp, rt) = _quant_rows(cfg, cache, K, V, row, dev)
    _require_device(dev)
    _require_here(stream, K, V, cache.rec, rt)
    _check(lib().pariskv_quantize_rows(cfg.c(), cp, kp, vp, int(K.shape[2]), int(src_row), r, rp, int(t), batch,
                                       _stream(stream)))


def dequantize_rows(cfg, cache, row, t, K, V, dst_row=0, stream=None):
    """The float16 values of t cache rows from `row` on (as in quantize_rows) into rows [dst_row, dst_row + t) of K, V
    [batch][Hkv][capacity][D]."""
    dev = []
    batch, kp, vp, cp, (r, rp, rt) = _quant_rows(cfg, cache, K, V, row, dev)
    _require_device(dev)
    _require_here(stream, K, V, cache.rec, rt)
    _check(lib().pariskv_dequantize_rows(cfg.c(), cp, r, rp, int(t), kp, vp, int(K.shape[2]), int(dst_row), batch,
                                         _stream(stream)))


def quant_attend(cfg, q, cache, idx, scale, out=None, stream=None):
    """sparse_attend over the rows idx of a quantised cache; returns out [batch][Hq][D] float32."""
    torch = _torch()
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    cp = _cache_arg(cfg, cache, batch, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    if out is None:
        out = _new((batch, cfg.n_q_heads, HEAD_DIM), torch.float32, q.device, stream)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    _require_device(dev)
    _require_here(stream, q, cache.rec, idx, out)
    _check(lib().pariskv_quant_attend(cfg.c(), qp, cp, xp, k, batch, float(scale), op, _stream(stream)))
    return out


def quant_tiered_attend(cfg, q, K_win, V_win, cache, idx, win, scale, out=None, stream=None):
    """tiered_attend with the retrieved rows in a quantised cache."""
    torch = _torch()
    dev = []
    qp, batch = _q_arg(cfg, q, dev)
    kwp, vwp, wcap = _kv_args(cfg, batch, K_win, V_win, False, dev, ("K_win", "V_win"))
    cp = _cache_arg(cfg, cache, batch, dev)
    xp, k = _idx_arg(cfg, idx, batch, dev)
    if out is None:
        out = _new((batch, cfg.n_q_heads, HEAD_DIM), torch.float32, q.device, stream)
    out, op = _out_arg(cfg, out, batch, q.device, dev)
    _require_device(dev)
    _require_here(stream, q, K_win, V_win, cache.rec, idx, out)
    _check(lib().pariskv_quant_tiered_attend(cfg.c(), qp, kwp, vwp, wcap, cp, xp, k, win.c(), batch, float(scale), op,
                                             _stream(stream)))
    return out


def _tokens_arg(cfg, q, dev):
    torch = _torch()
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a [batch][Hq][t][D] tensor")
    batch, t = int(q.shape[0]), int(q.shape[2])
    return _arg(q, "q", torch.float16, (batch, cfg.n_q_heads, t, HEAD_DIM), dev), batch, t


def _tokens_out(q, dtype, out, dev, stream):
    if out is None:
        out = _new(tuple(q.shape), dtype, q.device, stream)
    return out, _arg(out, "out", dtype, tuple(q.shape), dev)


def _workspace_arg(workspace, size, q, dev, stream):
    torch = _torch()
    if workspace is None:
        workspace = _new((max(256, size),), torch.uint8, q.device, stream)
    shape = workspace.shape if isinstance(workspace, torch.Tensor) and workspace.dim() == 1 else (None,)
    return workspace, _arg(workspace, "workspace", torch.uint8, shape, dev)


def tree_workspace_size(cfg, batch, n, t):
    """Bytes of a workspace for tree_attend and quant_tree_attend with these sizes and all smaller ones (0 on invalid
    sizes)."""
    return int(lib().pariskv_tree_workspace(cfg.c(), int(batch), int(n), int(t)))


def _tree_args(cfg, q, K_tree, V_tree, n, mask, lens, out, workspace, dev, stream):
    torch = _torch()
    qp, batch, t = _tokens_arg(cfg, q, dev)
    rows = (batch, cfg.n_kv_heads, t, HEAD_DIM)
    ktp, vtp = _arg(K_tree, "K_tree", torch.float16, rows, dev), _arg(V_tree, "V_tree", torch.float16, rows, dev)
    mp = _arg(mask, "mask", torch.int64, (batch, t), dev, optional=True)
    lp = _arg(lens, "lens", torch.int32, (batch,), dev, optional=True)
    out, op = _tokens_out(q, torch.float32, out, dev, stream)
    workspace, wp = _workspace_arg(workspace, 0 if workspace is not None else tree_workspace_size(cfg, batch, n, t), q,
                                   dev, stream)
    return (qp, ktp, vtp, mp, lp, op, wp), batch, t, out, workspace


def tree_attend(cfg, q, K, V, K_tree, V_tree, n, scale, mask=None, lens=None, out=None, workspace=None, stream=None):
    """Attention of t <= 64 drafted tokens per sequence, q [batch][Hq][t][D], over the n cached rows of K, V
    [batch][Hkv][kv_capacity][D] (or lens[b] of them, int32 [batch]) and the drafts' own rows K_tree, V_tree
    [batch][Hkv][t][D]: token i attends draft j when bit j of mask[b, i] (int64 [batch][t]) is set, without a mask when
    j <= i.  Drafts reach only the tokens that attend them.  Returns out [batch][Hq][t][D] float32."""
    dev = []
    (qp, ktp, vtp, mp, lp, op, wp), batch, t, out, workspace = _tree_args(cfg, q, K_tree, V_tree, n, mask, lens, out,
                                                                          workspace, dev, stream)
    kp, vp, cap = _kv_args(cfg, batch, K, V, False, dev)
    _require_device(dev)
    _require_here(stream, q, K, V, K_tree, V_tree, mask, lens, out, workspace)
    _check(lib().pariskv_tree_attend(cfg.c(), qp, kp, vp, cap, ktp, vtp, mp, int(n), lp, t, batch, float(scale), op,
                                     wp, workspace.numel(), _stream(stream)))
    return out


def quant_tree_attend(cfg, q, cache, K_tree, V_tree, n, scale, mask=None, lens=None, out=None, workspace=None,
                      stream=None):
    """tree_attend over the rows of a quantised cache on the GPU."""
    dev = []
    (qp, ktp, vtp, mp, lp, op, wp), batch, t, out, workspace = _tree_args(cfg, q, K_tree, V_tree, n, mask, lens, out,
                                                                          workspace, dev, stream)
    cp = _cache_arg(cfg, cache, batch, dev)
    _require_device(dev)
    _require_here(stream, q, cache.rec, K_tree, V_tree, mask, lens, out, workspace)
    _check(lib().pariskv_quant_tree_attend(cfg.c(), qp, cp, ktp, vtp, mp, int(n), lp, t, batch, float(scale), op, wp,
                                           workspace.numel(), _stream(stream)))
    return out


def sink_window_workspace_size(cfg, batch, pos, t, sink, window):
    """Bytes of a workspace for sink_window_attend with these sizes and all smaller ones (0 on invalid sizes)."""
    return int(lib().pariskv_sink_window_workspace(cfg.c(), int(batch), int(pos), int(t), int(sink), int(window)))


def sink_window_attend(cfg, q, K, V, pos, sink, window, scale, starts=None, counts=None, out=None, workspace=None,
                       stream=None):
    """Attention of t new tokens per sequence, q [batch][Hq][t][D] at positions pos .. pos + t - 1, over the cache rows
    (row = position) of K, V [batch][Hkv][kv_capacity][D] that each sees: j <= p with j < sink or j > p - window.
    starts (int32 [batch], at most pos) gives each sequence's first position, counts (int32 [batch]) how many of its t
    tokens there are; rows of out behind them are left as they were.  Returns out [batch][Hq][t][D] float16."""
    torch = _torch()
    dev = []
    qp, batch, t = _tokens_arg(cfg, q, dev)
    kp, vp, cap = _kv_args(cfg, batch, K, V, False, dev)
    sp = _arg(starts, "starts", torch.int32, (batch,), dev, optional=True)
    np_ = _arg(counts, "counts", torch.int32, (batch,), dev, optional=True)
    out, op = _tokens_out(q, torch.float16, out, dev, stream)
    size = 0 if workspace is not None else sink_window_workspace_size(cfg, batch, pos, t, sink, window)
    workspace, wp = _workspace_arg(workspace, size, q, dev, stream)
    _require_device(dev)
    _require_here(stream, q, K, V, starts, counts, out, workspace)
    _check(lib().pariskv_sink_window_attend(cfg.c(), qp, kp, vp, cap, int(pos), sp, t, np_, int(sink), int(window), batch,
                                            float(scale), op, wp, workspace.numel(), _stream(stream)))
    return out


# ---- paged K/V cache


def _tensors(specs):
    """Pointers of tensor arguments (tensor, name, dtype, shape, whether it may be None), checked as _arg does, with the
    tensors' devices: for calls that a decode step makes, where a microsecond shows."""
    Tensor = _torch().Tensor
    ptrs, devices = [], set()
    for t, name, dtype, shape, optional in specs:
        if not (isinstance(t, Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous()):
            _arg(t, name, dtype, shape, optional=optional)  # raises, or there is none
            ptrs.append(None)
            continue
        devices.add(t.get_device())
        ptrs.append(t.data_ptr())
    return ptrs, devices


def _require_on(devices, specs, stream):
    """What _require_device and _require_here say of tensors on these devices."""
    if -1 in devices:
        _require_device([(t, name) for t, name, *_ in specs if t is not None and not t.is_cuda])
    here = _torch().cuda.current_device()
    if devices != {here} or stream is not None:
        _require_here(stream, *(t for t, *_ in specs))


def _fit(x, bits=32):
    """A whole number, or the nearest one that `bits` bits hold, which the library judges (ctypes would wrap it)."""
    most = 2 ** (bits - 1) - 1
    return max(-most - 1, min(int(x), most))


class PagedCache:
    """A pool of pages (see ``pariskv_pages``): K, V [n_pages][Hkv][page_size][D] float16 on the GPU."""

    def __init__(self, K, V):
        self.K, self.V = K, V

    @classmethod
    def empty(cls, cfg, n_pages, page_size, device="cuda"):
        torch = _torch()
        shape = (n_pages, cfg.n_kv_heads, page_size, HEAD_DIM)
        return cls(*(torch.empty(shape, dtype=torch.float16, device=device) for _ in range(2)))

    @property
    def n_pages(self):
        return int(self.K.shape[0])

    @property
    def page_size(self):
        return int(self.K.shape[2])


def _pages_specs(cfg, cache):
    """The specs of a cache's tensors, its pages and their size."""
    if not isinstance(cache, PagedCache):
        raise TypeError("cache must be a PagedCache")
    half, K = _torch().float16, cache.K
    if not isinstance(K, _torch().Tensor) or K.dim() != 4:
        raise ValueError("cache.K must be a [n_pages][Hkv][page_size][D] float16 tensor")
    pages, _, size, _ = K.shape
    shape = (pages, cfg.n_kv_heads, size, HEAD_DIM)
    return (K, "cache.K", half, shape, False), (cache.V, "cache.V", half, shape, False), pages, size


class PagePlan:
    """What plan_pages writes, int32 on the GPU (see ``pariskv_page_step``): lens [batch] and n_free [1] after the step,
    offsets [batch + 1] of the sequences' tokens, counts [batch] granted, slots and positions [t] of the tokens."""

    def __init__(self, lens, n_free, offsets, counts, slots, positions):
        self.lens, self.n_free, self.offsets, self.counts = lens, n_free, offsets, counts
        self.slots, self.positions = slots, positions

    @classmethod
    def empty(cls, batch, t, device="cuda", stream=None):
        return cls(*(_new((n,), _torch().int32, device, stream) for n in (batch, 1, batch + 1, batch, t, t)))


def plan_pages(table, free, n_free, lens, counts, page_size, t=None, plan=None, stream=None):
    """Pages, slots and positions of a step's new tokens: counts[b] rows more for sequence b (below 0: rows given back)
    of lens[b].  table [batch][width] and the stack free [n_pages], of which n_free [1] are free, are written in place; all
    int32 on the GPU.  t: entries of slots and positions (without a plan).  A plan's lens and n_free may be lens and n_free
    themselves, its counts counts.  Returns the plan."""
    torch = _torch()
    i32 = torch.int32
    for x, nm, dims in ((table, "table [batch][width]", 2), (free, "free [n_pages]", 1)):
        if not isinstance(x, torch.Tensor) or x.dim() != dims:
            raise ValueError(f"{nm} must be an int32 tensor")
    batch, width = table.shape
    if plan is None:
        if t is None:
            raise ValueError("t is required without a plan")
        plan = PagePlan.empty(batch, int(t), table.device, stream)
    elif not isinstance(plan, PagePlan):
        raise TypeError("plan must be a PagePlan")
    if not isinstance(plan.slots, torch.Tensor) or plan.slots.dim() != 1:
        raise ValueError("plan.slots must be a [t] int32 tensor")
    n = plan.slots.shape[0]
    if t is not None and int(t) != n:
        raise ValueError(f"t is {t}, but the plan has {n} slots")
    one, each = (1,), (batch,)
    specs = ((table, "table", i32, (batch, width), False), (free, "free", i32, free.shape, False),
             (n_free, "n_free", i32, one, False), (lens, "lens", i32, each, False), (counts, "counts", i32, each, False),
             (plan.lens, "plan.lens", i32, each, False), (plan.n_free, "plan.n_free", i32, one, False),
             (plan.offsets, "plan.offsets", i32, (batch + 1,), False), (plan.counts, "plan.counts", i32, each, False),
             (plan.slots, "plan.slots", i32, (n,), False), (plan.positions, "plan.positions", i32, (n,), False))
    (tp, fp, np_, lp, cp, *outs), devices = _tensors(specs)
    _require_on(devices, specs, stream)
    step = _PageStep(tp, width, fp, free.shape[0], _fit(page_size), np_, lp, cp, _fit(batch), n, *outs)
    _check(lib().pariskv_plan_pages(ctypes.byref(step), _stream(stream)))
    return plan


def _token_rows(x, name, heads, t=None):
    """(pointer, values from one token to the next) of [t][heads][D] float16, a token's heads next to each other: a
    contiguous tensor or columns of a wider one."""
    torch = _torch()
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError(f"{name} must be a [t][heads][D] float16 tensor")
    if x.dtype is not torch.float16:
        raise TypeError(f"{name} must be {torch.float16}, got {x.dtype}")
    if t is None:
        t = x.shape[0]
    if x.shape != (t, heads, HEAD_DIM):
        raise ValueError(f"{name} must have shape [{t}, {heads}, {HEAD_DIM}], got {list(x.shape)}")
    step, head, dim = x.stride()
    if t > 0 and (dim != 1 or (heads > 1 and head != HEAD_DIM)):
        raise ValueError(f"{name} must have its heads next to each other")
    if t < 2:
        step = heads * HEAD_DIM
    ptr = x.data_ptr()
    if step < heads * HEAD_DIM or step % 8 or ptr % 16:
        raise ValueError(f"{name} must have its tokens a multiple of 8 values apart, at 16-byte addresses")
    return ptr, step


def rotate_rows(cfg, cache, q, k, v, positions, slots, freqs=None, q_weight=None, k_weight=None, eps=1e-6, pairs=False,
                q_out=None, stream=None):
    """Queries q [t][Hq][D] and keys k [t][Hkv][D] normalised (with a weight [D] float32) and rotated by positions times
    freqs (float32 [rot_dim / 2] radians; halves of the first rot_dim dims against each other, with pairs neighbours), keys
    and values v [t][Hkv][D] written to the slots of a PagedCache.  positions, slots int32 [t]; tokens whose slot lies outside
    the pages are left alone.  q, k and v may be columns of one tensor.  Returns q_out [t][Hq][D] float16."""
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    K, V, n_pages, size = _pages_specs(cfg, cache)
    qp, qs = _token_rows(q, "q", cfg.n_q_heads)
    t = q.shape[0]
    kp, ks = _token_rows(k, "k", cfg.n_kv_heads, t)
    vp, vs = _token_rows(v, "v", cfg.n_kv_heads, t)
    if freqs is not None and (not isinstance(freqs, torch.Tensor) or freqs.dim() != 1):
        raise ValueError("freqs must be a [rot_dim / 2] float32 tensor")
    half = 0 if freqs is None else freqs.shape[0]
    if q_out is None:
        q_out = _new((t, cfg.n_q_heads, HEAD_DIM), torch.float16, q.device, stream)
    specs = (K, V, (positions, "positions", i32, (t,), False), (slots, "slots", i32, (t,), False),
             (freqs, "freqs", f32, (half,), True), (q_weight, "q_weight", f32, (HEAD_DIM,), True),
             (k_weight, "k_weight", f32, (HEAD_DIM,), True),
             (q_out, "q_out", torch.float16, (t, cfg.n_q_heads, HEAD_DIM), False))
    (Kp, Vp, pp, sp, fp, qw, kw, op), devices = _tensors(specs)
    devices.update((q.get_device(), k.get_device(), v.get_device()))
    _require_on(devices, ((q, "q"), (k, "k"), (v, "v")) + specs, stream)
    _check(lib().pariskv_rotate_rows(cfg.c(), ctypes.byref(_Pages(Kp, Vp, n_pages, size)), qp, qs, kp, ks, vp, vs, t, pp, sp,
                                     fp, _fit(2 * half), bool(pairs), qw, kw, eps, op, _stream(stream)))
    return q_out


def paged_workspace_size(cfg, batch, t, max_tokens=None):
    """Bytes of a workspace for paged_attend with these sizes and all smaller ones (0 on invalid sizes)."""
    most = max(1, int(t)) if max_tokens is None else max_tokens
    return int(lib().pariskv_paged_workspace(cfg.c(), _fit(batch), _fit(t, 64), _fit(most, 64)))


def paged_attend(cfg, q, cache, table, lens, offsets, scale, counts=None, max_tokens=None, softcap=0.0, slopes=None,
                 out=None, workspace=None, stream=None):
    """Attention of the new tokens of a batch, q [t][Hq][D] with sequence b's at offsets[b] .. offsets[b + 1] (or the first
    counts[b] of them), over the pages that table [batch][width] names: the token at position p sees the rows up to p, the
    last one stands at lens[b] - 1; table, lens, offsets, counts int32.  max_tokens: the most tokens of a sequence (t without;
    1 for a decode step).  softcap c > 0 makes a score s c tanh(s / c), slopes (float32 [Hq]) take slope times the distance
    off it.  Returns out [t][Hq][D] float16; rows of tokens that no sequence has are left as they were."""
    torch = _torch()
    i32, half = torch.int32, torch.float16
    K, V, n_pages, size = _pages_specs(cfg, cache)
    qp, qs = _token_rows(q, "q", cfg.n_q_heads)
    t = q.shape[0]
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table must be a [batch][width] int32 tensor")
    batch, width = table.shape
    most = max(1, t) if max_tokens is None else _fit(max_tokens, 64)
    if out is None:
        out = _new(q.shape, half, q.device, stream)
    if workspace is None:
        workspace = _new((max(256, paged_workspace_size(cfg, batch, t, most)),), torch.uint8, q.device, stream)
    bytes_ = workspace.numel() if isinstance(workspace, torch.Tensor) and workspace.dim() == 1 else None
    specs = (K, V, (table, "table", i32, (batch, width), False), (lens, "lens", i32, (batch,), False),
             (offsets, "offsets", i32, (batch + 1,), False), (counts, "counts", i32, (batch,), True),
             (slopes, "slopes", torch.float32, (cfg.n_q_heads,), True), (out, "out", half, q.shape, False),
             (workspace, "workspace", torch.uint8, (bytes_,), False))
    (Kp, Vp, tp, lp, op, np_, sp, outp, wp), devices = _tensors(specs)
    devices.add(q.get_device())
    _require_on(devices, ((q, "q"),) + specs, stream)
    _check(lib().pariskv_paged_attend(cfg.c(), qp, qs, ctypes.byref(_Pages(Kp, Vp, n_pages, size)), tp, width, lp, op, np_, t,
                                      most, batch, scale, softcap, sp, outp, wp, bytes_, _stream(stream)))
    return out


def stream_copy(dst, src, stream=None):
    """Reference streaming copy of src into dst (device tensors of equal byte size, a
    multiple of 16): measurement only."""
    nb = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nb:
        raise ValueError("dst and src must hold the same number of bytes")
    _check(lib().pariskv_stream_copy(_ptr(dst, "dst"), _ptr(src, "src"), nb, _stream(stream)))


def stream_read(src, sink, key=0xFFFFFFFF, stream=None):
    """Reference streaming read of src (a device tensor, multiple of 16 bytes); writes sink
    (a 4-byte device tensor) only if the folded data equals key: measurement only."""
    if sink.numel() * sink.element_size() < 4:
        raise ValueError("sink needs 4 bytes")
    _check(lib().pariskv_stream_read(_ptr(src, "src"), src.numel() * src.element_size(), key,
                                     _ptr(sink, "sink"), _stream(stream)))


def quantizer_table(m=8):
    """(tau[7], a[8]) float64 of the library's offline Lloyd-Max quantizer."""
    tau = (ctypes.c_double * 7)()
    a = (ctypes.c_double * 8)()
    _check(lib().pariskv_quantizer_table(m, tau, a))
    return np.array(tau[:]), np.array(a[:])


def rotation_signs(seed, D=HEAD_DIM):
    """The library's seeded rotation signs s in {+1, -1}^D (int8), see pariskv_rotation_signs."""
    out = (ctypes.c_int8 * D)()
    _check(lib().pariskv_rotation_signs(ctypes.c_uint64(seed & (2**64 - 1)), D, out))
    return np.array(out[:], dtype=np.int8)


def profile_enable(on=True):
    _check(lib().pariskv_profile_enable(1 if on else 0))


def profile_reset():
    _check(lib().pariskv_profile_reset())


def profile_read(max_entries=64):
    """{kernel name: (launches, total ms)} from events recorded since the last reset."""
    names = (ctypes.c_char_p * max_entries)()
    launches = (ctypes.c_int64 * max_entries)()
    ms = (ctypes.c_double * max_entries)()
    n = lib().pariskv_profile_read(max_entries, names, launches, ms)
    if n < 0:
        _check(n)
    return {names[i].decode(): (launches[i], ms[i]) for i in range(min(n, max_entries))}
