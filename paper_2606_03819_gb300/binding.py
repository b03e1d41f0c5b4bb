"""ctypes binding of the TreeFlash C ABI (include/treeflash.h).

Argument marshalling only: every function here passes raw device pointers of torch tensors,
the current CUDA stream and the dims/weights structs to the function of the same name in
lib/libtreeflash.so and raises TreeFlashError if it returns a status other than TF_OK. All
computation happens in the library's CUDA kernels; nothing here computes any part of the
path, and there is no fallback: without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from functools import cached_property
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "lib", "libtreeflash.so")

TF_OK, TF_ERR_INVALID_ARG, TF_ERR_UNSUPPORTED, TF_ERR_WORKSPACE, TF_ERR_CUDA, TF_ERR_DEVICE_STATUS, \
    TF_ERR_TIMEOUT = range(7)
TF_BF16, TF_F32 = 0, 1
MODES = {"ar": 0, "marginal": 1, "marginal_mary": 2}
APPROX = {"swiglu": 0, "linear": 1, "swiglu_2prev": 2}
TF_DEV_BAD_TOKEN, TF_DEV_UNDERFULL, TF_DEV_NONFINITE, TF_DEV_TIMEOUT, TF_DEV_RECOMPUTED = 1, 2, 4, 8, 16
TF_DEV_POOL_EMPTY, TF_DEV_BAD_LENGTH, TF_DEV_BAD_PAGE = 32, 64, 128


class TreeFlashError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn}: {msg} (status {status})")
        self.status = status


class TfDims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("d", ctypes.c_int32), ("V", ctypes.c_int32),
                ("I", ctypes.c_int32), ("gamma", ctypes.c_int32), ("M", ctypes.c_int32),
                ("K2", ctypes.c_int32), ("B", ctypes.c_int32), ("temperature", ctypes.c_float),
                ("rms_eps", ctypes.c_float), ("dtype", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("approx", ctypes.c_int32)]


class TfWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("lm_head", "embed", "norm_h", "norm_e", "w_gate", "w_up", "w_down", "w_lin")]


class TfCacheDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "heads", "kv_heads", "head_dim", "page", "n_pages", "max_pages", "dtype")]


EXPORTS = ("tf_status_string", "tf_version", "tf_kernel_launches", "tf_builder_counts", "tf_workspace_size", "tf_status_reset", "tf_status_read",
           "tf_stage1_marginals", "tf_stage2_ar_approx", "tf_build_tree", "tf_tree_mask", "tf_build_tree_mask",
           "tf_draft_tree_host", "tf_lmhead_partials", "tf_lmhead_merge", "tf_ar_approx",
           "tf_workspace_h_prime", "tf_workspace_view", "tf_stage1_marginals_static", "tf_accept_walk",
           "tf_set_wait_limit_ns", "tf_cache_plan", "tf_cache_append", "tf_attention_workspace_size",
           "tf_tree_attention", "tf_sample")

_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load lib/libtreeflash.so (built by __graft_entry__.build()). Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"TreeFlash CUDA library not found at {p}; build it with "
                           "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(p)
    P, I32, SZ, A = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_char_p
    D, W, C = ctypes.POINTER(TfDims), ctypes.POINTER(TfWeights), ctypes.POINTER(TfCacheDims)
    sig = {
        "tf_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "tf_version": (I32, []),
        "tf_kernel_launches": (ctypes.c_uint64, []),
        "tf_builder_counts": (ctypes.c_int, [ctypes.POINTER(ctypes.c_uint64)]),
        "tf_set_wait_limit_ns": (ctypes.c_int, [ctypes.c_uint64]),
        "tf_workspace_size": (ctypes.c_int, [D, ctypes.POINTER(SZ)]),
        "tf_status_reset": (ctypes.c_int, [P, SZ, P]),
        "tf_status_read": (ctypes.c_int, [P, SZ, ctypes.POINTER(I32), P]),
        "tf_stage1_marginals": (ctypes.c_int, [D, W, P, P, P, P, SZ, P]),
        "tf_stage2_ar_approx": (ctypes.c_int, [D, W, P, P, P, P, P, P, SZ, P]),
        "tf_build_tree": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, P, P, P]),
        "tf_tree_mask": (ctypes.c_int, [D, P, P, P, P, P, P]),
        "tf_build_tree_mask": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, P, P, P, P, P, P]),
        "tf_draft_tree_host": (ctypes.c_int, [D, W, P, P, P, P, P, P, P, P, P, P, P, SZ, P]),
        "tf_lmhead_partials": (ctypes.c_int, [D, P, P, I32, P, SZ, P]),
        "tf_lmhead_merge": (ctypes.c_int, [D, P, P, I32, I32, P, P, P, SZ, P]),
        "tf_ar_approx": (ctypes.c_int, [D, W, P, P, P, P, P, SZ, P]),
        "tf_workspace_h_prime": (ctypes.c_int, [D, P, SZ, ctypes.POINTER(P)]),
        "tf_workspace_view": (ctypes.c_int, [D, P, SZ, I32, ctypes.POINTER(P), ctypes.POINTER(SZ)]),
        "tf_stage1_marginals_static": (ctypes.c_int, [D, W, P, P, P, P, P]),
        "tf_accept_walk": (ctypes.c_int, [D, P, P, P, P, P, P, P]),
        "tf_cache_plan": (ctypes.c_int, [C, A, P]),
        "tf_cache_append": (ctypes.c_int, [C, A, P]),
        "tf_attention_workspace_size": (ctypes.c_int, [C, I32, ctypes.POINTER(SZ)]),
        "tf_tree_attention": (ctypes.c_int, [C, A, P]),
        "tf_sample": (ctypes.c_int, [A, P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    if path is None:
        _lib = lib
    return lib


def _check(fn: str, status: int):
    if status != TF_OK:
        msg = load_library().tf_status_string(status).decode()
        raise TreeFlashError(fn, status, msg)


@dataclass(frozen=True)
class Dims:
    batch: int
    d: int
    V: int
    I: int
    gamma: int
    M: int
    K2: int
    B: int
    temperature: float = 1.0
    rms_eps: float = 1e-6
    dtype: str = "bf16"
    mode: str = "ar"
    approx: str = "swiglu"      # "swiglu" (Eq. 1); the ablations' "linear" and "swiglu_2prev"

    @property
    def R(self) -> int:
        if self.approx == "swiglu_2prev" and self.mode == "ar":
            return 1 if self.gamma == 1 else 1 + self.M + self.M * self.M * (self.gamma - 2)
        return 1 + self.M * (self.gamma - 1)

    @property
    def K1(self) -> int:
        return max(self.M, self.K2)

    @property
    def k_in(self) -> int:
        """Width of the approximator input x: 2d, or 3d with two previous tokens."""
        return (3 if self.approx == "swiglu_2prev" and self.mode == "ar" else 2) * self.d

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    @cached_property
    def ref(self):
        """ctypes reference to the C struct of these (immutable) dimensions, built once."""
        return ctypes.byref(self.c())

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "ref"}   # copies and pickles make their own

    def c(self) -> TfDims:
        return TfDims(self.batch, self.d, self.V, self.I, self.gamma, self.M, self.K2, self.B,
                      self.temperature, self.rms_eps, TF_BF16 if self.dtype == "bf16" else TF_F32,
                      MODES[self.mode], APPROX[self.approx])

    @classmethod
    def from_config(cls, cfg) -> "Dims":
        return cls(cfg.batch, cfg.d, cfg.V, cfg.I, cfg.gamma, cfg.M, cfg.K2, cfg.B, cfg.temperature,
                   cfg.rms_eps, cfg.dtype, cfg.mode, getattr(cfg, "approx", "swiglu"))


WEIGHT_KEYS = ("lm_head", "embed", "norm_h", "norm_e", "w_gate", "w_up", "w_down", "w_lin")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the TreeFlash ABI must be contiguous")
    return t.data_ptr()


# The handle of the current stream alone: a Stream object costs more than the rest of a call's
# marshalling (and the small calls are bound by the host).
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _current_raw_stream(torch.cuda.current_device())


def _stream_on(stream, gpu: int):
    """_stream for a caller that knows the current device."""
    return _stream(stream) if stream is not None or _current_raw_stream is None else _current_raw_stream(gpu)


def weights_struct(w: dict) -> TfWeights:
    get = w.get
    return TfWeights(*[None if (t := get(k)) is None else t.data_ptr() for k in WEIGHT_KEYS])


def tf_version() -> int:
    return load_library().tf_version()


def tf_kernel_launches() -> int:
    """Kernels launched by the library so far in this process."""
    return int(load_library().tf_kernel_launches())


def tf_builder_counts() -> tuple:
    """(trees that the builder by levels left to the queue, times it dropped nodes to make room), on the
    current device since the library was loaded. Synchronises the device."""
    n = (ctypes.c_uint64 * 2)()
    _check("tf_builder_counts", load_library().tf_builder_counts(n))
    return n[0], n[1]


def tf_set_wait_limit_ns(ns: int) -> None:
    """Limit of the tensor-core kernels' waits for progress, for every later launch (0 = the
    default 2 s); a limit below a copy's latency makes calls time out (TF_DEV_TIMEOUT)."""
    _check("tf_set_wait_limit_ns", load_library().tf_set_wait_limit_ns(int(ns)))


def tf_workspace_size(dims: Dims) -> int:
    n = ctypes.c_size_t(0)
    _check("tf_workspace_size", load_library().tf_workspace_size(dims.ref, ctypes.byref(n)))
    return n.value


def alloc_workspace(dims: Dims, device="cuda") -> torch.Tensor:
    """A torch-owned workspace (256-byte aligned) of tf_workspace_size bytes."""
    n = tf_workspace_size(dims)
    buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + n]


def tf_status_reset(ws: torch.Tensor, stream=None):
    _check("tf_status_reset", load_library().tf_status_reset(_ptr(ws), ws.numel(), _stream(stream)))


def tf_status_read(ws: torch.Tensor, stream=None, raise_on_error: bool = False) -> int:
    flags = ctypes.c_int32(0)
    st = load_library().tf_status_read(_ptr(ws), ws.numel(), ctypes.byref(flags), _stream(stream))
    if st == TF_ERR_CUDA or raise_on_error:
        _check("tf_status_read", st)
    return flags.value


def tf_stage1_marginals(dims: Dims, w: dict, hidden, top_ids, top_logp, ws, stream=None):
    _check("tf_stage1_marginals", load_library().tf_stage1_marginals(
        dims.ref, ctypes.byref(weights_struct(w)), _ptr(hidden), _ptr(top_ids),
        _ptr(top_logp), _ptr(ws), ws.numel(), _stream(stream)))


def tf_stage2_ar_approx(dims: Dims, w: dict, hidden, root_tok, top_ids, child_ids, child_logp, ws,
                        stream=None):
    _check("tf_stage2_ar_approx", load_library().tf_stage2_ar_approx(
        dims.ref, ctypes.byref(weights_struct(w)), _ptr(hidden), _ptr(root_tok),
        _ptr(top_ids), _ptr(child_ids), _ptr(child_logp), _ptr(ws), ws.numel(), _stream(stream)))


def tf_build_tree(dims: Dims, root_tok, top_ids, top_logp, child_ids, child_logp, node_tok, node_parent,
                  node_depth, node_score, dev_status, stream=None):
    _check("tf_build_tree", load_library().tf_build_tree(
        dims.ref, _ptr(root_tok), _ptr(top_ids), _ptr(top_logp), _ptr(child_ids),
        _ptr(child_logp), _ptr(node_tok), _ptr(node_parent), _ptr(node_depth), _ptr(node_score),
        _ptr(dev_status), _stream(stream)))


def tf_tree_mask(dims: Dims, node_parent, node_depth, root_pos, mask, pos_ids, stream=None):
    _check("tf_tree_mask", load_library().tf_tree_mask(
        dims.ref, _ptr(node_parent), _ptr(node_depth), _ptr(root_pos), _ptr(mask),
        _ptr(pos_ids), _stream(stream)))


def tf_build_tree_mask(dims: Dims, root_tok, root_pos, top_ids, top_logp, child_ids, child_logp, node_tok,
                       node_parent, node_depth, node_score, mask, pos_ids, dev_status, stream=None):
    _check("tf_build_tree_mask", load_library().tf_build_tree_mask(
        dims.ref, _ptr(root_tok), _ptr(root_pos), _ptr(top_ids), _ptr(top_logp), _ptr(child_ids),
        _ptr(child_logp), _ptr(node_tok), _ptr(node_parent), _ptr(node_depth), _ptr(node_score), _ptr(mask),
        _ptr(pos_ids), _ptr(dev_status), _stream(stream)))


def tf_draft_tree_host(dims: Dims, w: dict, hidden, root_tok, root_pos, node_tok, node_parent, node_depth,
                       node_score, mask, pos_ids, dev_status, ws, stream=None):
    """Host tensors in and out (pinned memory recommended); weights and workspace on the device."""
    st = load_library().tf_draft_tree_host(
        dims.ref, ctypes.byref(weights_struct(w)), _ptr(hidden), _ptr(root_tok),
        _ptr(root_pos), _ptr(node_tok), _ptr(node_parent), _ptr(node_depth), _ptr(node_score), _ptr(mask),
        _ptr(pos_ids), _ptr(dev_status), _ptr(ws), ws.numel(), _stream(stream))
    if st not in (TF_OK, TF_ERR_DEVICE_STATUS):
        _check("tf_draft_tree_host", st)
    return st


def tf_accept_walk(dims: Dims, node_tok, node_parent, verifier_tok, accept_len, accept_path, next_tok,
                   stream=None):
    _check("tf_accept_walk", load_library().tf_accept_walk(
        dims.ref, _ptr(node_tok), _ptr(node_parent), _ptr(verifier_tok), _ptr(accept_len),
        _ptr(accept_path), _ptr(next_tok), _stream(stream)))


def tf_lmhead_partials(dims: Dims, lm_head, x, n_rows: int, ws, stream=None):
    _check("tf_lmhead_partials", load_library().tf_lmhead_partials(
        dims.ref, _ptr(lm_head), _ptr(x), n_rows, _ptr(ws), ws.numel(), _stream(stream)))


def tf_lmhead_merge(dims: Dims, lm_head, x, n_rows: int, k: int, out_ids, out_logp, ws, stream=None):
    _check("tf_lmhead_merge", load_library().tf_lmhead_merge(
        dims.ref, _ptr(lm_head), _ptr(x), n_rows, k, _ptr(out_ids), _ptr(out_logp), _ptr(ws),
        ws.numel(), _stream(stream)))


def tf_ar_approx(dims: Dims, w: dict, hidden, root_tok, top_ids, h_prime, ws, stream=None):
    _check("tf_ar_approx", load_library().tf_ar_approx(
        dims.ref, ctypes.byref(weights_struct(w)), _ptr(hidden), _ptr(root_tok), _ptr(top_ids),
        _ptr(h_prime), _ptr(ws), ws.numel(), _stream(stream)))


def tf_workspace_h_prime(dims: Dims, ws) -> torch.Tensor:
    """h' [b, R, d] as a tensor view of the workspace (no copy)."""
    p = ctypes.c_void_p()
    _check("tf_workspace_h_prime", load_library().tf_workspace_h_prime(
        dims.ref, _ptr(ws), ws.numel(), ctypes.byref(p)))
    off = p.value - ws.data_ptr()
    esize = 2 if dims.dtype == "bf16" else 4
    n = dims.batch * dims.R * dims.d * esize
    return ws[off:off + n].view(dims.torch_dtype).view(dims.batch, dims.R, dims.d)


TF_VIEW_X, TF_VIEW_A, TF_VIEW_H_PRIME, TF_VIEW_HALVES, TF_VIEW_CHUNKS = 0, 1, 2, 3, 4


def tf_workspace_view(dims: Dims, ws, view: int, n_rows: Optional[int] = None) -> torch.Tensor:
    """x [b*R, k_in], A [b*R, I] or h' [b*R, d] as a tensor view of the workspace (no copy); for
    TF_VIEW_HALVES / TF_VIEW_CHUNKS the partials of the last LM-head pass over n_rows rows as
    float32 [n_tiles, 2 or 8, n_rows, 4]."""
    p, n = ctypes.c_void_p(), ctypes.c_size_t()
    _check("tf_workspace_view", load_library().tf_workspace_view(
        dims.ref, _ptr(ws), ws.numel(), view, ctypes.byref(p), ctypes.byref(n)))
    off = p.value - ws.data_ptr()
    if view in (TF_VIEW_HALVES, TF_VIEW_CHUNKS):
        n_tiles = (dims.V + 255) // 256
        parts = 2 if view == TF_VIEW_HALVES else 8
        nb = n_tiles * parts * n_rows * 16
        return ws[off:off + nb].view(torch.float32).view(n_tiles, parts, n_rows, 4)
    cols = {TF_VIEW_X: dims.k_in, TF_VIEW_A: dims.I, TF_VIEW_H_PRIME: dims.d}[view]
    return ws[off:off + n.value].view(dims.torch_dtype).view(dims.batch * dims.R, cols)


TF_STATIC_SCRATCH_BYTES = 8 << 20


def tf_stage1_marginals_static(dims: Dims, w: dict, hidden, top_ids, top_logp, dev_status, stream=None):
    """tf_stage1_marginals for callers that cannot allocate: no workspace, the library's own fixed
    scratch array instead. dev_status is a 1-element int32 device tensor that receives the call's
    TF_DEV_* flags. Calls that overlap on the GPU share that array and race."""
    _check("tf_stage1_marginals_static", load_library().tf_stage1_marginals_static(
        dims.ref, ctypes.byref(weights_struct(w)), _ptr(hidden), _ptr(top_ids),
        _ptr(top_logp), _ptr(dev_status), _stream(stream)))


# ---- the verifier's side ------------------------------------------------------------------------

@dataclass(frozen=True)
class CacheDims:
    """Sizes of the paged 8-bit cache and of the attention over it (tf_cache_dims)."""
    batch: int
    heads: int
    kv_heads: int
    head_dim: int
    page: int
    n_pages: int
    max_pages: int
    dtype: str = "bf16"

    @cached_property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    @cached_property
    def ref(self):
        """ctypes reference to the C struct of these (immutable) dimensions, built once."""
        return ctypes.byref(self.c())

    @cached_property
    def per_seq(self):
        return (self.batch,)

    @cached_property
    def table_shape(self):
        return (self.batch, self.max_pages)

    @cached_property
    def pages_shape(self):
        return (self.n_pages, self.kv_heads, self.page, self.head_dim)

    @cached_property
    def scales_shape(self):
        return (self.n_pages, self.kv_heads)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "ref"}   # copies and pickles make their own

    def c(self) -> TfCacheDims:
        return TfCacheDims(self.batch, self.heads, self.kv_heads, self.head_dim, self.page, self.n_pages,
                           self.max_pages, TF_BF16 if self.dtype == "bf16" else TF_F32)


# The argument structs of include/treeflash.h in their order ("@": the C compiler's alignment; P pointer, q int64, N
# size_t, f float, i int32). Packing one costs a fraction of what ctypes takes for as many arguments, and the calls of
# the verifier's side are bound by the host where a step is small.
_PLAN = struct.Struct("@8P2i")
_APPEND = struct.Struct("@2P2q7P2i")
_ATTENTION = struct.Struct("@3P3q11PNfi")
_SAMPLE = struct.Struct("@8Pq4i")

_I32, _F32, _U8 = torch.int32, torch.float32, torch.uint8


# The checks below are written out in one condition per call: a function call for each tensor would cost as much as the
# checks. Where the condition fails, _take finds the tensor that is to blame. Every tensor lies on the GPU that the call's
# kernels run on, the current one: they would read another pointer as it is.

def _take(name: str, t: torch.Tensor, dtype, shape) -> int:
    """Data pointer of a contiguous tensor of this type and shape."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)}, got "
                         f"{t.dtype} {tuple(t.shape)}{'' if t.is_contiguous() else ', not contiguous'}")
    return t.data_ptr()


def _take_rows(name: str, t: torch.Tensor, dtype, batch: int, heads: int, head_dim: int) -> tuple:
    """(rows per sequence, elements from one row to the next) of a [batch, n, heads, head_dim] tensor whose rows are
    contiguous inside and evenly spaced over the sequences: a slice of a fused projection's output is one."""
    shape, st = t.shape, t.stride()
    if t.dtype is not dtype or len(shape) != 4 or shape != (batch, shape[1], heads, head_dim):
        raise ValueError(f"{name}: expected {dtype} [{batch}, n, {heads}, {head_dim}], got {t.dtype} {tuple(shape)}")
    n, row = shape[1], st[1]
    if st == (n * row, row, head_dim, 1) and (n > 1 or batch > 1 and row >= heads * head_dim):
        return n, row
    # dimensions of one element may have any stride, also one that rows could not have
    if n == 1:
        row = st[0] if batch > 1 else row if row >= heads * head_dim and row % 16 == 0 else heads * head_dim
    if (head_dim > 1 and st[3] != 1) or (heads > 1 and st[2] != head_dim) or (batch > 1 and n > 0 and st[0] != n * row):
        raise ValueError(f"{name}: rows must be contiguous and evenly spaced, got strides {st}")
    return n, row


def _blame_device(*tensors):
    for name, t in tensors:
        if t is not None and (t.get_device() < 0 or t.get_device() != torch.cuda.current_device()):
            raise ValueError(f"{name}: expected a tensor on the current CUDA device, got one on {t.device}")
    raise ValueError("inconsistent tensors")


def _blame(*wants, rows=()):
    for name, t, dtype, shape in wants:
        if t is not None:
            _take(name, t, dtype, shape)
    _blame_device(*rows, *((name, t) for name, t, _, _ in wants))


def tf_cache_plan(dims: CacheDims, seq_len, delta, extra: int, block_table, free_list, free_count, slot_map, new_len,
                  dev_status, stream=None):
    """Change every sequence's length by delta + extra: pages taken and given back, block table kept, slots of the new
    tokens in slot_map [batch, width] (None: not wanted). new_len may be seq_len."""
    b, table, pool = dims.per_seq, dims.table_shape, (dims.n_pages,)
    width = 0 if slot_map is None else slot_map.shape[-1]
    if not (seq_len.dtype is _I32 and delta.dtype is _I32 and block_table.dtype is _I32 and free_list.dtype is _I32 and
            free_count.dtype is _I32 and new_len.dtype is _I32 and dev_status.dtype is _I32 and
            seq_len.shape == b and delta.shape == b and new_len.shape == b and dev_status.shape == b and
            block_table.shape == table and free_list.shape == pool and free_count.shape == (1,) and
            seq_len.is_contiguous() and delta.is_contiguous() and block_table.is_contiguous() and free_list.is_contiguous() and
            new_len.is_contiguous() and dev_status.is_contiguous() and
            (gpu := seq_len.get_device()) >= 0 and delta.get_device() == gpu and block_table.get_device() == gpu and
            free_list.get_device() == gpu and free_count.get_device() == gpu and new_len.get_device() == gpu and
            dev_status.get_device() == gpu and gpu == torch.cuda.current_device() and
            (slot_map is None or slot_map.dtype is _I32 and slot_map.shape == (dims.batch, width) and slot_map.is_contiguous() and
             slot_map.get_device() == gpu)):
        _blame(("seq_len", seq_len, _I32, b), ("delta", delta, _I32, b), ("block_table", block_table, _I32, table),
               ("free_list", free_list, _I32, pool), ("free_count", free_count, _I32, (1,)), ("new_len", new_len, _I32, b),
               ("dev_status", dev_status, _I32, b), ("slot_map", slot_map, _I32, (dims.batch, width)))
    args = _PLAN.pack(seq_len.data_ptr(), delta.data_ptr(), block_table.data_ptr(), free_list.data_ptr(), free_count.data_ptr(),
                      0 if slot_map is None else slot_map.data_ptr(), new_len.data_ptr(), dev_status.data_ptr(), extra, width)
    st = load_library().tf_cache_plan(dims.ref, args, _stream_on(stream, gpu))
    if st:
        _check("tf_cache_plan", st)


def tf_cache_append(dims: CacheDims, k, v, slot_map, src, k_cache, v_cache, k_scale, v_scale, dev_status, stream=None):
    """Quantise rows of k and v [batch, n, kv_heads, head_dim] into the slots of slot_map [batch, width]: row src[s, j]
    (None: row j) into slot j, one scale for each page and head."""
    b, dt, h, hd = dims.batch, dims.torch_dtype, dims.kv_heads, dims.head_dim
    n, k_row = _take_rows("k", k, dt, b, h, hd)
    vn, v_row = _take_rows("v", v, dt, b, h, hd)
    if vn != n:
        raise ValueError("k and v must have as many rows")
    slots, pages, scales = slot_map.shape, dims.pages_shape, dims.scales_shape
    if len(slots) != 2 or slots[0] != b:
        raise ValueError(f"slot_map: expected [{b}, width], got {tuple(slots)}")
    if not (slot_map.dtype is _I32 and k_cache.dtype is _U8 and v_cache.dtype is _U8 and k_scale.dtype is _F32 and
            v_scale.dtype is _F32 and dev_status.dtype is _I32 and k_cache.shape == pages and v_cache.shape == pages and
            k_scale.shape == scales and v_scale.shape == scales and dev_status.shape == dims.per_seq and
            slot_map.is_contiguous() and k_cache.is_contiguous() and v_cache.is_contiguous() and k_scale.is_contiguous() and
            v_scale.is_contiguous() and dev_status.is_contiguous() and
            (gpu := k.get_device()) >= 0 and v.get_device() == gpu and slot_map.get_device() == gpu and k_cache.get_device() == gpu and
            v_cache.get_device() == gpu and k_scale.get_device() == gpu and v_scale.get_device() == gpu and
            dev_status.get_device() == gpu and gpu == torch.cuda.current_device() and
            (src is None or src.dtype is _I32 and src.shape == slots and src.is_contiguous() and src.get_device() == gpu)):
        _blame(("slot_map", slot_map, _I32, slots), ("src", src, _I32, slots), ("k_cache", k_cache, _U8, pages),
               ("v_cache", v_cache, _U8, pages), ("k_scale", k_scale, _F32, scales), ("v_scale", v_scale, _F32, scales),
               ("dev_status", dev_status, _I32, dims.per_seq), rows=(("k", k), ("v", v)))
    args = _APPEND.pack(k.data_ptr(), v.data_ptr(), k_row, v_row, slot_map.data_ptr(), 0 if src is None else src.data_ptr(),
                        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), dev_status.data_ptr(), n,
                        slots[1])
    st = load_library().tf_cache_append(dims.ref, args, _stream_on(stream, gpu))
    if st:
        _check("tf_cache_append", st)


def tf_attention_workspace_size(dims: CacheDims, n: int) -> int:
    size = ctypes.c_size_t(0)
    _check("tf_attention_workspace_size", load_library().tf_attention_workspace_size(dims.ref, n, ctypes.byref(size)))
    return size.value


def alloc_attention_workspace(dims: CacheDims, n: int, device="cuda") -> torch.Tensor:
    """A torch-owned workspace (256-byte aligned) for tf_tree_attention with n new tokens per sequence."""
    size = tf_attention_workspace_size(dims, n)
    buf = torch.empty(size + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + size]


def tf_tree_attention(dims: CacheDims, q, k, v, k_cache, v_cache, k_scale, v_scale, block_table, seq_len, mask,
                      scale: float, out, lse, dev_status, ws, stream=None):
    """Attention of q [batch, n, heads, head_dim] over each sequence's cached tokens and over the new tokens' own k and
    v [batch, n, kv_heads, head_dim]; mask [batch, n, n] uint8 (None: causal among the new tokens)."""
    b, dt, hq, h, hd = dims.batch, dims.torch_dtype, dims.heads, dims.kv_heads, dims.head_dim
    n, q_row = _take_rows("q", q, dt, b, hq, hd)
    kn, k_row = _take_rows("k", k, dt, b, h, hd)
    vn, v_row = _take_rows("v", v, dt, b, h, hd)
    if kn != n or vn != n:
        raise ValueError("q, k and v must have as many rows")
    pages, scales, per_seq, table = dims.pages_shape, dims.scales_shape, dims.per_seq, dims.table_shape
    if not (k_cache.dtype is _U8 and v_cache.dtype is _U8 and k_scale.dtype is _F32 and v_scale.dtype is _F32 and
            block_table.dtype is _I32 and seq_len.dtype is _I32 and dev_status.dtype is _I32 and out.dtype is dt and
            k_cache.shape == pages and v_cache.shape == pages and k_scale.shape == scales and v_scale.shape == scales and
            block_table.shape == table and seq_len.shape == per_seq and dev_status.shape == per_seq and
            out.shape == (b, n, hq, hd) and k_cache.is_contiguous() and v_cache.is_contiguous() and
            k_scale.is_contiguous() and v_scale.is_contiguous() and block_table.is_contiguous() and
            seq_len.is_contiguous() and dev_status.is_contiguous() and out.is_contiguous() and
            (gpu := q.get_device()) >= 0 and k.get_device() == gpu and v.get_device() == gpu and k_cache.get_device() == gpu and
            v_cache.get_device() == gpu and k_scale.get_device() == gpu and v_scale.get_device() == gpu and
            block_table.get_device() == gpu and seq_len.get_device() == gpu and dev_status.get_device() == gpu and
            out.get_device() == gpu and ws.get_device() == gpu and gpu == torch.cuda.current_device() and
            (mask is None or mask.dtype is _U8 and mask.shape == (b, n, n) and mask.is_contiguous() and mask.get_device() == gpu) and
            (lse is None or lse.dtype is _F32 and lse.shape == (b, n, hq) and lse.is_contiguous() and lse.get_device() == gpu) and
            ws.dtype is _U8 and ws.is_contiguous()):
        _blame(("k_cache", k_cache, _U8, pages), ("v_cache", v_cache, _U8, pages), ("k_scale", k_scale, _F32, scales),
               ("v_scale", v_scale, _F32, scales), ("block_table", block_table, _I32, table), ("seq_len", seq_len, _I32, per_seq),
               ("mask", mask, _U8, (b, n, n)), ("out", out, dt, (b, n, hq, hd)), ("lse", lse, _F32, (b, n, hq)),
               ("dev_status", dev_status, _I32, per_seq), ("ws", ws, _U8, ws.shape), rows=(("q", q), ("k", k), ("v", v)))
    args = _ATTENTION.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_row, k_row, v_row, k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(),
        v_scale.data_ptr(), block_table.data_ptr(), seq_len.data_ptr(), 0 if mask is None else mask.data_ptr(), out.data_ptr(),
        0 if lse is None else lse.data_ptr(), dev_status.data_ptr(), ws.data_ptr(), ws.numel(), scale, n)
    st = load_library().tf_tree_attention(dims.ref, args, _stream_on(stream, gpu))
    if st:
        _check("tf_tree_attention", st)


def tf_sample(logits, u, tok, logp=None, temperature=None, top_k=None, top_p=None, min_p=None, rows_per_seq: int = 1,
              stream=None):
    """One token for each row of logits [rows, V] (bf16 or fp32, rows may be strided) from the uniform numbers u
    [rows]: tok [rows] int32, logp [rows]. Parameters are per sequence: [ceil(rows / rows_per_seq)] each, None leaves
    its filter out."""
    dt, shape, st = logits.dtype, logits.shape, logits.stride()
    if len(shape) != 2 or (dt is not torch.bfloat16 and dt is not _F32) or (shape[1] > 1 and st[1] != 1):
        raise ValueError("logits: expected bf16 or fp32 [rows, V] with contiguous rows")
    rows, V = shape
    per_row, seqs = (rows,), (-(-rows // max(1, rows_per_seq)),)
    args = _SAMPLE.pack(
        logits.data_ptr(), 0 if temperature is None else _take("temperature", temperature, _F32, seqs),
        0 if top_k is None else _take("top_k", top_k, _I32, seqs), 0 if top_p is None else _take("top_p", top_p, _F32, seqs),
        0 if min_p is None else _take("min_p", min_p, _F32, seqs), _take("u", u, _F32, per_row), _take("tok", tok, _I32, per_row),
        0 if logp is None else _take("logp", logp, _F32, per_row), st[0] if rows > 1 else V, rows, V,
        TF_F32 if dt is _F32 else TF_BF16, rows_per_seq)
    if not ((gpu := logits.get_device()) >= 0 and u.get_device() == gpu and tok.get_device() == gpu and
            (logp is None or logp.get_device() == gpu) and (temperature is None or temperature.get_device() == gpu) and
            (top_k is None or top_k.get_device() == gpu) and (top_p is None or top_p.get_device() == gpu) and
            (min_p is None or min_p.get_device() == gpu) and gpu == torch.cuda.current_device()):
        _blame_device(("logits", logits), ("u", u), ("tok", tok), ("logp", logp), ("temperature", temperature), ("top_k", top_k),
                      ("top_p", top_p), ("min_p", min_p))
    status = load_library().tf_sample(args, _stream_on(stream, gpu))
    if status:
        _check("tf_sample", status)
