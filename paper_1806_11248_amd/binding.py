"""Thin ctypes binding of libgbt.so.

Argument marshalling only: every step of the path runs inside the library's HIP
kernels.  torch supplies device memory (``tensor.data_ptr()``) and the stream.
There is no fallback: if the library has not been built, or there is no
MI355X, loading or ``Context()`` raises.
"""
from __future__ import annotations

import array
import contextlib
import ctypes as C
import math
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgbt.so")

OK, EINVAL, ENOMEM, EHIP, EUNSUPPORTED = 0, -1, -2, -3, -4
GROW_PLANNED = 16   # GBT_GROW_PLANNED
PARTITION_STATIC_MAX_ROWS = 1 << 22   # GBT_PARTITION_STATIC_MAX_ROWS
OBJECTIVES = {"squared": 0, "logistic": 1}

# every symbol include/gbt.h declares
SYMBOLS = [
    "gbt_create", "gbt_destroy", "gbt_last_error", "gbt_version",
    "gbt_quantise_workspace_bytes", "gbt_quantise", "gbt_quantise_packed", "gbt_bits", "gbt_packed_words", "gbt_compress",
    "gbt_gradients", "gbt_gpair_fixed", "gbt_sum_gpair", "gbt_build_hist", "gbt_hist_subtract",
    "gbt_hist_export_f64", "gbt_eval_split", "gbt_partition_workspace_bytes", "gbt_partition",
    "gbt_partition_static",
    "gbt_grow_tree_workspace_bytes", "gbt_grow_tree_path", "gbt_grow_tree_form", "gbt_grow_tree",
    "gbt_grow_tree_lossguide_workspace_bytes", "gbt_grow_tree_lossguide", "gbt_boost_round",
    "gbt_predict_workspace_bytes", "gbt_predict",
    "gbt_profile_enable", "gbt_profile_read", "gbt_measure_stream_read",
    "gbt_sparse_entry_bytes", "gbt_sparse_capacity", "gbt_compress_sparse_workspace_bytes", "gbt_compress_sparse_count", "gbt_compress_sparse",
    "gbt_build_hist_sparse", "gbt_grow_tree_sparse_workspace_bytes", "gbt_grow_tree_sparse", "gbt_predict_sparse",
    "gbt_grow_tree_sparse_lossguide_workspace_bytes", "gbt_grow_tree_sparse_lossguide",
    "gbt_attention_workspace_bytes", "gbt_attention", "gbt_attention_backward_workspace_bytes", "gbt_attention_backward",
    "gbt_gradient_list_bytes", "gbt_gradient_list", "gbt_clip_gradients",
    "gbt_embedding", "gbt_embedding_backward_workspace_bytes", "gbt_embedding_backward",
    "gbt_norm_rotate", "gbt_norm_rotate_backward_workspace_bytes", "gbt_norm_rotate_backward",
    "gbt_matrix_list_bytes", "gbt_matrix_list", "gbt_orthogonalise_workspace_bytes", "gbt_orthogonalise",
]

PROF_LEVELS = 18   # GBT_PROF_LEVELS
PROF_CLASSES = ["hist_root", "hist_node", "partition", "eval", "clear", "other", "hist_first", "hist_inplace"]


class GbtError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"libgbt error {code}: {text}")
        self.code = code


class Params(C.Structure):
    _fields_ = [("max_depth", C.c_int32), ("max_bins", C.c_int32), ("lambda_", C.c_double),
                ("gamma", C.c_double), ("min_child_weight", C.c_double), ("eta", C.c_double),
                ("objective", C.c_int32), ("base_margin", C.c_float)]


class Split(C.Structure):
    _fields_ = [("feature", C.c_int32), ("bin", C.c_int32), ("default_left", C.c_int32),
                ("valid", C.c_int32), ("gain", C.c_double), ("GL", C.c_double), ("HL", C.c_double),
                ("GR", C.c_double), ("HR", C.c_double), ("GLq", C.c_int64), ("HLq", C.c_int64)]


class Profile(C.Structure):
    _fields_ = [("ms", C.c_double * 8), ("bytes", C.c_double * 8), ("launches", C.c_int64 * 8),
                ("alg_bytes", C.c_double * 8), ("level_ms", C.c_double * PROF_LEVELS),
                ("level_alg_bytes", C.c_double * PROF_LEVELS), ("level_row_features", C.c_double * PROF_LEVELS),
                ("level_launches", C.c_int64 * PROF_LEVELS)]


class Tree(C.Structure):
    _fields_ = [("capacity", C.c_int32), ("n_nodes", C.c_int32),
                ("feature", C.c_void_p), ("bin", C.c_void_p), ("default_left", C.c_void_p),
                ("left", C.c_void_p), ("right", C.c_void_p), ("threshold", C.c_void_p),
                ("weight", C.c_void_p), ("gain", C.c_void_p), ("sumG", C.c_void_p),
                ("sumH", C.c_void_p), ("n_rows", C.c_void_p)]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class AttentionParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_seq", C.c_int32), ("max_q", C.c_int32), ("max_k", C.c_int32), ("causal", C.c_int32),
                ("n_buckets", C.c_int32), ("scale", C.c_float), ("q_rows", C.c_int64), ("k_rows", C.c_int64),
                ("q_ptr", C.c_void_p), ("k_ptr", C.c_void_p), ("k_len", C.c_void_p), ("bias", C.c_void_p),
                ("cuts", C.c_void_p)]


class Gradient(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


class EmbeddingParams(C.Structure):
    _fields_ = [("table_dtype", C.c_int32), ("out_dtype", C.c_int32), ("id_bytes", C.c_int32), ("width", C.c_int32), ("n_ids", C.c_int64),
                ("n_rows", C.c_int64), ("table_stride", C.c_int64), ("out_stride", C.c_int64), ("ids", C.c_void_p), ("scale", C.c_float)]


class NormRotateParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("turned", C.c_int32),
                ("halves", C.c_int32), ("store", C.c_int32), ("n_seq", C.c_int32), ("position_bytes", C.c_int32), ("eps", C.c_float),
                ("rows", C.c_int64), ("out_rows", C.c_int64), ("q_ptr", C.c_void_p), ("k_ptr", C.c_void_p), ("k_len", C.c_void_p),
                ("positions", C.c_void_p), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("turns", C.c_void_p)]


class Matrix(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("dtype", C.c_int32), ("scale", C.c_float)]


_NO_STREAM = contextlib.nullcontext()
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # GBT_F32, GBT_BF16, GBT_F16

_TREE_FIELDS = [("feature", np.int32), ("bin", np.int32), ("default_left", np.int32), ("left", np.int32),
                ("right", np.int32), ("threshold", np.float32), ("weight", np.float64),
                ("gain", np.float64), ("sumG", np.float64), ("sumH", np.float64), ("n_rows", np.int64)]

_lib = None


def load():
    """Load libgbt.so (built in-tree by ``paper_1806_11248_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1806_11248_amd.build` "
                           "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    L.gbt_version.restype = C.c_char_p
    L.gbt_last_error.restype = C.c_char_p
    L.gbt_last_error.argtypes = [C.c_void_p]
    L.gbt_create.argtypes = [C.POINTER(C.c_void_p), C.c_int32, C.c_void_p]
    L.gbt_destroy.argtypes = [C.c_void_p]
    L.gbt_bits.argtypes = [C.c_uint32]
    L.gbt_packed_words.restype = C.c_int64
    L.gbt_packed_words.argtypes = [C.c_int64, C.c_int32, C.c_int32]
    for nm in ("gbt_quantise_workspace_bytes", "gbt_partition_workspace_bytes",
               "gbt_grow_tree_workspace_bytes", "gbt_predict_workspace_bytes"):
        getattr(L, nm).restype = C.c_size_t
    L.gbt_quantise_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int64, C.c_int32]
    L.gbt_partition_workspace_bytes.argtypes = [C.c_int64]
    L.gbt_grow_tree_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    L.gbt_grow_tree_lossguide_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    L.gbt_grow_tree_lossguide_workspace_bytes.restype = C.c_size_t
    L.gbt_grow_tree_path.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    L.gbt_grow_tree_path.restype = C.c_int32
    L.gbt_grow_tree_form.argtypes = [C.c_void_p, C.c_int64] + [C.c_int32] * 5
    L.gbt_grow_tree_form.restype = C.c_int32
    L.gbt_predict_workspace_bytes.argtypes = [C.c_void_p, C.c_int32]
    vp, i32, i64, u32, f64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_double, C.c_size_t
    L.gbt_quantise.argtypes = [vp, vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, vp, vp, vp, sz]
    L.gbt_compress.argtypes = [vp, vp, i64, i32, u32, vp, vp]
    L.gbt_gradients.argtypes = [vp, i32, vp, vp, i64, vp]
    L.gbt_gpair_fixed.argtypes = [vp, vp, i64, vp, vp, vp, sz]
    L.gbt_sum_gpair.argtypes = [vp, vp, vp, i64, vp, vp, sz]
    L.gbt_build_hist.argtypes = [vp, vp, i32, i64, i32, i32, i32, vp, i64, vp, vp]
    L.gbt_hist_subtract.argtypes = [vp, vp, vp, vp, i64]
    L.gbt_hist_export_f64.argtypes = [vp, vp, i32, i32, vp, vp]
    L.gbt_eval_split.argtypes = [vp, vp, vp, i32, i32, i64, i64, vp, vp, vp, vp, sz]
    L.gbt_partition.argtypes = [vp, vp, i32, i64, i32, vp, i64, i64, i32, i32, i32, i32, vp, sz, vp]
    L.gbt_partition_static.argtypes = [vp, vp, i32, i64, i32, vp, i64, i64, i32, i32, i32, i32, vp]
    L.gbt_grow_tree.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    L.gbt_grow_tree_lossguide.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz]
    L.gbt_boost_round.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    L.gbt_predict.argtypes = [vp, vp, i32, vp, i32, i32, vp, i64, i32, f64, vp, vp, sz]
    L.gbt_sparse_entry_bytes.argtypes = [i32, i32]
    L.gbt_sparse_capacity.argtypes = [i64]
    L.gbt_sparse_capacity.restype = i64
    L.gbt_compress_sparse_workspace_bytes.argtypes = [i64]
    L.gbt_compress_sparse_workspace_bytes.restype = sz
    L.gbt_compress_sparse_count.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, sz]
    L.gbt_compress_sparse.argtypes = [vp, vp, i64, i32, i32, i32, vp, i64, vp, i64]
    L.gbt_build_hist_sparse.argtypes = [vp, vp, vp, i64, i32, i32, i64, i64, vp, vp]
    L.gbt_grow_tree_sparse_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
    L.gbt_grow_tree_sparse_workspace_bytes.restype = sz
    L.gbt_grow_tree_sparse.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    L.gbt_grow_tree_sparse_lossguide_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
    L.gbt_grow_tree_sparse_lossguide_workspace_bytes.restype = sz
    L.gbt_grow_tree_sparse_lossguide.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz]
    L.gbt_predict_sparse.argtypes = [vp, vp, i32, vp, vp, i64, i32, i32, f64, vp, vp, sz]
    L.gbt_attention_workspace_bytes.argtypes = [vp]
    L.gbt_attention_workspace_bytes.restype = sz
    L.gbt_attention.argtypes = [vp] * 9 + [sz]
    L.gbt_attention_backward_workspace_bytes.argtypes = [vp]
    L.gbt_attention_backward_workspace_bytes.restype = sz
    L.gbt_attention_backward.argtypes = [vp] * 14 + [sz]
    L.gbt_gradient_list_bytes.argtypes = [vp, i64]
    L.gbt_gradient_list_bytes.restype = sz
    L.gbt_gradient_list.argtypes = [vp, vp, i64, vp, sz, vp]
    L.gbt_clip_gradients.argtypes = [vp, vp, i32, f64, vp, vp, sz]
    L.gbt_embedding.argtypes = [vp, vp, vp, vp]
    L.gbt_embedding_backward_workspace_bytes.argtypes = [vp]
    L.gbt_embedding_backward_workspace_bytes.restype = sz
    L.gbt_embedding_backward.argtypes = [vp, vp, vp, vp, i32, vp, sz]
    L.gbt_norm_rotate.argtypes = [vp] * 8
    L.gbt_norm_rotate_backward_workspace_bytes.argtypes = [vp]
    L.gbt_norm_rotate_backward_workspace_bytes.restype = sz
    L.gbt_norm_rotate_backward.argtypes = [vp] * 11 + [sz]
    L.gbt_matrix_list_bytes.argtypes = [vp, i64]
    L.gbt_matrix_list_bytes.restype = sz
    L.gbt_matrix_list.argtypes = [vp, vp, i64, vp, sz]
    L.gbt_orthogonalise_workspace_bytes.argtypes = [vp, i64]
    L.gbt_orthogonalise_workspace_bytes.restype = sz
    f32 = C.c_float
    L.gbt_orthogonalise.argtypes = [vp, vp, vp, i64, i32, f32, f32, f32, vp, sz]
    L.gbt_profile_enable.argtypes = [vp, i32]
    L.gbt_profile_read.argtypes = [vp, vp]
    L.gbt_measure_stream_read.argtypes = [vp, vp, sz, i32, vp, vp, sz]
    _lib = L
    return L


def bits_for(max_value: int) -> int:
    return int(load().gbt_bits(max_value))


def packed_words(n: int, F: int, bits: int) -> int:
    return int(load().gbt_packed_words(n, F, bits))


def make_params(*, max_depth, max_bins, lam=1.0, gamma=0.0, min_child_weight=1.0, eta=1.0,
                objective="squared", base_margin=0.0) -> Params:
    return Params(max_depth, max_bins, lam, gamma, min_child_weight, eta,
                  OBJECTIVES.get(objective, 0), base_margin)


def new_tree(max_depth: int) -> dict:
    cap = 2 ** (max_depth + 1) - 1
    t = {nm: np.zeros(cap, dt) for nm, dt in _TREE_FIELDS}
    t["capacity"] = cap
    t["n_nodes"] = 0
    return t


def new_tree_leaves(max_leaves: int) -> dict:
    """Arrays for a tree of at most max_leaves leaves (2*max_leaves - 1 nodes)."""
    cap = max(1, 2 * max_leaves - 1)   # a bad budget is the library's to refuse
    t = {nm: np.zeros(cap, dt) for nm, dt in _TREE_FIELDS}
    t["capacity"] = cap
    t["n_nodes"] = 0
    return t


def _address(a) -> int:
    try:
        return C.addressof(C.c_char.from_buffer(a))   # a third of the time of a.ctypes.data
    except (TypeError, ValueError, BufferError):      # read-only, empty or strided
        return a.ctypes.data


_TREE_NAMES = [nm for nm, _ in _TREE_FIELDS]


def _tree_struct(t: dict) -> Tree:
    return Tree(int(t["capacity"]), int(t["n_nodes"]), *[_address(t[nm]) for nm in _TREE_NAMES])


# what prediction reads of a tree, in gbt_tree's order; the other addresses stay NULL
_WALK_NAMES = ["feature", "bin", "default_left", "left", "right", "threshold", "weight"]
_WORDS = C.sizeof(Tree) // 8


def _tree_table(trees):
    """An array of gbt_tree for prediction, filled as 64-bit words: a model has hundreds of trees and seven addresses each,
    and field by field that took longer than the walk itself (100 trees: 0.7 ms)."""
    arr = (Tree * len(trees))()
    if not trees:
        return arr
    words = np.zeros((len(trees), _WORDS), np.int64)
    counts = words.view(np.int32)                 # the two counts share the first word
    counts[:, 0] = [t["capacity"] for t in trees]
    counts[:, 1] = [t["n_nodes"] for t in trees]
    view, at = C.c_char.from_buffer, C.addressof
    try:
        flat = [at(view(t[nm])) for t in trees for nm in _WALK_NAMES]
    except (TypeError, ValueError, BufferError):
        flat = [_address(t[nm]) for t in trees for nm in _WALK_NAMES]
    words[:, 1:1 + len(_WALK_NAMES)] = np.array(flat, np.int64).reshape(len(trees), -1)
    C.memmove(arr, words.ctypes.data, words.nbytes)
    return arr


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _need(t, dtype, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: expected a contiguous CUDA tensor of {dtype}")
    return t


def distance_cuts(n_buckets: int, far: int, causal: bool = True) -> list:
    """Cuts between n_buckets buckets of distance (0 = the query's own place, negative = the past): about half of them
    one distance each, the others growing geometrically up to `far`; in both directions alike unless causal."""
    n = n_buckets - 1
    back = n if causal else (n + 1) // 2
    near = max(1, back // 2)
    steps = []
    for i in range(back):
        at = i if i < near else near * (far / near) ** ((i - near + 1) / (back - near))
        steps.append(max(int(round(at)), steps[-1] + 1) if steps else 0)
    return [-s for s in reversed(steps)] + [s + 1 for s in steps[:n - back]]


def rotation_turns(turned: int, base: float = 10_000.0, device="cuda") -> torch.Tensor:
    """What norm_rotate turns each pair of the first `turned` elements by, in revolutions per position: base ** (-2 i / turned) radians."""
    i = torch.arange(0, turned, 2, dtype=torch.float64)
    return (base ** (-i / max(1, turned)) / (2 * math.pi)).to(device)


def _rows_of(t, name, device, n=None, width=None):
    """The distance between rows of a tensor [n][width] whose last axis is contiguous."""
    if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype in DTYPES and t.dim() == 2 and n in (None, t.shape[0]) and width in (None, t.shape[1])):
        raise TypeError(f"{name}: expected a tensor [{'rows' if n is None else n}][{'width' if width is None else width}] of float32, bfloat16 or float16 on {device}")
    row, one = t.stride()
    if one != 1 and t.shape[1] > 1 and t.shape[0]:
        raise TypeError(f"{name}: expected a contiguous last axis")
    return row if t.shape[0] > 1 else t.shape[1]


def _heads(t, name, dtype, shape=None):
    """gbt_heads of a tensor [rows][heads][head_dim] (of that shape) whose last axis is contiguous."""
    n, h, d = shape or t.shape
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == (n, h, d)):
        raise TypeError(f"{name}: expected a CUDA tensor [{n}][{h}][{d}] of {dtype}")
    row, head, one = t.stride()
    if one != 1 and n and h and d > 1:
        raise TypeError(f"{name}: expected a contiguous last axis")
    return Heads(t.data_ptr(), row if n > 1 else h * d, head if h > 1 else d)     # an axis of one element has no stride to speak of


def _new_heads(like, shape):
    """A tensor of that shape, and its gbt_heads."""
    t = like.new_empty(shape)
    return t, Heads(t.data_ptr(), shape[1] * shape[2], shape[2])


class GradientList:
    """Tensors laid out for Context.clip_gradients; holds on to them, and to the memory that they had then."""

    def __init__(self, tensors, outs, table, pieces):
        self.tensors, self.outs, self.table, self.pieces = tensors, outs, table, pieces
        self.memory = [t.untyped_storage() for t in tensors + outs]     # the table's addresses, also of tensors that are given other memory later
        self.both = tensors + outs + [table]


class MatrixList:
    """Matrices laid out for Context.orthogonalise; holds on to them, and to the memory that they had then."""

    def __init__(self, tensors, outs, table, arr, bytes_needed):
        self.tensors, self.outs, self.table, self.arr, self.workspace_bytes = tensors, outs, table, arr, bytes_needed
        self.memory = [t.untyped_storage() for t in tensors + outs]
        self.all = tensors + outs + [table]


class Context:
    """One libgbt context bound to a device and to torch's current stream."""

    def __init__(self, device: int = 0, stream=None):
        self.lib = load()
        if not torch.cuda.is_available():
            raise RuntimeError("libgbt needs a GPU: no HIP device is visible")
        self.device = torch.device("cuda", device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        h = C.c_void_p()
        st = self.lib.gbt_create(C.byref(h), device, C.c_void_p(self.stream.cuda_stream))
        if st != OK:
            raise GbtError(st, "gbt_create failed (see stderr)")
        self.h = h
        self._ws = {}

    def close(self):
        if getattr(self, "h", None):
            self.lib.gbt_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers -----------------------------------------------------------
    def _check(self, st):
        if st != OK:
            raise GbtError(st, self.lib.gbt_last_error(self.h).decode())

    def workspace(self, key: str, nbytes: int) -> torch.Tensor:
        """A cached byte buffer of at least nbytes (device memory comes from torch)."""
        w = self._ws.get(key)
        if w is None or w.numel() < nbytes:
            self._ws.pop(key, None)
            w = torch.empty(max(int(nbytes), 4096), dtype=torch.uint8, device=self.device)
            self._ws[key] = w
        return w

    def empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    # -- measurement -----------------------------------------------------------
    def profile_enable(self, on: bool = True):
        self._check(self.lib.gbt_profile_enable(self.h, int(on)))

    def profile_read(self) -> dict:
        p = Profile()
        self._check(self.lib.gbt_profile_read(self.h, C.byref(p)))
        out = {nm: dict(ms=p.ms[i], bytes=p.bytes[i], alg_bytes=p.alg_bytes[i], launches=p.launches[i])
               for i, nm in enumerate(PROF_CLASSES)}
        self.last_profile_levels = [dict(level=k, ms=p.level_ms[k], alg_bytes=p.level_alg_bytes[k],
                                         row_features=p.level_row_features[k], launches=p.level_launches[k])
                                    for k in range(PROF_LEVELS) if p.level_launches[k]]
        return out

    def measure_stream_read(self, buf, reps: int = 5) -> float:
        """GB/s of a kernel that only reads `buf` (a device tensor), best of `reps` launches."""
        ws = self.workspace("small", 4096)
        out = C.c_double()
        self._check(self.lib.gbt_measure_stream_read(self.h, _ptr(buf), buf.numel() * buf.element_size(), reps,
                                                     C.byref(out), _ptr(ws), ws.numel()))
        return out.value

    # -- Sec. 2.1 ------------------------------------------------------------
    def quantise(self, X=None, csr=None, *, max_bins: int, n=None, F=None):
        """Returns (cuts [F][max_bins-1], nb [F], sym uint16 [n][F], max_value, missing_sym)."""
        if X is not None:
            _need(X, torch.float32, "X")
            n, F = X.shape
            n_values = n * F
            args = (_ptr(X), None, None, None)
        else:
            indptr, indices, values = csr
            _need(indptr, torch.int64, "indptr"); _need(indices, torch.int32, "indices")
            _need(values, torch.float32, "values")
            n_values = values.numel()
            args = (None, _ptr(indptr), _ptr(indices), _ptr(values))
        cuts = self.empty((F, max_bins - 1), torch.float32)
        nb = self.empty((F,), torch.int32)
        sym = self.empty((n, F), torch.uint16)
        ws_bytes = self.lib.gbt_quantise_workspace_bytes(n, F, n_values, max_bins)
        ws = self.workspace("quantise", ws_bytes)
        mv, ms = C.c_int32(), C.c_int32()
        self._check(self.lib.gbt_quantise(self.h, *args, n, F, max_bins, _ptr(cuts), _ptr(nb), _ptr(sym),
                                          C.byref(mv), C.byref(ms), _ptr(ws), ws.numel()))
        self._ws.pop("quantise", None)   # large and used once
        return cuts, nb, sym, mv.value, ms.value

    def quantise_packed(self, X=None, csr=None, *, max_bins: int, n=None, F=None):
        """Cuts and the packed matrix in one call (no symbol matrix in between).
        Returns (cuts [F][max_bins-1], nb [F], packed int32 words, bits, max_value, missing_sym)."""
        if X is not None:
            _need(X, torch.float32, "X")
            n, F = X.shape
            n_values = n * F
            args = (_ptr(X), None, None, None)
        else:
            indptr, indices, values = csr
            _need(indptr, torch.int64, "indptr"); _need(indices, torch.int32, "indices")
            _need(values, torch.float32, "values")
            n_values = values.numel()
            args = (None, _ptr(indptr), _ptr(indices), _ptr(values))
        cuts = self.empty((F, max_bins - 1), torch.float32)
        nb = self.empty((F,), torch.int32)
        cap = packed_words(n, F, bits_for(max_bins))      # no symbol exceeds max_bins
        packed = self.empty((cap,), torch.int32)
        ws_bytes = self.lib.gbt_quantise_workspace_bytes(n, F, n_values, max_bins)
        ws = self.workspace("quantise", ws_bytes)
        mv, ms, b = C.c_int32(), C.c_int32(), C.c_int32()
        self._check(self.lib.gbt_quantise_packed(self.h, *args, n, F, max_bins, _ptr(cuts), _ptr(nb), _ptr(packed),
                                                 C.c_int64(cap), C.byref(b), C.byref(mv), C.byref(ms), _ptr(ws),
                                                 ws.numel()))
        self._ws.pop("quantise", None)   # large and used once
        return cuts, nb, packed[:packed_words(n, F, b.value)], b.value, mv.value, ms.value

    # -- Sec. 2.2 ------------------------------------------------------------
    def compress(self, sym, max_value: int):
        _need(sym, torch.uint16, "sym")
        n, F = sym.shape
        bits = bits_for(max_value)
        packed = self.empty((packed_words(n, F, bits),), torch.int32)
        b = C.c_int32()
        self._check(self.lib.gbt_compress(self.h, _ptr(sym), n, F, max_value, _ptr(packed), C.byref(b)))
        return packed, b.value

    def compress_sparse(self, sym, max_bins: int, missing_sym: int):
        """Sparse rows of sym[n][F]: (rowptr uint32[n+1] as int32 tensor, ent[capacity], nnz); the entries are
        uint16 where F * max_bins <= 65536, else uint32."""
        _need(sym, torch.uint16, "sym")
        n, F = sym.shape
        rowptr = self.empty((n + 1,), torch.int32)
        ws_bytes = self.lib.gbt_compress_sparse_workspace_bytes(n)
        ws = self.workspace("small", max(ws_bytes, 4096))
        nnz = C.c_int64()
        self._check(self.lib.gbt_compress_sparse_count(self.h, _ptr(sym), n, F, missing_sym, _ptr(rowptr),
                                                       C.byref(nnz), _ptr(ws), ws.numel()))
        cap = int(self.lib.gbt_sparse_capacity(nnz.value))
        width = int(self.lib.gbt_sparse_entry_bytes(F, max_bins))
        if width == 0:
            raise GbtError(EUNSUPPORTED, f"gbt_sparse_entry_bytes rejected F = {F}, max_bins = {max_bins}")
        ent = self.empty((cap,), torch.uint16 if width == 2 else torch.uint32)
        self._check(self.lib.gbt_compress_sparse(self.h, _ptr(sym), n, F, max_bins, missing_sym, _ptr(rowptr),
                                                 nnz.value, _ptr(ent), cap))
        return rowptr, ent, nnz.value

    # -- Sec. 2.5 ------------------------------------------------------------
    def gradients(self, objective: str, margin, label, out=None):
        _need(margin, torch.float32, "margin"); _need(label, torch.float32, "label")
        n = margin.numel()
        gp = out if out is not None else self.empty((n, 2), torch.float32)
        self._check(self.lib.gbt_gradients(self.h, OBJECTIVES[objective], _ptr(margin), _ptr(label), n, _ptr(gp)))
        return gp

    # -- histograms ----------------------------------------------------------
    def gpair_fixed(self, gpair):
        _need(gpair, torch.float32, "gpair")
        n = gpair.shape[0]
        gq = self.empty((n, 2), torch.int32)
        scale = (C.c_double * 2)()
        ws = self.workspace("small", 4096)
        self._check(self.lib.gbt_gpair_fixed(self.h, _ptr(gpair), n, _ptr(gq), scale, _ptr(ws), ws.numel()))
        return gq, (scale[0], scale[1])

    def _rows_ptr(self, row_idx):
        # NULL means "all rows"; an empty list still needs a non-null address
        if row_idx is not None and row_idx.numel() == 0:
            return _ptr(self.workspace("small", 4096))
        return _ptr(row_idx)

    def sum_gpair(self, gq, row_idx=None):
        n_rows = gq.shape[0] if row_idx is None else row_idx.numel()
        out = (C.c_int64 * 2)()
        ws = self.workspace("small", 4096)
        self._check(self.lib.gbt_sum_gpair(self.h, _ptr(gq), self._rows_ptr(row_idx), n_rows, out, _ptr(ws),
                                           ws.numel()))
        return int(out[0]), int(out[1])

    def build_hist(self, packed, bits, n, F, B, missing_sym, gq, row_idx=None, out=None):
        hist = out if out is not None else self.empty((F, B, 2), torch.int64)
        n_rows = 0 if row_idx is None else row_idx.numel()
        self._check(self.lib.gbt_build_hist(self.h, _ptr(packed), bits, n, F, B, missing_sym,
                                            self._rows_ptr(row_idx), n_rows, _ptr(gq), _ptr(hist)))
        return hist

    def build_hist_sparse(self, rowptr, ent, n, F, B, gq, row_begin=0, n_rows=None, out=None):
        hist = out if out is not None else self.empty((F, B, 2), torch.int64)
        self._check(self.lib.gbt_build_hist_sparse(self.h, _ptr(rowptr), _ptr(ent), n, F, B, row_begin,
                                                   n if n_rows is None else n_rows, _ptr(gq), _ptr(hist)))
        return hist

    def hist_subtract(self, parent, child):
        out = torch.empty_like(parent)
        self._check(self.lib.gbt_hist_subtract(self.h, _ptr(parent), _ptr(child), _ptr(out), parent.numel()))
        return out

    def hist_export_f64(self, hist, scale):
        F, B, _ = hist.shape
        out = self.empty((F, B, 2), torch.float64)
        sc = (C.c_double * 2)(*scale)
        self._check(self.lib.gbt_hist_export_f64(self.h, _ptr(hist), F, B, sc, _ptr(out)))
        return out

    # -- split ---------------------------------------------------------------
    def eval_split(self, hist, nb, Gq, Hq, scale, params: Params) -> dict:
        F, B, _ = hist.shape
        sc = (C.c_double * 2)(*scale)
        sp = Split()
        ws = self.workspace("small", 4096)
        self._check(self.lib.gbt_eval_split(self.h, _ptr(hist), _ptr(nb), F, B, Gq, Hq, sc, C.byref(params),
                                            C.byref(sp), _ptr(ws), ws.numel()))
        return {k: getattr(sp, k) for k, _ in Split._fields_}

    # -- partition -----------------------------------------------------------
    def partition(self, packed, bits, n, F, row_idx, begin, end, feature, bin_, default_left, missing_sym) -> int:
        _need(row_idx, torch.int32, "row_idx")
        ws_bytes = self.lib.gbt_partition_workspace_bytes(end - begin)
        ws = self.workspace("partition", ws_bytes)
        nl = C.c_int64()
        self._check(self.lib.gbt_partition(self.h, _ptr(packed), bits, n, F, _ptr(row_idx), begin, end, feature,
                                           bin_, default_left, missing_sym, _ptr(ws), ws.numel(), C.byref(nl)))
        return nl.value

    def partition_static(self, packed, bits, n, F, row_idx, begin, end, feature, bin_, default_left, missing_sym) -> int:
        """gbt_partition_static: the same partition over the library's static scratch array (no workspace)."""
        _need(row_idx, torch.int32, "row_idx")
        nl = C.c_int64()
        self._check(self.lib.gbt_partition_static(self.h, _ptr(packed), bits, n, F, _ptr(row_idx), begin, end, feature,
                                                  bin_, default_left, missing_sym, C.byref(nl)))
        return nl.value

    # -- Alg. 1 --------------------------------------------------------------
    def grow_tree(self, packed, bits, n, F, missing_sym, nb, cuts, gpair, params: Params, want_leaf=True,
                  row_idx_out=None, leaf_out=None, want_rows=True):
        """Returns (tree dict of numpy arrays, row_idx int32 tensor [n], leaf_of_row int32 tensor [n]).
        want_rows=False: the final row order is not produced (row_idx is None), which lets the library
        take its faster partition paths; leaf_of_row is still available (want_leaf)."""
        t = new_tree(params.max_depth)
        ts = _tree_struct(t)
        if not want_rows:
            row_idx = None
        else:
            row_idx = row_idx_out if row_idx_out is not None else self.empty((n,), torch.int32)
        leaf = (leaf_out if leaf_out is not None else self.empty((n,), torch.int32)) if want_leaf else None
        ws_bytes = self.lib.gbt_grow_tree_workspace_bytes(n, F, bits, params.max_bins, params.max_depth)
        if ws_bytes == 0:
            raise GbtError(EINVAL, "gbt_grow_tree_workspace_bytes rejected the shape")
        ws = self.workspace("grow", ws_bytes)
        self._check(self.lib.gbt_grow_tree(self.h, _ptr(packed), bits, n, F, missing_sym, _ptr(nb), _ptr(cuts),
                                           _ptr(gpair), C.byref(params), C.byref(ts), _ptr(row_idx), _ptr(leaf),
                                           _ptr(ws), ws.numel()))
        t["n_nodes"] = int(ts.n_nodes)
        return t, row_idx, leaf

    def boost_round(self, packed, bits, n, F, missing_sym, nb, cuts, label, margin_in, margin_out, gpair, params: Params):
        """Gradients of margin_in, one depth-wise tree, margin_out = margin_in + eta * leaf weight.  Returns the tree."""
        for t_, nm in ((label, "label"), (margin_in, "margin_in"), (margin_out, "margin_out"), (gpair, "gpair")):
            _need(t_, torch.float32, nm)
        t = new_tree(params.max_depth)
        ts = _tree_struct(t)
        ws_bytes = self.lib.gbt_grow_tree_workspace_bytes(n, F, bits, params.max_bins, params.max_depth)
        if ws_bytes == 0:
            raise GbtError(EINVAL, "gbt_grow_tree_workspace_bytes rejected the shape")
        ws = self.workspace("grow", ws_bytes)
        self._check(self.lib.gbt_boost_round(self.h, _ptr(packed), bits, n, F, missing_sym, _ptr(nb), _ptr(cuts),
                                             _ptr(label), _ptr(margin_in), _ptr(margin_out), _ptr(gpair),
                                             C.byref(params), C.byref(ts), _ptr(ws), ws.numel()))
        t["n_nodes"] = int(ts.n_nodes)
        return t

    def grow_tree_sparse(self, rowptr, ent, n, nnz, F, nb, cuts, gpair, params: Params, want_leaf=True,
                         want_rows=True):
        """grow_tree over sparse rows (compress_sparse); returns what grow_tree returns."""
        t = new_tree(params.max_depth)
        ts = _tree_struct(t)
        row_idx = self.empty((n,), torch.int32) if want_rows else None
        leaf = self.empty((n,), torch.int32) if want_leaf else None
        ws_bytes = self.lib.gbt_grow_tree_sparse_workspace_bytes(n, nnz, F, params.max_bins, params.max_depth)
        if ws_bytes == 0:
            raise GbtError(EINVAL, "gbt_grow_tree_sparse_workspace_bytes rejected the shape")
        ws = self.workspace("grow", ws_bytes)
        self._check(self.lib.gbt_grow_tree_sparse(self.h, _ptr(rowptr), _ptr(ent), n, nnz, F, _ptr(nb), _ptr(cuts),
                                                  _ptr(gpair), C.byref(params), C.byref(ts), _ptr(row_idx),
                                                  _ptr(leaf), _ptr(ws), ws.numel()))
        t["n_nodes"] = int(ts.n_nodes)
        return t, row_idx, leaf

    def grow_tree_sparse_lossguide(self, rowptr, ent, n, nnz, F, nb, cuts, gpair, params: Params, max_leaves,
                                   want_leaf=True, want_rows=True):
        """Loss-guided growth (Sec. 2.3) over sparse rows; returns what grow_tree returns."""
        t = new_tree_leaves(max_leaves)
        ts = _tree_struct(t)
        row_idx = self.empty((n,), torch.int32) if want_rows else None
        leaf = self.empty((n,), torch.int32) if want_leaf else None
        ws_bytes = self.lib.gbt_grow_tree_sparse_lossguide_workspace_bytes(n, nnz, F, params.max_bins, max_leaves)
        if ws_bytes == 0:
            raise GbtError(EINVAL, "gbt_grow_tree_sparse_lossguide_workspace_bytes rejected the shape")
        ws = self.workspace("grow", ws_bytes)
        self._check(self.lib.gbt_grow_tree_sparse_lossguide(self.h, _ptr(rowptr), _ptr(ent), n, nnz, F, _ptr(nb),
                                                            _ptr(cuts), _ptr(gpair), C.byref(params), max_leaves,
                                                            C.byref(ts), _ptr(row_idx), _ptr(leaf), _ptr(ws), ws.numel()))
        t["n_nodes"] = int(ts.n_nodes)
        return t, row_idx, leaf

    def grow_tree_lossguide(self, packed, bits, n, F, missing_sym, nb, cuts, gpair, params: Params, max_leaves,
                            want_leaf=True, want_rows=True):
        """Loss-guided growth (Sec. 2.3); returns what grow_tree returns."""
        t = new_tree_leaves(max_leaves)
        ts = _tree_struct(t)
        row_idx = self.empty((n,), torch.int32) if want_rows else None
        leaf = self.empty((n,), torch.int32) if want_leaf else None
        ws_bytes = self.lib.gbt_grow_tree_lossguide_workspace_bytes(n, F, bits, params.max_bins, max_leaves)
        if ws_bytes == 0:
            raise GbtError(EINVAL, "gbt_grow_tree_lossguide_workspace_bytes rejected the shape")
        ws = self.workspace("grow", ws_bytes)
        self._check(self.lib.gbt_grow_tree_lossguide(self.h, _ptr(packed), bits, n, F, missing_sym, _ptr(nb),
                                                     _ptr(cuts), _ptr(gpair), C.byref(params), max_leaves,
                                                     C.byref(ts), _ptr(row_idx), _ptr(leaf), _ptr(ws), ws.numel()))
        t["n_nodes"] = int(ts.n_nodes)
        return t, row_idx, leaf

    def grow_tree_path(self, F, bits, max_bins, track_rows=True):
        """0: three-launch partition, 1: one-launch partition, 2: partition + histogram in one launch."""
        r = self.lib.gbt_grow_tree_path(self.h, F, bits, max_bins, 1 if track_rows else 0)
        if r < 0:
            self._check(r)
        return r

    def grow_tree_form(self, n, F, bits, max_bins, max_depth, track_rows=True):
        """(path, planned): what depth-wise growth of n rows takes, and whether its levels are planned on the device."""
        r = self.lib.gbt_grow_tree_form(self.h, n, F, bits, max_bins, max_depth, 1 if track_rows else 0)
        if r < 0:
            self._check(r)
        return r % GROW_PLANNED, r >= GROW_PLANNED

    # -- Sec. 2.4 ------------------------------------------------------------
    def predict_sparse(self, trees, margin, eta: float, rowptr, ent, n, F, max_bins):
        arr = _tree_table(trees)
        ws_bytes = self.lib.gbt_predict_workspace_bytes(arr, len(trees))
        ws = self.workspace("predict", ws_bytes)
        self._check(self.lib.gbt_predict_sparse(self.h, arr, len(trees), _ptr(rowptr), _ptr(ent), n, F, max_bins, eta,
                                                _ptr(margin), _ptr(ws), ws.numel()))
        return margin

    def predict(self, trees, margin, eta: float, *, packed=None, bits=0, missing_sym=0, X=None, n=None, F=None):
        arr = _tree_table(trees)
        if X is not None:
            n, F = X.shape
        ws_bytes = self.lib.gbt_predict_workspace_bytes(arr, len(trees))
        ws = self.workspace("predict", ws_bytes)
        self._check(self.lib.gbt_predict(self.h, arr, len(trees), _ptr(packed), bits, missing_sym, _ptr(X), n, F,
                                         eta, _ptr(margin), _ptr(ws), ws.numel()))
        return margin

    # -- rows with a history ---------------------------------------------------
    def _on_stream(self, tensors=()):
        """None where the context's stream is torch's current one.  Else outputs are to be allocated on it, within the manager returned, and
        the inputs' memory is kept from reuse until this call's work is done (waiting for their contents is the caller's, as for every
        call)."""
        if torch._C._cuda_getCurrentRawStream(self.device.index) == self.stream.cuda_stream:
            return None
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)
        return torch.cuda.stream(self.stream)

    def _scratch(self, key, nbytes):
        """The workspace of that name.  A graph that is being recorded gets memory of its own: the workspace is given back when a larger
        one takes its place, and replays would go on writing there."""
        if torch.cuda.is_current_stream_capturing():
            return self.empty((max(nbytes, 16),), torch.uint8)
        return self.workspace(key, nbytes)

    def _longest(self, q_ptr, k_ptr, k_len):
        """The most rows that a sequence has by the pointers given, read from the device; None while a graph is being recorded, when nothing can
        be read."""
        if torch.cuda.is_current_stream_capturing():
            return None
        with torch.cuda.stream(self.stream):
            most = []
            for ptr, used in ((q_ptr, None), (k_ptr, k_len)):
                if ptr is not False and not (most and ptr is q_ptr and used is None):
                    lengths = ptr[1:] - ptr[:-1]
                    most.append((lengths if used is None else torch.minimum(lengths, used)).max())
            most = [max(0, x) for x in torch.stack(most).tolist()]       # one wait for both
        return most[0], most[-1]

    def _attention_params(self, q, k, q_ptr, k_ptr, k_len, max_q, max_k, causal, scale, bias, cuts):
        """(gbt_attention_params, what it points to on the host)."""
        if not (isinstance(q, torch.Tensor) and q.dim() == 3 and isinstance(k, torch.Tensor) and k.dim() == 3):
            raise TypeError("q, k: expected tensors [rows][heads][head_dim]")
        rows, heads, dim = q.shape
        k_rows, kv_heads, _ = k.shape
        if not (q.is_cuda and k.is_cuda):
            raise TypeError("q, k: expected CUDA tensors")
        n_q = n_k = n_len = at_q = at_k = at_len = None
        if q_ptr is not None:
            n_q, at_q = _need(q_ptr, torch.int64, "q_ptr").numel() - 1, q_ptr.data_ptr()
        if k_ptr is not None:
            n_k, at_k = (n_q, at_q) if k_ptr is q_ptr else (_need(k_ptr, torch.int64, "k_ptr").numel() - 1, k_ptr.data_ptr())
        if k_len is not None:
            n_len, at_len = _need(k_len, torch.int32, "k_len").numel(), k_len.data_ptr()
        n_seq = n_q if n_q is not None else n_k if n_k is not None else 1 if n_len is None else n_len
        if (n_k is not None and n_k != n_seq) or (n_len is not None and n_len != n_seq):
            raise TypeError("q_ptr, k_ptr and k_len do not describe the same number of sequences")
        if q_ptr is None:
            each = rows // max(1, n_seq)
            if each * n_seq != rows or max_q not in (None, each):
                raise TypeError(f"q: without q_ptr all of {n_seq} sequences have the same length")
            max_q = each
        if k_ptr is None:
            each = k_rows // max(1, n_seq)
            if each * n_seq != k_rows or max_k not in (None, each):
                raise TypeError(f"k: without k_ptr all of {n_seq} sequences have the same length")
            max_k = each
        if max_q is None or max_k is None:
            longest = self._longest(max_q is None and q_ptr, max_k is None and k_ptr, k_len) if n_seq > 1 else None
            of_q, of_k = longest or (rows, k_rows)
            max_q, max_k = min(rows, of_q) if max_q is None else max_q, min(k_rows, of_k) if max_k is None else max_k
        n_buckets, table, edges = 0, None, None
        if bias is not None:
            _need(bias, torch.float32, "bias")
            shape = bias.shape
            if len(shape) != 2 or shape[1] != heads or shape[0] < 1:
                raise TypeError(f"bias: expected [n_buckets][{heads}], not {tuple(shape)}")
            n_buckets, table = shape[0], bias.data_ptr()
            if cuts is None or len(cuts) != n_buckets - 1:
                raise TypeError(f"cuts: expected {n_buckets - 1} of them")
            edges = array.array("i", cuts if type(cuts) is list else cuts.tolist() if hasattr(cuts, "tolist") else cuts)
        p = AttentionParams(DTYPES.get(q.dtype, -1), heads, kv_heads, dim, n_seq, max_q, max_k, causal,
                            n_buckets, dim ** -0.5 if scale is None else scale, rows, k_rows, at_q, at_k, at_len, table,
                            None if edges is None else edges.buffer_info()[0])
        return p, edges

    def attention(self, q, k, v, *, q_ptr=None, k_ptr=None, k_len=None, max_q=None, max_k=None, causal=False, scale=None,
                  bias=None, cuts=None, save=False, out=None):
        """Attention of q [rows][heads][head_dim] over k, v [rows][kv_heads][head_dim], sequence by sequence.

        q_ptr, k_ptr  int64[n_seq + 1] on the device: where each sequence's rows begin (None: sequences of one length)
        k_len         int32[n_seq] on the device: how many rows of each slot of k and v are in use (None: all)
        max_q, max_k  the longest sequence.  None: read from the pointers, which waits for the device (some 30 us a call); in a graph that is being
                      recorded, all rows, which costs idle workgroups and is refused for many sequences
        bias, cuts    float32 [n_buckets][heads] and the ascending cuts between buckets of distance, on the host
        Rows of no sequence, and queries without keys, get zeros; a bias below GBT_BIAS_SHUT (-1e5) shuts its bucket out.
        save          also return what attention_backward needs: (out, saved)
        No graph of derivatives is recorded, whether or not the inputs require gradients: attention_backward is the gradient.
        """
        p, edges = self._attention_params(q, k, q_ptr, k_ptr, k_len, max_q, max_k, causal, scale, bias, cuts)
        dtype = q.dtype
        of_q = rows, heads, dim = q.shape
        of_k = p.k_rows, p.kv_heads, dim
        hq, hk, hv = _heads(q, "q", dtype, of_q), _heads(k, "k", dtype, of_k), _heads(v, "v", dtype, of_k)
        lib, at = self.lib, C.byref(p)
        ws_bytes = lib.gbt_attention_workspace_bytes(at)
        lse = rest = None
        with self._on_stream((q, k, v, q_ptr, k_ptr, k_len, bias, out)) or _NO_STREAM:
            if out is None:
                out = q.new_empty(rows, heads, dim)
            if save:
                lse, rest = q.new_empty((heads, rows), dtype=torch.float32), q.new_empty(rows, heads, dim)
            ws = self._scratch("attention", ws_bytes) if ws_bytes else None
        ho = _heads(out, "out", dtype, of_q)
        st = lib.gbt_attention(self.h, at, C.byref(hq), C.byref(hk), C.byref(hv), C.byref(ho), lse.data_ptr() if save else None,
                               rest.data_ptr() if save else None, ws.data_ptr() if ws_bytes else None, ws_bytes)
        if st:
            self._check(st)
        return (out, (lse, rest)) if save else out

    def attention_backward(self, dout, q, k, v, out, saved, *, q_ptr=None, k_ptr=None, k_len=None, max_q=None, max_k=None, causal=False,
                           scale=None, bias=None, cuts=None):
        """(dq, dk, dv, dbias) of attention(..., save=True) with the same arguments; dbias is None without a bias.  Rows of no
        sequence get zeros, rows beyond k_len too."""
        p, edges = self._attention_params(q, k, q_ptr, k_ptr, k_len, max_q, max_k, causal, scale, bias, cuts)
        dtype = q.dtype
        of_q = rows, heads, dim = q.shape
        of_k = k_rows, kv_heads, dim = p.k_rows, p.kv_heads, dim
        lse, rest = saved
        _need(lse, torch.float32, "saved[0]")
        if rest is not None:
            _need(rest, dtype, "saved[1]")
        if lse.shape != (heads, rows) or (rest is not None and rest.shape != of_q):
            raise TypeError(f"saved: not of a call with q of {tuple(q.shape)}")
        hg, hq, ho = _heads(dout, "dout", dtype, of_q), _heads(q, "q", dtype, of_q), _heads(out, "out", dtype, of_q)
        hk, hv = _heads(k, "k", dtype, of_k), _heads(v, "v", dtype, of_k)
        lib, at = self.lib, C.byref(p)
        ws_bytes = lib.gbt_attention_backward_workspace_bytes(at)
        with self._on_stream((dout, q, k, v, out, lse, rest, q_ptr, k_ptr, k_len, bias)) or _NO_STREAM:
            dq, dk, dv = q.new_empty(rows, heads, dim), q.new_empty(k_rows, kv_heads, dim), q.new_empty(k_rows, kv_heads, dim)
            dbias = None if bias is None else torch.empty_like(bias)
            ws = self._scratch("attention", ws_bytes)
        hdq, hdk, hdv = Heads(dq.data_ptr(), heads * dim, dim), Heads(dk.data_ptr(), kv_heads * dim, dim), Heads(dv.data_ptr(), kv_heads * dim, dim)
        st = lib.gbt_attention_backward(self.h, at, C.byref(hg), C.byref(hq), C.byref(hk), C.byref(hv), C.byref(ho), lse.data_ptr(),
                                        None if rest is None else rest.data_ptr(), C.byref(hdq), C.byref(hdk), C.byref(hdv),
                                        None if dbias is None else dbias.data_ptr(), ws.data_ptr(), ws.numel())
        if st:
            self._check(st)
        return dq, dk, dv, dbias

    def gradient_list(self, tensors, outs=None) -> GradientList:
        """Lays gradient tensors out for clip_gradients; outs receive the results (None: the tensors themselves).  Good for as long
        as the tensors stay where they are: the list holds on to the memory that they have now and goes on with it, also where a tensor is
        given other memory or another takes its place.  Gradients that are allocated anew each step need a list each step.  Refused while a
        graph is being recorded on the context's stream: lists are laid out before."""
        tensors = list(tensors)
        outs = tensors if outs is None else list(outs)
        if len(outs) != len(tensors):
            raise TypeError("outs: expected one for each tensor")
        arr = (Gradient * max(1, len(tensors)))()
        for i, (t, o) in enumerate(zip(tensors, outs)):
            if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype in DTYPES):
                raise TypeError(f"tensors[{i}]: expected a contiguous CUDA tensor of float32, bfloat16 or float16")
            _need(o, t.dtype, f"outs[{i}]")
            if o.numel() != t.numel():
                raise TypeError(f"outs[{i}]: expected {t.numel()} elements")
            arr[i] = Gradient(t.data_ptr(), o.data_ptr(), t.numel(), DTYPES[t.dtype])
        nbytes = self.lib.gbt_gradient_list_bytes(arr, len(tensors))
        with self._on_stream() or _NO_STREAM:
            table = self.empty((max(16, nbytes),), torch.uint8)
        pieces = C.c_int32()
        self._check(self.lib.gbt_gradient_list(self.h, arr, len(tensors), _ptr(table), table.numel(), C.byref(pieces)))
        return GradientList(tensors, outs, table, pieces.value)

    def clip_gradients(self, gradients: GradientList, max_norm: float):
        """Scales every tensor of the list by min(1, max_norm / (norm + 1e-6)) into its out; returns the global norm, a float32 scalar
        on the device.  A norm that is not finite leaves the values as they are."""
        with self._on_stream(gradients.both) or _NO_STREAM:
            norm = gradients.table.new_empty((), dtype=torch.float32)
            ws = self._scratch("clip", 16384)
        st = self.lib.gbt_clip_gradients(self.h, gradients.table.data_ptr(), gradients.pieces, max_norm, norm.data_ptr(), ws.data_ptr(), ws.numel())
        if st:
            self._check(st)
        return norm

    # -- around a tower over histories ---------------------------------------------
    def _embedding_params(self, ids, n_rows, table_dtype, out_dtype, width, table_stride, out_stride, scale):
        if not (isinstance(ids, torch.Tensor) and ids.device == self.device and ids.dtype in (torch.int32, torch.int64) and ids.is_contiguous()):
            raise TypeError(f"ids: expected a contiguous tensor of int32 or int64 on {self.device}")
        return EmbeddingParams(DTYPES[table_dtype], DTYPES[out_dtype], ids.element_size(), width, ids.numel(), n_rows, table_stride, out_stride,
                               ids.data_ptr(), scale)

    def embedding(self, table, ids, *, scale=1.0, dtype=None, out=None):
        """Rows of table [rows][width] by ids of any shape, times scale: [*ids.shape][width] of `dtype` (None: the table's).  An id
        outside the table gives zeros, a padding id of -1 for instance.

        out           [ids][width], rows any distance apart, apart from table and ids: written to, and returned
        No graph of derivatives is recorded: embedding_backward is the table's gradient.
        """
        stride = _rows_of(table, "table", self.device)
        n_rows, width = table.shape
        if out is not None:
            of_out = _rows_of(out, "out", self.device, ids.numel() if isinstance(ids, torch.Tensor) else None, width)
            if dtype not in (None, out.dtype):
                raise TypeError(f"out: expected {dtype}")
            dtype = out.dtype
        else:
            of_out, dtype = width, table.dtype if dtype is None else dtype
        if dtype not in DTYPES:
            raise TypeError("dtype: expected float32, bfloat16 or float16")
        p = self._embedding_params(ids, n_rows, table.dtype, dtype, width, stride, of_out, scale)
        if out is None:
            with self._on_stream((table, ids)) or _NO_STREAM:
                out = table.new_empty((*ids.shape, width), dtype=dtype)
        else:
            self._on_stream((table, ids, out))
        st = self.lib.gbt_embedding(self.h, C.byref(p), table.data_ptr(), out.data_ptr())
        if st:
            self._check(st)
        return out

    def embedding_backward(self, dout, ids, rows=None, *, scale=1.0, dtype=torch.float32, out=None, accumulate=False):
        """The gradient [rows][width] of embedding's table, of `dtype`, from that of its result [*ids.shape][width]: for each row the sum over
        the places that hold its id, in 32 bits and a fixed order, times scale; zeros for rows without one.  The gradient's rows may be any
        distance apart, or all the same; a row's elements lie side by side (one expanded along its last axis is refused: .contiguous()).

        out           [rows][width], rows any distance apart, apart from dout and ids: written to, and returned
        accumulate    add to what `out` holds
        """
        if not (isinstance(dout, torch.Tensor) and isinstance(ids, torch.Tensor) and dout.dim() >= 1 and dout.shape[:-1] in (ids.shape, (ids.numel(),))):
            raise TypeError("dout: expected a tensor [*ids.shape][width]")
        width = dout.shape[-1]
        if dout.dim() != 2:
            with self._on_stream((dout,)) or _NO_STREAM:   # it may be a copy
                dout = dout.reshape(ids.numel(), width)
        of_out = _rows_of(dout, "dout", self.device)
        if out is not None:
            stride = _rows_of(out, "out", self.device, rows, width)
            rows, dtype = out.shape[0], out.dtype
        elif accumulate or rows is None:
            raise TypeError("out: expected a tensor to add to" if accumulate else "rows: expected the number of the table's rows")
        else:
            stride = width
        if dtype not in DTYPES:
            raise TypeError("dtype: expected float32, bfloat16 or float16")
        p = self._embedding_params(ids, rows, dtype, dout.dtype, width, stride, of_out, scale)
        ws_bytes = self.lib.gbt_embedding_backward_workspace_bytes(C.byref(p))
        with self._on_stream((dout, ids, out)) or _NO_STREAM:
            if out is None:
                out = dout.new_empty((rows, width), dtype=dtype)
            ws = self._scratch("embedding", ws_bytes) if ws_bytes else None
        st = self.lib.gbt_embedding_backward(self.h, C.byref(p), dout.data_ptr(), out.data_ptr(), bool(accumulate), ws.data_ptr() if ws_bytes else None, ws_bytes)
        if st:
            self._check(st)
        return out

    def _norm_rotate_params(self, q, k, q_weight, k_weight, turns, q_ptr, k_ptr, k_len, positions, eps, halves, store_rows):
        if not (isinstance(q, torch.Tensor) and q.dim() == 3 and isinstance(k, torch.Tensor) and k.dim() == 3 and q.device == self.device):
            raise TypeError(f"q, k: expected tensors [rows][heads][head_dim] on {self.device}")
        rows, heads, dim = q.shape
        counts = []
        if q_ptr is not None:
            counts.append(_need(q_ptr, torch.int64, "q_ptr").numel() - 1)
        if k_ptr is not None:
            counts.append(_need(k_ptr, torch.int64, "k_ptr").numel() - 1)
        if k_len is not None:
            counts.append(_need(k_len, torch.int32, "k_len").numel())
        n_seq = counts[0] if counts else 1
        if len(counts) > 1 and any(n != n_seq for n in counts):
            raise TypeError("q_ptr, k_ptr and k_len do not describe the same number of sequences")
        if q_ptr is None and n_seq > 0 and rows % n_seq:
            raise TypeError(f"q: without q_ptr all of {n_seq} sequences have the same length")
        if store_rows is not None and k_ptr is None and n_seq > 0 and store_rows % n_seq:
            raise TypeError(f"k_out: without k_ptr all of {n_seq} slots have the same length")
        if q_weight is not None and _need(q_weight, torch.float32, "q_weight").shape != (dim,) or \
                k_weight is not None and _need(k_weight, torch.float32, "k_weight").shape != (dim,):
            raise TypeError(f"q_weight, k_weight: expected [{dim}]")
        turned = 0
        if turns is not None:
            if _need(turns, torch.float64, "turns").dim() != 1:
                raise TypeError("turns: expected [turned / 2]")
            turned = 2 * turns.numel()
        wide = 4
        if positions is not None:
            if positions.dtype is not torch.int32:
                _need(positions, torch.int64, "positions")
                wide = 8
            if _need(positions, positions.dtype, "positions").shape != (rows,):
                raise TypeError(f"positions: expected [{rows}]")
        return NormRotateParams(DTYPES.get(q.dtype, -1), heads, k.shape[1], dim, turned, bool(halves), store_rows is not None, n_seq, wide, eps, rows,
                                rows if store_rows is None else store_rows,
                                *[None if x is None else x.data_ptr() for x in (q_ptr, k_ptr, k_len, positions, q_weight, k_weight, turns)])

    def norm_rotate(self, q, k, q_weight, k_weight, turns, *, v=None, q_ptr=None, k_ptr=None, k_len=None, positions=None, eps=1e-6, halves=True,
                    q_out=None, k_out=None, v_out=None):
        """Every head of q [rows][heads][head_dim] and k [rows][kv_heads][head_dim] divided by its root mean square (of its elements; eps is added
        to the mean), times a weight float32 [head_dim] (None: ones), its pairs turned by position * turns revolutions (float64 [turned / 2],
        rotation_turns; None: not turned).  Returns (q_out, k_out), and v_out with v.

        q_ptr, k_ptr, k_len   the rows of sequences, as for attention: row i of nq has place i + nk - nq, and nk is nq without k_ptr and k_len
        positions     int32 or int64 [rows] on the device (None: the places)
        halves        a pair is elements i and i + turned / 2; else 2 i and 2 i + 1
        k_out, v_out  with k_ptr or k_len: stores, in which a row's keys and values (v, as they are) go to the place in its sequence's slot;
                      nothing else there is touched
        Outputs may be the inputs themselves.  Rows of no sequence get zeros, except in stores.
        No graph of derivatives is recorded: norm_rotate_backward is the gradient.
        """
        if (v is None) != (v_out is None) and (v is None or k_out is not None):
            raise TypeError("v, v_out: one without the other")
        store = k_out is not None and (k_ptr is not None or k_len is not None)
        if store and not (isinstance(k_out, torch.Tensor) and k_out.dim() == 3):
            raise TypeError("k_out: expected a tensor [rows][kv_heads][head_dim]")
        p = self._norm_rotate_params(q, k, q_weight, k_weight, turns, q_ptr, k_ptr, k_len, positions, eps, halves, k_out.shape[0] if store else None)
        dtype = q.dtype
        of_q = rows, heads, dim = q.shape
        of_k, of_out = (rows, p.kv_heads, dim), (p.out_rows, p.kv_heads, dim)
        hq, hk = _heads(q, "q", dtype, of_q), _heads(k, "k", dtype, of_k)
        hv = None if v is None else _heads(v, "v", dtype, of_k)
        with self._on_stream((q, k, v, q_weight, k_weight, turns, q_ptr, k_ptr, k_len, positions, q_out, k_out, v_out)) or _NO_STREAM:
            q_out, hq_out = _new_heads(q, of_q) if q_out is None else (q_out, _heads(q_out, "q_out", dtype, of_q))
            k_out, hk_out = _new_heads(q, of_k) if k_out is None else (k_out, _heads(k_out, "k_out", dtype, of_out))
            if v is not None:
                v_out, hv_out = _new_heads(q, of_k) if v_out is None else (v_out, _heads(v_out, "v_out", dtype, of_out))
        if v is None:
            st = self.lib.gbt_norm_rotate(self.h, C.byref(p), C.byref(hq), C.byref(hk), None, C.byref(hq_out), C.byref(hk_out), None)
        else:
            st = self.lib.gbt_norm_rotate(self.h, C.byref(p), C.byref(hq), C.byref(hk), C.byref(hv), C.byref(hq_out), C.byref(hk_out), C.byref(hv_out))
        if st:
            self._check(st)
        return (q_out, k_out) if v is None else (q_out, k_out, v_out)

    def norm_rotate_backward(self, dq_out, dk_out, q, k, q_weight, k_weight, turns, *, q_ptr=None, k_ptr=None, k_len=None, positions=None, eps=1e-6,
                             halves=True, dq=None, dk=None):
        """(dq, dk, dq_weight, dk_weight) of norm_rotate with the same arguments and packed outputs, from the gradients of q_out and k_out.  dq and
        dk: written to where given (parts of one tensor for the projection's gradient, say; or dq_out and dk_out themselves).  Rows of no
        sequence get zeros."""
        p = self._norm_rotate_params(q, k, q_weight, k_weight, turns, q_ptr, k_ptr, k_len, positions, eps, halves, None)
        dtype = q.dtype
        of_q = rows, heads, dim = q.shape
        of_k = rows, p.kv_heads, dim
        hq, hk = _heads(q, "q", dtype, of_q), _heads(k, "k", dtype, of_k)
        hdq_out, hdk_out = _heads(dq_out, "dq_out", dtype, of_q), _heads(dk_out, "dk_out", dtype, of_k)
        ws_bytes = self.lib.gbt_norm_rotate_backward_workspace_bytes(C.byref(p))
        with self._on_stream((dq_out, dk_out, q, k, q_weight, k_weight, turns, q_ptr, k_ptr, k_len, positions, dq, dk)) or _NO_STREAM:
            dq, hdq = _new_heads(q, of_q) if dq is None else (dq, _heads(dq, "dq", dtype, of_q))
            dk, hdk = _new_heads(q, of_k) if dk is None else (dk, _heads(dk, "dk", dtype, of_k))
            weights = q.new_empty((2, dim), dtype=torch.float32)
            ws = self._scratch("norm_rotate", ws_bytes)
        of_weights = weights.data_ptr()
        st = self.lib.gbt_norm_rotate_backward(self.h, C.byref(p), C.byref(hdq_out), C.byref(hdk_out), C.byref(hq), C.byref(hk), C.byref(hdq), C.byref(hdk),
                                               of_weights, of_weights + 4 * dim, ws.data_ptr(), ws_bytes)
        if st:
            self._check(st)
        return (dq, dk, *weights.unbind(0))

    def matrix_list(self, tensors, outs=None, *, scales=1.0) -> MatrixList:
        """Lays matrices [rows][cols] out for orthogonalise; outs receive the results (None: the tensors themselves), times scales (one for
        each, or one for all).  Good for as long as the tensors stay where they are, as a gradient_list is.  No out may share memory with another matrix, nor
        with part of its own.  Refused while a graph is being recorded on the context's stream."""
        tensors = list(tensors)
        outs = tensors if outs is None else list(outs)
        scales = [float(scales)] * len(tensors) if isinstance(scales, (int, float)) else [float(x) for x in scales]
        if len(outs) != len(tensors) or len(scales) != len(tensors):
            raise TypeError("outs, scales: expected one for each tensor")
        arr = (Matrix * max(1, len(tensors)))()
        for i, (t, o, scale) in enumerate(zip(tensors, outs, scales)):
            if not (isinstance(t, torch.Tensor) and t.device == self.device and t.dim() == 2 and t.is_contiguous() and t.dtype in DTYPES):
                raise TypeError(f"tensors[{i}]: expected a contiguous tensor [rows][cols] of float32, bfloat16 or float16 on {self.device}")
            if _need(o, t.dtype, f"outs[{i}]").shape != t.shape:
                raise TypeError(f"outs[{i}]: expected {tuple(t.shape)}")
            arr[i] = Matrix(t.data_ptr(), o.data_ptr(), *t.shape, DTYPES[t.dtype], scale)
        nbytes = self.lib.gbt_matrix_list_bytes(arr, len(tensors))
        with self._on_stream() or _NO_STREAM:
            table = self.empty((max(16, nbytes),), torch.uint8)
        self._check(self.lib.gbt_matrix_list(self.h, arr, len(tensors), _ptr(table), table.numel()))
        return MatrixList(tensors, outs, table, arr, self.lib.gbt_orthogonalise_workspace_bytes(arr, len(tensors)))

    def orthogonalise(self, matrices: MatrixList, *, steps=5, coefficients=(3.4445, -4.7750, 2.0315)):
        """Every matrix of the list divided by its norm, then `steps` times X <- (a I + b A + c A^2) X with A = X X^T, times its scale, into its
        out: all singular values end near one.  The same coefficients in all steps, under which no singular value passes 4, nor its factor 64.  A matrix of zeros gives zeros, one that is not finite NaN.  Returns the outs."""
        a, b, c = coefficients
        with self._on_stream(matrices.all) or _NO_STREAM:
            ws = self._scratch("orthogonalise", matrices.workspace_bytes)
        st = self.lib.gbt_orthogonalise(self.h, matrices.table.data_ptr(), matrices.arr, len(matrices.tensors), steps, a, b, c, ws.data_ptr(), ws.numel())
        if st:
            self._check(st)
        return matrices.outs
