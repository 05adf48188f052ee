"""Binding of libkvcomm.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/kvcomm.h) and does
nothing but turn torch tensors into (pointer, strides) descriptors, allocate outputs that
the caller did not pass, and raise on a non-zero status.  All arithmetic of the reuse step
runs inside the library's HIP kernels.  torch is used for device memory and streams only.

Calls whose arguments are plain (device tensors, lists, numbers) are marshalled by the native module _marshal
(csrc/marshal.cpp), which declines all others; those take the ctypes code below, which converts or refuses them.  Without
a _marshal built for this torch and Python every call does (a warning says so: small calls then take longer on the host).
"""
import contextlib
import ctypes
import os
import sys
import warnings
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# KVCOMM_LIBRARY selects another build of the same library (e.g. a tuning variant); default: the in-tree build
_LIB_PATH = os.environ.get("KVCOMM_LIBRARY") or os.path.join(_HERE, "libkvcomm.so")

W_TOKEN = 0
W_LAYER_HEAD_TOKEN = 1
W_SEGMENT = 2
MAX_ANCHORS = 64
MAX_BATCH = 8
MAX_ROTATIONS = MAX_ANCHORS + 1   # of all segments of a batched update
COMPUTE_UNITS = 256
ATTN_MIN_SPLIT_KEYS = 512   # shorter caches never use the attention's scratch
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3   # statuses of a call that has launched nothing
RULE_L2_SOFTMAX = 0
RULE_NEAREST = 1
RULE_COSINE_SOFTMAX = 2

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class KVCommError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"libkvcomm: {message} (status {status})")
        self.status = status


class _CModel(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rope_theta", ctypes.c_double)]


class _CTensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_layer", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_token", ctypes.c_int64)]


class _CTensor4(ctypes.Structure):
    _fields_ = [("codes", _CTensor), ("scales", _CTensor)]


class _CPages(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("stride_layer", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_page", ctypes.c_int64), ("stride_token", ctypes.c_int64)]


class _CBatch(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("table_width", ctypes.c_int32), ("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("max_rows", ctypes.c_int32)]


class _CAlignJob(ctypes.Structure):
    _fields_ = [("base_k", _CTensor), ("base_v", _CTensor), ("out_k", _CTensor), ("out_v", _CTensor),
                ("seg_len", ctypes.c_int32), ("delta_pos", ctypes.c_int32),
                ("anchor_dk", ctypes.POINTER(ctypes.c_void_p)), ("anchor_dv", ctypes.POINTER(ctypes.c_void_p)),
                ("anchor_len", ctypes.POINTER(ctypes.c_int32)), ("anchor_delta_pos", ctypes.POINTER(ctypes.c_int32)),
                ("n_anchors", ctypes.c_int32), ("weights", ctypes.c_void_p), ("weights_slots", ctypes.c_int64)]


class _CAlignQ8Job(ctypes.Structure):
    _fields_ = [("base_k", _CTensor), ("base_v", _CTensor), ("out_k", _CTensor), ("out_v", _CTensor),
                ("seg_len", ctypes.c_int32), ("delta_pos", ctypes.c_int32),
                ("anchor_dk", ctypes.POINTER(ctypes.c_void_p)), ("anchor_dv", ctypes.POINTER(ctypes.c_void_p)),
                ("anchor_len", ctypes.POINTER(ctypes.c_int32)), ("anchor_delta_pos", ctypes.POINTER(ctypes.c_int32)),
                ("anchor_scale_k", ctypes.POINTER(ctypes.c_float)), ("anchor_scale_v", ctypes.POINTER(ctypes.c_float)),
                ("n_anchors", ctypes.c_int32), ("weights", ctypes.c_void_p), ("weights_slots", ctypes.c_int64)]


class _CWeightsJob(ctypes.Structure):
    _fields_ = [("seg_base_k", _CTensor), ("seg_len", ctypes.c_int32),
                ("anchor_base_k", ctypes.POINTER(ctypes.c_void_p)), ("anchor_len", ctypes.POINTER(ctypes.c_int32)),
                ("n_anchors", ctypes.c_int32), ("weights_out", ctypes.c_void_p), ("nearest_out", ctypes.c_void_p),
                ("selected_out", ctypes.c_void_p)]


@dataclass(frozen=True)
class Model:
    """Shape of the model whose KV-cache is handled (kvcomm_model of the C header)."""
    n_layers: int
    n_kv_heads: int
    n_q_heads: int
    head_dim: int
    dtype: torch.dtype
    rope_theta: float

    def c(self):
        if self.dtype not in _DTYPES:
            raise KVCommError(-2, f"unsupported dtype {self.dtype}")
        return _CModel(self.n_layers, self.n_kv_heads, self.n_q_heads, self.head_dim, _DTYPES[self.dtype],
                       float(self.rope_theta))


@dataclass(frozen=True)
class Batch:
    """Sequences whose keys and values lie in the pages of a pool (kvcomm_batch of the C header), as int32 device tensors: table [B, W] the pages of
    each, lens [B] its tokens, the new ones included, starts [B + 1] its rows of the queries (None: one row each); max_rows: about
    the most rows of a sequence, 0: not known.  What the tensors hold is read when a call's kernels run, so a captured graph follows its changes."""
    table: torch.Tensor
    lens: torch.Tensor
    starts: Optional[torch.Tensor] = None
    max_rows: int = 0


_lib = None
_native = None   # the module _marshal or _Declines, set with _lib

# What _marshal is built against: it reads torch's and Python's objects through their internal layout
MARSHAL_FOR = f"torch {torch.__version__}, Python {sys.version_info[0]}.{sys.version_info[1]}"


class _Declines:
    """In the place of _marshal: takes no call."""
    def __getattr__(self, name):
        return lambda *args: None


def _load_native(lib):
    try:
        from . import _marshal
        built_for = getattr(_marshal, "built_for", None)
        if built_for != MARSHAL_FOR:
            raise ImportError(f"built for {built_for}, this is {MARSHAL_FOR}")
    except ImportError as e:
        warnings.warn(f"the native module _marshal is not used ({e}): build it with `python -m paper_2510_12872_amd.build`; small "
                      "calls take longer on the host without it", RuntimeWarning, stacklevel=3)
        return _Declines()
    _marshal.bind({n: ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _NATIVE_CALLS}, Model, torch.cuda.current_device,
                  _raw_current_stream, Batch)
    return _marshal


_NATIVE_CALLS = ("kvcomm_weight_slots", "kvcomm_suffix_attn_workspace", "kvcomm_anchor_weights_rule",
                 "kvcomm_anchor_weights_batch", "kvcomm_align_kv_batch", "kvcomm_align_kv_batch_beside", "kvcomm_align_kv_q8_batch", "kvcomm_align_kv",
                 "kvcomm_align_kv_q8", "kvcomm_suffix_attn", "kvcomm_suffix_attn_confined_ws", "kvcomm_anchor_predict",
                 "kvcomm_capture_offsets", "kvcomm_quantize_deltas", "kvcomm_place_qkv", "kvcomm_quantize_kv4", "kvcomm_dequantize_kv4",
                 "kvcomm_suffix_attn_kv4_workspace", "kvcomm_suffix_attn_kv4", "kvcomm_suffix_attn_window_workspace",
                 "kvcomm_suffix_attn_window", "kvcomm_place_qkv_paged", "kvcomm_paged_attn_workspace", "kvcomm_paged_attn",
                 "kvcomm_paged_attn_prefix_workspace", "kvcomm_paged_attn_prefix")


def library_path():
    return _LIB_PATH


def load_library():
    """Load libkvcomm.so (built by paper_2510_12872_amd.build); raises if it is missing."""
    global _lib, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2510_12872_amd.build` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    mp = ctypes.POINTER(_CModel)
    lib.kvcomm_weight_slots.argtypes = [mp, i32, i32]
    lib.kvcomm_weight_slots.restype = sz
    lib.kvcomm_anchor_weights_workspace.argtypes = [mp, i32, i32, i32]
    lib.kvcomm_anchor_weights_workspace.restype = sz
    lib.kvcomm_anchor_weights.argtypes = [mp, i32, f32, _CTensor, i32, ctypes.POINTER(vp), _CTensor,
                                          ctypes.POINTER(i32), i32, vp, vp, vp, vp, sz, vp]
    lib.kvcomm_anchor_weights.restype = ctypes.c_int
    lib.kvcomm_anchor_weights_static_capacity.argtypes = []
    lib.kvcomm_anchor_weights_static_capacity.restype = sz
    lib.kvcomm_anchor_weights_static.argtypes = [mp, i32, f32, _CTensor, i32, ctypes.POINTER(vp), _CTensor,
                                                 ctypes.POINTER(i32), i32, vp, vp, vp, vp]
    lib.kvcomm_anchor_weights_static.restype = ctypes.c_int
    lib.kvcomm_align_kv.argtypes = [mp, i32, _CTensor, _CTensor, i32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                    _CTensor, ctypes.POINTER(i32), i32, vp, i32, ctypes.POINTER(i32),
                                    _CTensor, _CTensor, vp]
    lib.kvcomm_align_kv.restype = ctypes.c_int
    lib.kvcomm_suffix_attn_workspace.argtypes = [mp, i32, i32]
    lib.kvcomm_suffix_attn_workspace.restype = sz
    lib.kvcomm_suffix_attn.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, i32, f32, _CTensor, vp, vp, sz, vp]
    lib.kvcomm_suffix_attn.restype = ctypes.c_int
    lib.kvcomm_suffix_attn_confined.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, i32, f32, _CTensor, vp, i32, vp]
    lib.kvcomm_suffix_attn_confined.restype = ctypes.c_int
    lib.kvcomm_suffix_attn_confined_ws.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, i32, f32, _CTensor, vp, i32,
                                                   vp, sz, vp]
    lib.kvcomm_suffix_attn_confined_ws.restype = ctypes.c_int
    lib.kvcomm_anchor_weights_rule_workspace.argtypes = [mp, i32, i32, i32, i32]
    lib.kvcomm_anchor_weights_rule_workspace.restype = sz
    lib.kvcomm_anchor_weights_rule.argtypes = [mp, i32, i32, f32, _CTensor, i32, ctypes.POINTER(vp), _CTensor,
                                               ctypes.POINTER(i32), i32, vp, vp, vp, vp, sz, vp]
    lib.kvcomm_anchor_weights_rule.restype = ctypes.c_int
    lib.kvcomm_anchor_predict_workspace.argtypes = [ctypes.c_int64]
    lib.kvcomm_anchor_predict_workspace.restype = sz
    lib.kvcomm_anchor_predict.argtypes = [vp, ctypes.c_int64, ctypes.POINTER(i32), i32, i32, f32, vp, vp, vp, sz, vp]
    lib.kvcomm_anchor_predict.restype = ctypes.c_int
    lib.kvcomm_capture_offsets.argtypes = [mp, _CTensor, _CTensor, _CTensor, _CTensor, i32, i32, _CTensor, _CTensor,
                                           vp]
    lib.kvcomm_capture_offsets.restype = ctypes.c_int
    lib.kvcomm_align_kv_batch.argtypes = [mp, i32, _CTensor, ctypes.POINTER(_CAlignJob), i32, vp]
    lib.kvcomm_align_kv_batch.restype = ctypes.c_int
    lib.kvcomm_align_kv_batch_beside.argtypes = [mp, i32, _CTensor, ctypes.POINTER(_CAlignJob), i32, i32, vp]
    lib.kvcomm_align_kv_batch_beside.restype = ctypes.c_int
    lib.kvcomm_anchor_weights_batch_workspace.argtypes = [mp, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), i32]
    lib.kvcomm_anchor_weights_batch_workspace.restype = sz
    lib.kvcomm_anchor_weights_batch.argtypes = [mp, i32, i32, f32, _CTensor, ctypes.POINTER(_CWeightsJob), i32, vp,
                                                sz, vp]
    lib.kvcomm_anchor_weights_batch.restype = ctypes.c_int
    lib.kvcomm_quantize_deltas.argtypes = [mp, _CTensor, i32, f32, _CTensor, vp]
    lib.kvcomm_quantize_deltas.restype = ctypes.c_int
    lib.kvcomm_align_kv_q8.argtypes = [mp, i32, _CTensor, _CTensor, i32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                       _CTensor, ctypes.POINTER(i32), ctypes.POINTER(f32), ctypes.POINTER(f32), i32,
                                       vp, i32, ctypes.POINTER(i32), _CTensor, _CTensor, vp]
    lib.kvcomm_align_kv_q8.restype = ctypes.c_int
    lib.kvcomm_align_kv_q8_batch.argtypes = [mp, i32, _CTensor, ctypes.POINTER(_CAlignQ8Job), i32, vp]
    lib.kvcomm_align_kv_q8_batch.restype = ctypes.c_int
    i64 = ctypes.c_int64
    lib.kvcomm_place_qkv.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, i32, vp, vp, i64, i64, f32, _CTensor, _CTensor, _CTensor, vp]
    lib.kvcomm_place_qkv.restype = ctypes.c_int
    lib.kvcomm_quantize_kv4.argtypes = [mp, _CTensor, _CTensor, i32, _CTensor4, _CTensor4, vp]
    lib.kvcomm_quantize_kv4.restype = ctypes.c_int
    lib.kvcomm_dequantize_kv4.argtypes = [mp, _CTensor4, _CTensor4, i32, _CTensor, _CTensor, vp]
    lib.kvcomm_dequantize_kv4.restype = ctypes.c_int
    lib.kvcomm_suffix_attn_kv4_workspace.argtypes = [mp, i32, i32]
    lib.kvcomm_suffix_attn_kv4_workspace.restype = sz
    lib.kvcomm_suffix_attn_kv4.argtypes = [mp, _CTensor, _CTensor4, _CTensor4, i32, i32, f32, _CTensor, vp, vp, sz, vp]
    lib.kvcomm_suffix_attn_kv4.restype = ctypes.c_int
    lib.kvcomm_suffix_attn_window_workspace.argtypes = [mp, i32, i32, i32, i32]
    lib.kvcomm_suffix_attn_window_workspace.restype = sz
    lib.kvcomm_suffix_attn_window.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, i32, i32, i32, f32, _CTensor, vp, vp, sz, vp]
    lib.kvcomm_suffix_attn_window.restype = ctypes.c_int
    bp = ctypes.POINTER(_CBatch)
    lib.kvcomm_place_qkv_paged.argtypes = [mp, _CTensor, _CTensor, _CTensor, bp, i32, vp, vp, i64, i64, f32, _CTensor, _CPages, _CPages, vp]
    lib.kvcomm_place_qkv_paged.restype = ctypes.c_int
    lib.kvcomm_paged_attn_workspace.argtypes = [mp, bp]
    lib.kvcomm_paged_attn_workspace.restype = sz
    lib.kvcomm_paged_attn.argtypes = [mp, _CTensor, _CPages, _CPages, bp, f32, _CTensor, vp, vp, sz, vp]
    lib.kvcomm_paged_attn.restype = ctypes.c_int
    lib.kvcomm_paged_attn_prefix_workspace.argtypes = [mp, i32, bp]
    lib.kvcomm_paged_attn_prefix_workspace.restype = sz
    lib.kvcomm_paged_attn_prefix.argtypes = [mp, _CTensor, _CTensor, _CTensor, i32, _CPages, _CPages, bp, f32, _CTensor, vp, vp, sz, vp]
    lib.kvcomm_paged_attn_prefix.restype = ctypes.c_int
    lib.kvcomm_status_string.argtypes = [ctypes.c_int]
    lib.kvcomm_status_string.restype = ctypes.c_char_p
    lib.kvcomm_version.argtypes = []
    lib.kvcomm_version.restype = ctypes.c_int
    _native = _load_native(lib)
    _lib = lib
    return lib


def _check(status):
    if status != 0:
        raise KVCommError(status, load_library().kvcomm_status_string(status).decode())


def _done(status):
    """Status of a call of the native module: False if it declined (nothing has been enqueued), else the call is made."""
    if status is None:
        return False
    if status != 0:
        _check(status)
    return True


INT32_MAX = 2 ** 31 - 1


def _int32(x, what):
    """A number for the library.  ctypes would pass on its last 32 bits."""
    x = int(x)
    if not -INT32_MAX - 1 <= x <= INT32_MAX:
        raise KVCommError(EINVAL, f"{what}: {x} does not fit 32 bits")
    return x


def _int32s(xs, n, what):
    """The same of a list, as an array of n elements (one at least)."""
    return (ctypes.c_int32 * max(n, 1))(*[_int32(x, what) for x in xs])


def _at_most_int32(x, what):
    """A number of tokens of which more than a cache can hold means all of them."""
    return _int32(min(int(x), INT32_MAX), what)


def _not_a_tensor(what, dtype):
    return KVCommError(-1, f"{what}: expected a 4-d {dtype} device tensor with contiguous channels")


# The functions below run once or more per library call; for small segments their cost is the call's cost, so each
# property of a tensor is read once.
def _desc(t, dtype, what):
    """[layer, head, token, channel] tensor -> kvcomm_tensor."""
    st = t.stride()
    if t.dtype != dtype or len(st) != 4 or st[3] != 1 or not t.is_cuda:
        raise _not_a_tensor(what, dtype)
    return _CTensor(t.data_ptr(), st[0], st[1], st[2])


_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # the handle without a Stream object around it


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_current_stream is not None:
        return _raw_current_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def on_stream(stream):
    """Context for allocations that kernels on `stream` (None: the current one) work in and that are dropped before these have run: they
    belong to that stream, so the allocator does not hand them out under the kernels."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream))


def _workspace(need, device, stream):
    """Scratch of one call."""
    with on_stream(stream):
        return torch.empty((need,), dtype=torch.uint8, device=device)


def _anchor_ptrs(anchors, dtype, what):
    """List of same-layout anchor tensors -> (host pointer array, layout descriptor)."""
    n = len(anchors)
    if n == 0:
        return None, _CTensor(None, 0, 0, 0)
    layout = _desc(anchors[0], dtype, what)
    st = anchors[0].stride()
    for a in anchors:
        if a.stride() != st or a.dtype != dtype or not a.is_cuda:
            _desc(a, dtype, what)
            raise KVCommError(-1, f"{what}: all anchors must share one layout (pad them to a common capacity)")
    return (ctypes.c_void_p * n)(*[a.data_ptr() for a in anchors]), layout


def _anchor_args(anchors, anchor_len, dtype, what):
    """List of same-layout anchor tensors -> (host pointer array, layout descriptor, host length array)."""
    ptrs, layout = _anchor_ptrs(anchors, dtype, what)
    if ptrs is None:
        return None, layout, None
    n = len(anchors)
    if anchor_len is None:
        anchor_len = [a.shape[2] for a in anchors]
    lens = _int32s(anchor_len, n, "anchor_len")
    return ptrs, layout, lens


def kvcomm_weight_slots(model, seg_len, gran=W_TOKEN):
    return int(load_library().kvcomm_weight_slots(ctypes.byref(model.c()), seg_len, gran))


def kvcomm_anchor_weights_workspace(model, seg_len, n_anchors, gran=W_TOKEN):
    return int(load_library().kvcomm_anchor_weights_workspace(ctypes.byref(model.c()), seg_len, n_anchors, gran))


def kvcomm_anchor_weights(model, seg_base_k, anchor_base_k, anchor_len=None, temperature=1.0, gran=W_TOKEN,
                          weights_out=None, nearest_out=None, selected_out=None, workspace=None, stream=None):
    """Anchor matching.  Returns (weights [n, A] fp32, nearest [n] int32, selected [A] int32)."""
    lib = load_library()
    seg_len = seg_base_k.shape[2]
    A = len(anchor_base_k)
    dev = seg_base_k.device
    if weights_out is None or nearest_out is None:
        n = kvcomm_weight_slots(model, seg_len, gran)
        if weights_out is None:
            weights_out = torch.empty((n, A), dtype=torch.float32, device=dev)
        if nearest_out is None:
            nearest_out = torch.empty((n,), dtype=torch.int32, device=dev)
    if selected_out is None:
        selected_out = torch.empty((A,), dtype=torch.int32, device=dev)
    if workspace is None:
        need = kvcomm_anchor_weights_workspace(model, seg_len, A, gran)
        workspace = _workspace(max(need, 1), dev, stream)
    if _done(_native.anchor_weights(model, gran, RULE_L2_SOFTMAX, temperature, seg_base_k, anchor_base_k, anchor_len, weights_out,
                                    nearest_out, selected_out, workspace, stream)):
        return weights_out, nearest_out, selected_out
    ptrs, layout, lens = _anchor_args(anchor_base_k, anchor_len, model.dtype, "anchor_base_k")
    _check(lib.kvcomm_anchor_weights(ctypes.byref(model.c()), gran, float(temperature),
                                     _desc(seg_base_k, model.dtype, "seg_base_k"), seg_len, ptrs, layout, lens, A,
                                     weights_out.data_ptr(), nearest_out.data_ptr(), selected_out.data_ptr(),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                     _stream_ptr(stream)))
    return weights_out, nearest_out, selected_out


def kvcomm_anchor_weights_static_capacity():
    return int(load_library().kvcomm_anchor_weights_static_capacity())


def kvcomm_anchor_weights_static(model, seg_base_k, anchor_base_k, weights_out, nearest_out, selected_out,
                                 anchor_len=None, temperature=1.0, gran=W_TOKEN, stream=None):
    """kvcomm_anchor_weights without a workspace argument (the library's fixed scratch array).  The caller
    passes every output; nothing is allocated here or in the library."""
    lib = load_library()
    ptrs, layout, lens = _anchor_args(anchor_base_k, anchor_len, model.dtype, "anchor_base_k")
    _check(lib.kvcomm_anchor_weights_static(ctypes.byref(model.c()), gran, float(temperature),
                                            _desc(seg_base_k, model.dtype, "seg_base_k"), seg_base_k.shape[2], ptrs,
                                            layout, lens, len(anchor_base_k), weights_out.data_ptr(),
                                            None if nearest_out is None else nearest_out.data_ptr(),
                                            None if selected_out is None else selected_out.data_ptr(),
                                            _stream_ptr(stream)))
    return weights_out, nearest_out, selected_out


def kvcomm_align_kv(model, base_k, base_v, anchor_dk, anchor_dv, weights, delta_pos, out_k, out_v,
                    anchor_len=None, anchor_delta_pos=None, gran=W_TOKEN, stream=None):
    """Positional alignment + offset approximation into out_k / out_v (views of the agent cache)."""
    lib = load_library()
    if _done(_native.align_kv(model, gran, base_k, base_v, anchor_dk, anchor_dv, weights, delta_pos, out_k, out_v, anchor_len,
                              anchor_delta_pos, stream)):
        return out_k, out_v
    seg_len = base_k.shape[2]
    A = len(anchor_dk)
    if len(anchor_dv) != A:
        raise KVCommError(-1, "anchor_dk and anchor_dv differ in length")
    pk, layout, lens = _anchor_args(anchor_dk, anchor_len, model.dtype, "anchor_dk")
    pv, layout_v = _anchor_ptrs(anchor_dv, model.dtype, "anchor_dv")
    if A and (layout.stride_layer, layout.stride_head, layout.stride_token) != (
            layout_v.stride_layer, layout_v.stride_head, layout_v.stride_token):
        raise KVCommError(-1, "anchor_dk and anchor_dv must share one layout")
    adp = None
    if anchor_delta_pos is not None:
        if len(anchor_delta_pos) != A:
            raise KVCommError(-1, "anchor_delta_pos must have one entry per anchor")
        adp = _int32s(anchor_delta_pos, A, "anchor_delta_pos")
    if A:
        if weights is None or weights.dtype != torch.float32 or not weights.is_contiguous():
            raise KVCommError(-1, "weights: expected a contiguous fp32 device tensor [n, A]")
        if weights.numel() != kvcomm_weight_slots(model, seg_len, gran) * A:
            raise KVCommError(-1, "weights: wrong number of elements for this granularity")
    _check(lib.kvcomm_align_kv(ctypes.byref(model.c()), gran, _desc(base_k, model.dtype, "base_k"),
                               _desc(base_v, model.dtype, "base_v"), seg_len, pk, pv, layout, lens, A,
                               None if weights is None else weights.data_ptr(), _int32(delta_pos, "delta_pos"), adp,
                               _desc(out_k, model.dtype, "out_k"), _desc(out_v, model.dtype, "out_v"),
                               _stream_ptr(stream)))
    return out_k, out_v


def kvcomm_suffix_attn_workspace(model, n_ctx, tq):
    return int(load_library().kvcomm_suffix_attn_workspace(ctypes.byref(model.c()), _int32(n_ctx, "n_ctx"), _int32(tq, "tq")))


def _in_private_pool(t):
    """Does t lie in one of the allocator's private pools, as all that is allocated under torch.cuda.graph does?  (Slow, asked
    during captures only.)"""
    p = t.data_ptr()
    return any(seg["address"] <= p < seg["address"] + seg["total_size"] and tuple(seg["segment_pool_id"]) != (0, 0)
               for seg in torch.cuda.memory_snapshot())


def _attn_scratch(need, device, stream):
    """Scratch of the attention, `need` bytes, or None.  Where there is no memory for it, or a graph that torch does not manage is being captured (the
    allocator would hand the memory out again while the graph's replays write to it), the call does without: same result
    up to rounding, only slower."""
    try:
        with on_stream(stream):
            workspace = torch.empty((need,), dtype=torch.uint8, device=device)
            capturing = torch.cuda.is_current_stream_capturing()
    except torch.OutOfMemoryError:
        return None
    return None if capturing and not _in_private_pool(workspace) else workspace


def apart(own, groups, each=()):
    """Do the tensors of the lists `groups` and of `each` come nowhere near a byte of the tensors `own`, and those of `each` not near each
    other?  (By the range from their first to their last element.)"""
    load_library()
    answer = _native.apart(own, groups, each)
    if answer is None:
        def span(t):
            return t.data_ptr(), t.data_ptr() + (1 + sum(max(0, n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size()
        meet = lambda a, b: a[0] < b[1] and b[0] < a[1]
        own, others, each = [span(t) for t in own], [span(t) for g in (*groups, each) for t in g], [span(t) for t in each]
        answer = not (any(meet(a, b) for a in own for b in others) or any(meet(a, b) for i, a in enumerate(each) for b in each[:i]))
    return bool(answer)


def _attn_workspace(cmodel, n_ctx, tq, workspace, device, stream):
    """(pointer, bytes, tensor to keep until the call has returned) of the attention's scratch, made here if not given."""
    if workspace is None:
        need = load_library().kvcomm_suffix_attn_workspace(ctypes.byref(cmodel), n_ctx, tq)
        workspace = _attn_scratch(need, device, stream) if need else None
        if workspace is None:
            return None, 0, None
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _suffix_attn(model, q, cache_k, cache_v, n_ctx, max_blocks, softmax_scale, out, lse_out, want_lse, stream, workspace):
    """Both attention calls; max_blocks None: the plain launch."""
    lib = load_library()
    tq = q.shape[2]
    if cache_k.shape[2] != n_ctx + tq or cache_v.shape[2] != n_ctx + tq:
        raise KVCommError(-1, "cache_k / cache_v must hold n_ctx + tq tokens")
    if out is None:
        out = torch.empty_like(q)
    if want_lse and lse_out is None:
        lse_out = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    need = 0   # bytes of scratch to be made here; None: not asked yet
    if workspace is None and n_ctx + tq >= ATTN_MIN_SPLIT_KEYS:
        need = _native.suffix_attn_workspace(model, n_ctx, tq)
    if need:
        workspace = _attn_scratch(need, q.device, stream)
    if need is not None and _done(_native.suffix_attn(model, q, cache_k, cache_v, n_ctx, softmax_scale, out, lse_out, max_blocks,
                                                      workspace, stream)):
        return (out, lse_out) if want_lse else out
    cmodel = model.c()
    ws, ws_bytes, _keep = None, 0, None
    if workspace is not None or need is None:
        ws, ws_bytes, _keep = _attn_workspace(cmodel, _int32(n_ctx, "n_ctx"), _int32(tq, "tq"), workspace, q.device, stream)
    args = (ctypes.byref(cmodel), _desc(q, model.dtype, "q"), _desc(cache_k, model.dtype, "cache_k"),
            _desc(cache_v, model.dtype, "cache_v"), _int32(n_ctx, "n_ctx"), _int32(tq, "tq"), float(softmax_scale), _desc(out, model.dtype, "out"),
            None if lse_out is None else lse_out.data_ptr())
    if max_blocks is None:
        _check(lib.kvcomm_suffix_attn(*args, ws, ws_bytes, _stream_ptr(stream)))
    else:
        _check(lib.kvcomm_suffix_attn_confined_ws(*args, _int32(max_blocks, "max_blocks"), ws, ws_bytes, _stream_ptr(stream)))
    return (out, lse_out) if want_lse else out


def kvcomm_suffix_attn(model, q, cache_k, cache_v, n_ctx, softmax_scale=0.0, out=None, lse_out=None,
                       want_lse=False, stream=None, workspace=None):
    """Causal attention of the suffix queries q [L,Hq,Tq,D] over cache_k/v [L,Hkv,n_ctx+Tq,D].

    workspace: kvcomm_suffix_attn_workspace() bytes on the device (made here if not given)."""
    return _suffix_attn(model, q, cache_k, cache_v, n_ctx, None, softmax_scale, out, lse_out, want_lse, stream, workspace)


def kvcomm_suffix_attn_confined(model, q, cache_k, cache_v, n_ctx, max_blocks, softmax_scale=0.0, out=None,
                                lse_out=None, want_lse=False, stream=None):
    """kvcomm_suffix_attn as at most max_blocks persistent thread blocks (one per compute unit)."""
    return kvcomm_suffix_attn_confined_ws(model, q, cache_k, cache_v, n_ctx, max_blocks, softmax_scale, out, lse_out,
                                          want_lse, stream)


def kvcomm_suffix_attn_confined_ws(model, q, cache_k, cache_v, n_ctx, max_blocks, softmax_scale=0.0, out=None,
                                   lse_out=None, want_lse=False, stream=None, workspace=None):
    """kvcomm_suffix_attn_confined with the scratch of kvcomm_suffix_attn (made here if not given): the same bits as
    kvcomm_suffix_attn with a workspace."""
    return _suffix_attn(model, q, cache_k, cache_v, n_ctx, int(max_blocks), softmax_scale, out, lse_out, want_lse, stream,
                        workspace)


def kvcomm_anchor_weights_rule_workspace(model, seg_len, n_anchors, gran=W_TOKEN, rule=RULE_L2_SOFTMAX):
    return int(load_library().kvcomm_anchor_weights_rule_workspace(ctypes.byref(model.c()), seg_len, n_anchors, gran,
                                                                   rule))


def kvcomm_anchor_weights_rule(model, rule, seg_base_k, anchor_base_k, anchor_len=None, temperature=1.0, gran=W_TOKEN,
                               weights_out=None, nearest_out=None, selected_out=None, workspace=None, stream=None):
    """Anchor matching under one of the weighting variants.  Returns (weights, nearest, selected)."""
    lib = load_library()
    seg_len = seg_base_k.shape[2]
    A = len(anchor_base_k)
    dev = seg_base_k.device
    if weights_out is None or nearest_out is None:
        n = kvcomm_weight_slots(model, seg_len, gran)
        if weights_out is None:
            weights_out = torch.empty((n, A), dtype=torch.float32, device=dev)
        if nearest_out is None:
            nearest_out = torch.empty((n,), dtype=torch.int32, device=dev)
    if selected_out is None:
        selected_out = torch.empty((A,), dtype=torch.int32, device=dev)
    if workspace is None:
        need = kvcomm_anchor_weights_rule_workspace(model, seg_len, A, gran, rule)
        workspace = _workspace(max(need, 1), dev, stream)
    if _done(_native.anchor_weights(model, gran, rule, temperature, seg_base_k, anchor_base_k, anchor_len, weights_out, nearest_out,
                                    selected_out, workspace, stream)):
        return weights_out, nearest_out, selected_out
    ptrs, layout, lens = _anchor_args(anchor_base_k, anchor_len, model.dtype, "anchor_base_k")
    _check(lib.kvcomm_anchor_weights_rule(ctypes.byref(model.c()), gran, int(rule), float(temperature),
                                          _desc(seg_base_k, model.dtype, "seg_base_k"), seg_len, ptrs, layout, lens,
                                          A, weights_out.data_ptr(), nearest_out.data_ptr(), selected_out.data_ptr(),
                                          workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                          _stream_ptr(stream)))
    return weights_out, nearest_out, selected_out


def kvcomm_anchor_predict_workspace(n_slots):
    return int(load_library().kvcomm_anchor_predict_workspace(int(n_slots)))


def kvcomm_anchor_predict(weights, anchor_len, seg_len, gamma, entropy_out=None, result_out=None, workspace=None,
                          want_entropy=False, stream=None):
    """Eq. "pred" on the device.  weights [n, A] fp32.  Returns result [2] (decision, mean entropy)
    and, with want_entropy, the per-slot entropies [n]."""
    lib = load_library()
    if weights.dim() != 2 or weights.dtype != torch.float32 or not weights.is_contiguous() or not weights.is_cuda:
        raise KVCommError(-1, "weights: expected a contiguous fp32 device tensor [n, A]")
    n, A = weights.shape
    if len(anchor_len) != A:
        raise KVCommError(-1, "anchor_len must have one entry per anchor")
    dev = weights.device
    if want_entropy and entropy_out is None:
        entropy_out = torch.empty((n,), dtype=torch.float32, device=dev)
    if result_out is None:
        result_out = torch.empty((2,), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _workspace(max(kvcomm_anchor_predict_workspace(n), 8), dev, stream)
    if _done(_native.anchor_predict(weights, anchor_len, seg_len, gamma, entropy_out, result_out, workspace, stream)):
        return (result_out, entropy_out) if want_entropy else result_out
    lens = _int32s(anchor_len, A, "anchor_len")
    _check(lib.kvcomm_anchor_predict(weights.data_ptr(), n, lens, A, _int32(seg_len, "seg_len"), float(gamma),
                                     None if entropy_out is None else entropy_out.data_ptr(), result_out.data_ptr(),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                     _stream_ptr(stream)))
    return (result_out, entropy_out) if want_entropy else result_out


def kvcomm_capture_offsets(model, base_k, base_v, real_k, real_v, delta_pos, out_dk=None, out_dv=None, stream=None):
    """Offset capture: (real - re-positioned base) for keys and values of one segment."""
    lib = load_library()
    seg_len = base_k.shape[2]
    for t in (base_v, real_k, real_v):
        if t.shape != base_k.shape:
            raise KVCommError(-1, "base and real tensors must have one shape")
    if out_dk is None:
        out_dk = torch.empty(base_k.shape, dtype=model.dtype, device=base_k.device)
    if out_dv is None:
        out_dv = torch.empty(base_k.shape, dtype=model.dtype, device=base_k.device)
    if _done(_native.capture_offsets(model, base_k, base_v, real_k, real_v, delta_pos, out_dk, out_dv, stream)):
        return out_dk, out_dv
    d = lambda t, what: _desc(t, model.dtype, what)
    _check(lib.kvcomm_capture_offsets(ctypes.byref(model.c()), d(base_k, "base_k"), d(base_v, "base_v"),
                                      d(real_k, "real_k"), d(real_v, "real_v"), seg_len, _int32(delta_pos, "delta_pos"),
                                      d(out_dk, "out_dk"), d(out_dv, "out_dv"), _stream_ptr(stream)))
    return out_dk, out_dv


def _same_layout(a, b):
    return (a.stride_layer, a.stride_head, a.stride_token) == (b.stride_layer, b.stride_head, b.stride_token)


def kvcomm_anchor_weights_batch_workspace(model, seg_lens, n_anchors, gran=W_TOKEN, rule=RULE_L2_SOFTMAX):
    n = len(seg_lens)
    sl, na = _int32s(seg_lens, n, "seg_lens"), _int32s(n_anchors, n, "n_anchors")
    return int(load_library().kvcomm_anchor_weights_batch_workspace(ctypes.byref(model.c()), gran, rule, sl, na, n))


def kvcomm_anchor_weights_batch(model, jobs, temperature=1.0, gran=W_TOKEN, rule=RULE_L2_SOFTMAX, workspace=None,
                                stream=None):
    """Anchor matching of several segments in one launch per stage.

    jobs: list of dicts with seg_base_k, anchor_base_k (list of tensors) and optionally anchor_len,
    weights_out, nearest_out, selected_out.  Returns a list of (weights, nearest, selected)."""
    lib = load_library()
    n = len(jobs)
    outs = []
    for jd in jobs:
        w, nr, so = jd.get("weights_out"), jd.get("nearest_out"), jd.get("selected_out")
        if w is None or nr is None or so is None:
            seg, A = jd["seg_base_k"], len(jd["anchor_base_k"])
            if w is None or nr is None:
                slots = kvcomm_weight_slots(model, seg.shape[2], gran)
                w = torch.empty((slots, A), dtype=torch.float32, device=seg.device) if w is None else w
                nr = torch.empty((slots,), dtype=torch.int32, device=seg.device) if nr is None else nr
            so = torch.empty((A,), dtype=torch.int32, device=seg.device) if so is None else so
        outs.append((w, nr, so))
    if workspace is None:
        need = kvcomm_anchor_weights_batch_workspace(model, [jd["seg_base_k"].shape[2] for jd in jobs],
                                                     [len(jd["anchor_base_k"]) for jd in jobs], gran, rule)
        workspace = _workspace(max(need, 256), jobs[0]["seg_base_k"].device, stream)
    if _done(_native.anchor_weights_batch(model, gran, rule, temperature, jobs, outs, workspace, stream)):
        return outs
    cjobs = (_CWeightsJob * max(n, 1))()
    keep, layout = [], None
    for j, (jd, (w, nr, so)) in enumerate(zip(jobs, outs)):
        seg = jd["seg_base_k"]
        S, A = seg.shape[2], len(jd["anchor_base_k"])
        ptrs, lay, lens = _anchor_args(jd["anchor_base_k"], jd.get("anchor_len"), model.dtype, "anchor_base_k")
        if layout is None:
            layout = lay
        elif A and not _same_layout(layout, lay):
            raise KVCommError(-1, "all anchors of a batched call must share one layout")
        keep.append((ptrs, lens))
        cjobs[j] = _CWeightsJob(_desc(seg, model.dtype, "seg_base_k"), S, ptrs, lens, A, w.data_ptr(), nr.data_ptr(),
                                so.data_ptr())
    _check(lib.kvcomm_anchor_weights_batch(ctypes.byref(model.c()), gran, int(rule), float(temperature),
                                           layout if layout is not None else _CTensor(None, 0, 0, 0), cjobs, n,
                                           workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                           _stream_ptr(stream)))
    return outs


def kvcomm_align_kv_batch(model, jobs, gran=W_TOKEN, stream=None):
    """Positional alignment + offset approximation of several segments in one launch.

    jobs: list of dicts with base_k, base_v, anchor_dk, anchor_dv (lists of tensors), weights, delta_pos,
    out_k, out_v and optionally anchor_len, anchor_delta_pos."""
    _align_kv_batch(model, jobs, None, gran, stream)


def kvcomm_align_kv_batch_beside(model, jobs, units, gran=W_TOKEN, stream=None):
    """kvcomm_align_kv_batch (the same bits) as a launch beside other work that leaves it about `units` of the COMPUTE_UNITS."""
    _align_kv_batch(model, jobs, units, gran, stream)


def _align_kv_batch(model, jobs, units, gran, stream):
    """Both batched updates; units None: the plain launch."""
    lib = load_library()
    if _done(_native.align_kv_batch(model, gran, jobs, units, stream)):
        return
    n = len(jobs)
    cjobs = (_CAlignJob * max(n, 1))()
    keep, layout = [], None
    for j, jd in enumerate(jobs):
        A = len(jd["anchor_dk"])
        if len(jd["anchor_dv"]) != A:
            raise KVCommError(-1, "anchor_dk and anchor_dv differ in length")
        pk, lay, lens = _anchor_args(jd["anchor_dk"], jd.get("anchor_len"), model.dtype, "anchor_dk")
        pv, lay_v = _anchor_ptrs(jd["anchor_dv"], model.dtype, "anchor_dv")
        if A:
            if not _same_layout(lay, lay_v) or (layout is not None and not _same_layout(layout, lay)):
                raise KVCommError(-1, "all anchors of a batched call must share one layout")
            layout = lay
        adp = None
        if jd.get("anchor_delta_pos") is not None:
            if len(jd["anchor_delta_pos"]) != A:
                raise KVCommError(-1, "anchor_delta_pos must have one entry per anchor")
            adp = _int32s(jd["anchor_delta_pos"], A, "anchor_delta_pos")
        w = jd.get("weights")
        S = jd["base_k"].shape[2]
        if A:
            if w is None or w.dtype != torch.float32 or not w.is_contiguous():
                raise KVCommError(-1, "weights: expected a contiguous fp32 device tensor [n, A]")
            if w.numel() % A:
                raise KVCommError(-1, "weights: expected [n, A]")
        keep.append((pk, pv, lens, adp))
        d = lambda t, what: _desc(t, model.dtype, what)
        cjobs[j] = _CAlignJob(d(jd["base_k"], "base_k"), d(jd["base_v"], "base_v"), d(jd["out_k"], "out_k"),
                              d(jd["out_v"], "out_v"), S, _int32(jd["delta_pos"], "delta_pos"), pk, pv, lens, adp, A,
                              None if w is None else w.data_ptr(), 0 if (w is None or not A) else w.numel() // A)
    args = (ctypes.byref(model.c()), gran, layout if layout is not None else _CTensor(None, 0, 0, 0), cjobs, n)
    if units is None:
        _check(lib.kvcomm_align_kv_batch(*args, _stream_ptr(stream)))
    else:
        _check(lib.kvcomm_align_kv_batch_beside(*args, _int32(units, "units"), _stream_ptr(stream)))


def _desc_q8(t, what):
    """[layer, head, token, channel] uint8 tensor of E4M3 codes -> kvcomm_tensor (strides in bytes)."""
    st = t.stride()
    if t.dtype != torch.uint8 or len(st) != 4 or st[3] != 1 or not t.is_cuda:
        raise KVCommError(-1, f"{what}: expected a 4-d uint8 device tensor with contiguous channels")
    return _CTensor(t.data_ptr(), st[0], st[1], st[2])


def _anchor_ptrs_q8(dk8, dv8):
    """Compressed deviations (at least one anchor) -> (key pointers, value pointers, their common layout)."""
    n = len(dk8)
    layout = _desc_q8(dk8[0], "anchor_dk8")
    st = dk8[0].stride()
    for anchors in (dk8, dv8):
        for a in anchors:
            if a.stride() != st or a.dtype != torch.uint8 or not a.is_cuda:
                _desc_q8(a, "anchor deviations")
                raise KVCommError(-1, "all compressed anchors must share one layout")
    return (ctypes.c_void_p * n)(*[a.data_ptr() for a in dk8]), (ctypes.c_void_p * n)(*[a.data_ptr() for a in dv8]), layout


def kvcomm_quantize_deltas(model, x, scale, out=None, stream=None):
    """Stored deviation x [L,Hkv,n,D] (model dtype) -> E4M3 codes (uint8) of x / scale; scale a power of two."""
    lib = load_library()
    if out is None:
        out = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    if _done(_native.quantize_deltas(model, x, scale, out, stream)):
        return out
    _check(lib.kvcomm_quantize_deltas(ctypes.byref(model.c()), _desc(x, model.dtype, "x"), x.shape[2], float(scale),
                                      _desc_q8(out, "out"), _stream_ptr(stream)))
    return out


def kvcomm_align_kv_q8(model, base_k, base_v, anchor_dk8, anchor_dv8, scale_k, scale_v, weights, delta_pos, out_k,
                       out_v, anchor_len=None, anchor_delta_pos=None, gran=W_TOKEN, stream=None):
    """kvcomm_align_kv with E4M3-compressed deviations (uint8 tensors) and their per-anchor scales."""
    lib = load_library()
    if _done(_native.align_kv_q8(model, gran, base_k, base_v, anchor_dk8, anchor_dv8, scale_k, scale_v, weights, delta_pos, out_k,
                                 out_v, anchor_len, anchor_delta_pos, stream)):
        return out_k, out_v
    seg_len = base_k.shape[2]
    A = len(anchor_dk8)
    if len(anchor_dv8) != A or len(scale_k) != A or len(scale_v) != A:
        raise KVCommError(-1, "anchor lists and scales differ in length")
    if A:
        pk, pv, layout = _anchor_ptrs_q8(anchor_dk8, anchor_dv8)
        lens = _int32s(anchor_len if anchor_len is not None else [a.shape[2] for a in anchor_dk8], A, "anchor_len")
        sk = (ctypes.c_float * A)(*[float(x) for x in scale_k])
        sv = (ctypes.c_float * A)(*[float(x) for x in scale_v])
        if weights is None or weights.dtype != torch.float32 or not weights.is_contiguous():
            raise KVCommError(-1, "weights: expected a contiguous fp32 device tensor [n, A]")
        if weights.numel() != kvcomm_weight_slots(model, seg_len, gran) * A:
            raise KVCommError(-1, "weights: wrong number of elements for this granularity")
    else:
        layout, pk, pv, lens, sk, sv = _CTensor(None, 0, 0, 0), None, None, None, None, None
    adp = None
    if anchor_delta_pos is not None:
        adp = _int32s(anchor_delta_pos, A, "anchor_delta_pos")
    _check(lib.kvcomm_align_kv_q8(ctypes.byref(model.c()), gran, _desc(base_k, model.dtype, "base_k"),
                                  _desc(base_v, model.dtype, "base_v"), seg_len, pk, pv, layout, lens, sk, sv, A,
                                  None if weights is None else weights.data_ptr(), _int32(delta_pos, "delta_pos"), adp,
                                  _desc(out_k, model.dtype, "out_k"), _desc(out_v, model.dtype, "out_v"),
                                  _stream_ptr(stream)))
    return out_k, out_v


def kvcomm_align_kv_q8_batch(model, jobs, gran=W_TOKEN, stream=None):
    """The compressed update of several segments in one launch.

    jobs: list of dicts with base_k, base_v, anchor_dk8, anchor_dv8 (lists of uint8 tensors), scale_k, scale_v
    (lists of floats), weights, delta_pos, out_k, out_v and optionally anchor_len, anchor_delta_pos."""
    lib = load_library()
    if _done(_native.align_kv_q8_batch(model, gran, jobs, None, stream)):
        return
    n = len(jobs)
    cjobs = (_CAlignQ8Job * max(n, 1))()
    keep, layout = [], None
    for j, jd in enumerate(jobs):
        dk8, dv8 = jd["anchor_dk8"], jd["anchor_dv8"]
        A = len(dk8)
        if len(dv8) != A or len(jd["scale_k"]) != A or len(jd["scale_v"]) != A:
            raise KVCommError(-1, "anchor lists and scales differ in length")
        pk = pv = lens = sk = sv = adp = None
        if A:
            pk, pv, lay = _anchor_ptrs_q8(dk8, dv8)
            if layout is not None and not _same_layout(layout, lay):
                raise KVCommError(-1, "all anchors of a batched call must share one layout")
            layout = lay
            al = jd.get("anchor_len")
            lens = _int32s(al if al is not None else [a.shape[2] for a in dk8], A, "anchor_len")
            sk = (ctypes.c_float * A)(*[float(x) for x in jd["scale_k"]])
            sv = (ctypes.c_float * A)(*[float(x) for x in jd["scale_v"]])
        if jd.get("anchor_delta_pos") is not None:
            if len(jd["anchor_delta_pos"]) != A:
                raise KVCommError(-1, "anchor_delta_pos must have one entry per anchor")
            adp = _int32s(jd["anchor_delta_pos"], A, "anchor_delta_pos")
        w = jd.get("weights")
        if A and (w is None or w.dtype != torch.float32 or not w.is_contiguous() or w.numel() % A):
            raise KVCommError(-1, "weights: expected a contiguous fp32 device tensor [n, A]")
        keep.append((pk, pv, lens, sk, sv, adp))
        d = lambda t, what: _desc(t, model.dtype, what)
        cjobs[j] = _CAlignQ8Job(d(jd["base_k"], "base_k"), d(jd["base_v"], "base_v"), d(jd["out_k"], "out_k"),
                                d(jd["out_v"], "out_v"), jd["base_k"].shape[2], _int32(jd["delta_pos"], "delta_pos"), pk, pv, lens, adp,
                                sk, sv, A, None if w is None else w.data_ptr(),
                                0 if (w is None or not A) else w.numel() // A)
    _check(lib.kvcomm_align_kv_q8_batch(ctypes.byref(model.c()), gran,
                                        layout if layout is not None else _CTensor(None, 0, 0, 0), cjobs, n,
                                        _stream_ptr(stream)))


def _sized(t, dtype, shape, what):
    """Descriptor of a tensor of exactly this shape."""
    d = _desc(t, dtype, what)
    if tuple(t.shape) != shape:
        raise KVCommError(EINVAL, f"{what}: expected shape {shape}, not {tuple(t.shape)}")
    return d


def _on_stream_of(tensors, stream):
    """The stream's handle, if the tensors of a call all lie on its device."""
    dev = getattr(stream, "device_index", None)
    dev = torch.cuda.current_device() if dev is None else dev
    if any(t is not None and (not t.is_cuda or t.get_device() != dev) for t in tensors):
        raise KVCommError(EINVAL, f"all tensors of a call have to lie on the device of its stream ({dev})")
    return _stream_ptr(stream)


def _compact(model, pair, n, what):
    """(codes, scales) of a tensor in 4 bits -> descriptor."""
    codes, scales = pair
    head = (model.n_layers, model.n_kv_heads, n)
    return _CTensor4(_sized(codes, torch.uint8, head + (model.head_dim // 2,), what + " codes"),
                     _sized(scales, torch.uint8, head + (model.head_dim // 32,), what + " scales"))


def _new_compact(model, n, device):
    head = (model.n_layers, model.n_kv_heads, n)
    return (torch.empty(head + (model.head_dim // 2,), dtype=torch.uint8, device=device),
            torch.empty(head + (model.head_dim // 32,), dtype=torch.uint8, device=device))


def _norm_weights(model, q_weight, k_weight, norm_eps):
    """(pointer, elements from layer to layer) of the weights of queries and keys."""
    if norm_eps != 0 and ctypes.c_float(float(norm_eps)).value == 0:
        raise KVCommError(EINVAL, f"norm_eps: {norm_eps} is 0 in fp32, which means no norm")
    weights = []
    for w, what in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None and (w.dtype != model.dtype or not w.is_cuda or w.stride(-1) != 1 or
                              tuple(w.shape) not in ((model.head_dim,), (model.n_layers, model.head_dim))):
            raise KVCommError(EINVAL, f"{what}: expected a {model.dtype} device tensor [D] or [L, D] with contiguous channels")
        weights.append((None, 0) if w is None else (w.data_ptr(), w.stride(0) if w.dim() == 2 else 0))
    return weights


def kvcomm_place_qkv(model, q, k, v, first_pos, q_out=None, k_out=None, v_out=None, q_weight=None, k_weight=None, norm_eps=0.0, stream=None):
    """Projections of a suffix q [L,Hq,n,D], k, v [L,Hkv,n,D] -> (q_out, k_out, v_out): per-head RMS norm of q and k where norm_eps > 0 (times
    q_weight, k_weight [D] or [L, D]), rotation of token i to position first_pos + i, v copied.  k_out and v_out are normally views of the agent's
    cache; outputs that are not passed are made.  None in the place of q, k or v leaves it out."""
    lib = load_library()
    if (q_out is None and q is not None) or (k_out is None and k is not None) or (v_out is None and v is not None):
        with on_stream(stream):
            q_out, k_out, v_out = (torch.empty(x.shape, dtype=x.dtype, device=x.device) if y is None and x is not None else y
                                   for x, y in ((q, q_out), (k, k_out), (v, v_out)))
    if _done(_native.place_qkv(model, q, k, v, first_pos, q_weight, k_weight, norm_eps, q_out, k_out, v_out, stream)):
        return q_out, k_out, v_out
    ins, outs = (q, k, v), (q_out, k_out, v_out)
    n = _int32(next((x.shape[2] for x in ins if x is not None), 0), "tokens")
    none = _CTensor(None, 0, 0, 0)
    cin, cout = [none] * 3, [none] * 3
    for i, (x, y, what) in enumerate(zip(ins, outs, "qkv")):
        if (x is None) != (y is None):
            raise KVCommError(EINVAL, f"{what}_out without {what}")
        if x is not None:
            shape = (model.n_layers, model.n_kv_heads if i else model.n_q_heads, n, model.head_dim)
            cin[i], cout[i] = _sized(x, model.dtype, shape, what), _sized(y, model.dtype, shape, what + "_out")
    weights = _norm_weights(model, q_weight, k_weight, norm_eps)
    _check(lib.kvcomm_place_qkv(ctypes.byref(model.c()), *cin, n, _int32(first_pos, "first_pos"), weights[0][0], weights[1][0], weights[0][1], weights[1][1],
                                float(norm_eps), *cout, _on_stream_of((*ins, *outs, q_weight, k_weight), stream)))
    return outs


def kvcomm_quantize_kv4(model, k, v, out_k=None, out_v=None, stream=None):
    """Rows of keys and values [L,Hkv,n,D] -> (codes [L,Hkv,n,D/2], scales [L,Hkv,n,D/32]) of each, uint8 (made if not passed): a compact cache's
    rows, 4 bits per value and a power-of-two scale per 32 channels."""
    lib = load_library()
    n = k.shape[2]
    with on_stream(stream) if out_k is None or out_v is None else contextlib.nullcontext():
        out_k = _new_compact(model, n, k.device) if out_k is None else out_k
        out_v = _new_compact(model, n, k.device) if out_v is None else out_v
    if _done(_native.quantize_kv4(model, k, v, out_k, out_v, stream)):
        return out_k, out_v
    _int32(n, "tokens")
    shape = (model.n_layers, model.n_kv_heads, n, model.head_dim)
    _check(lib.kvcomm_quantize_kv4(ctypes.byref(model.c()), _sized(k, model.dtype, shape, "k"), _sized(v, model.dtype, shape, "v"), n,
                                   _compact(model, out_k, n, "out_k"), _compact(model, out_v, n, "out_v"),
                                   _on_stream_of((k, v, *out_k, *out_v), stream)))
    return out_k, out_v


def kvcomm_dequantize_kv4(model, k, v, out_k=None, out_v=None, stream=None):
    """The values [L,Hkv,n,D] that compact keys and values (each a pair of codes and scales) hold, in the model's type."""
    lib = load_library()
    n = k[0].shape[2]
    shape = (model.n_layers, model.n_kv_heads, n, model.head_dim)
    with on_stream(stream) if out_k is None or out_v is None else contextlib.nullcontext():
        out_k = torch.empty(shape, dtype=model.dtype, device=k[0].device) if out_k is None else out_k
        out_v = torch.empty(shape, dtype=model.dtype, device=k[0].device) if out_v is None else out_v
    if _done(_native.dequantize_kv4(model, k, v, out_k, out_v, stream)):
        return out_k, out_v
    _int32(n, "tokens")
    _check(lib.kvcomm_dequantize_kv4(ctypes.byref(model.c()), _compact(model, k, n, "k"), _compact(model, v, n, "v"), n,
                                     _sized(out_k, model.dtype, shape, "out_k"), _sized(out_v, model.dtype, shape, "out_v"),
                                     _on_stream_of((*k, *v, out_k, out_v), stream)))
    return out_k, out_v


def kvcomm_suffix_attn_kv4_workspace(model, n_ctx, tq):
    return int(load_library().kvcomm_suffix_attn_kv4_workspace(ctypes.byref(model.c()), _int32(n_ctx, "n_ctx"), _int32(tq, "tq")))


def kvcomm_suffix_attn_window_workspace(model, n_ctx, tq, window, n_sinks=0):
    return int(load_library().kvcomm_suffix_attn_window_workspace(ctypes.byref(model.c()), _int32(n_ctx, "n_ctx"), _int32(tq, "tq"),
                                                                  _at_most_int32(window, "window"), _at_most_int32(n_sinks, "n_sinks")))


def _attn_outputs(q, out, lse_out, want_lse, stream):
    if out is None or (want_lse and lse_out is None):
        with on_stream(stream):
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
            if want_lse and lse_out is None:
                lse_out = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    return out, lse_out


def _attn_checked(model, q, out, lse_out, workspace):
    """(descriptor of q, of out, pointer of lse_out, pointer and bytes of workspace) of a call that the native module declined."""
    _int32(q.shape[2], "tq")
    shape = (model.n_layers, model.n_q_heads, q.shape[2], model.head_dim)
    cq, cout = _sized(q, model.dtype, shape, "q"), _sized(out, model.dtype, shape, "out")
    if lse_out is not None and (lse_out.dtype != torch.float32 or not lse_out.is_cuda or not lse_out.is_contiguous() or
                                lse_out.numel() != shape[0] * shape[1] * shape[2]):
        raise KVCommError(EINVAL, "lse_out: expected a contiguous fp32 device tensor [L, Hq, tq]")
    ws = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return cq, cout, None if lse_out is None else lse_out.data_ptr(), ws


def kvcomm_suffix_attn_kv4(model, q, cache_k, cache_v, n_ctx, softmax_scale=0.0, out=None, lse_out=None, want_lse=False, stream=None,
                           workspace=None):
    """kvcomm_suffix_attn over a compact cache: cache_k / cache_v are pairs of codes [L,Hkv,n_ctx+Tq,D/2] and scales [L,Hkv,n_ctx+Tq,D/32].

    workspace: kvcomm_suffix_attn_kv4_workspace() bytes on the device (made here if not given)."""
    lib = load_library()
    tq = q.shape[2]
    out, lse_out = _attn_outputs(q, out, lse_out, want_lse, stream)
    if workspace is None:
        need = _native.suffix_attn_kv4_workspace(model, n_ctx, tq)
        need = kvcomm_suffix_attn_kv4_workspace(model, n_ctx, tq) if need is None else need
        workspace = _attn_scratch(need, q.device, stream) if need else None
    if not _done(_native.suffix_attn_kv4(model, q, cache_k, cache_v, n_ctx, softmax_scale, out, lse_out, workspace, stream)):
        cq, cout, lse, ws = _attn_checked(model, q, out, lse_out, workspace)
        n_ctx = _int32(n_ctx, "n_ctx")
        N = n_ctx + tq
        _check(lib.kvcomm_suffix_attn_kv4(ctypes.byref(model.c()), cq, _compact(model, cache_k, N, "cache_k"), _compact(model, cache_v, N, "cache_v"),
                                          n_ctx, tq, float(softmax_scale), cout, lse, *ws,
                                          _on_stream_of((q, *cache_k, *cache_v, out, lse_out, workspace), stream)))
    return (out, lse_out) if want_lse else out


def kvcomm_suffix_attn_window(model, q, cache_k, cache_v, n_ctx, window, n_sinks=0, softmax_scale=0.0, out=None, lse_out=None, want_lse=False,
                              stream=None, workspace=None):
    """kvcomm_suffix_attn where the query at position p sees the tokens (p - window, p] and the cache's first n_sinks tokens.

    workspace: kvcomm_suffix_attn_window_workspace() bytes on the device (made here if not given)."""
    lib = load_library()
    tq = q.shape[2]
    out, lse_out = _attn_outputs(q, out, lse_out, want_lse, stream)
    if workspace is None:
        need = _native.suffix_attn_window_workspace(model, n_ctx, tq, window, n_sinks)
        need = kvcomm_suffix_attn_window_workspace(model, n_ctx, tq, window, n_sinks) if need is None else need
        workspace = _attn_scratch(need, q.device, stream) if need else None
    if not _done(_native.suffix_attn_window(model, q, cache_k, cache_v, n_ctx, window, n_sinks, softmax_scale, out, lse_out, workspace, stream)):
        cq, cout, lse, ws = _attn_checked(model, q, out, lse_out, workspace)
        n_ctx, window, n_sinks = _int32(n_ctx, "n_ctx"), _at_most_int32(window, "window"), _at_most_int32(n_sinks, "n_sinks")
        shape = (model.n_layers, model.n_kv_heads, n_ctx + tq, model.head_dim)
        _check(lib.kvcomm_suffix_attn_window(ctypes.byref(model.c()), cq, _sized(cache_k, model.dtype, shape, "cache_k"),
                                             _sized(cache_v, model.dtype, shape, "cache_v"), n_ctx, tq, window, n_sinks,
                                             float(softmax_scale), cout, lse, *ws,
                                             _on_stream_of((q, cache_k, cache_v, out, lse_out, workspace), stream)))
    return (out, lse_out) if want_lse else out


def _int32_tensor(t, dim, what):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.dim() != dim or not t.is_cuda or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise KVCommError(EINVAL, f"{what}: expected a {dim}-d int32 device tensor, contiguous along its last axis")
    return t


def _batch(batch, n_rows, page_size, n_pages):
    """kvcomm_batch of a batch over a pool of these pages."""
    table, lens = _int32_tensor(batch.table, 2, "table"), _int32_tensor(batch.lens, 1, "lens")
    B, starts = lens.shape[0], batch.starts
    if table.shape[0] != B:
        raise KVCommError(EINVAL, f"table: {table.shape[0]} rows for {B} sequences")
    if starts is not None and _int32_tensor(starts, 1, "starts").shape[0] != B + 1:
        raise KVCommError(EINVAL, f"starts: expected {B + 1} entries, not {starts.shape[0]}")
    return _CBatch(table.data_ptr() or None, lens.data_ptr() or None, None if starts is None else starts.data_ptr(), table.stride(0) if B > 1 else 0,
                   _int32(table.shape[1], "table"), _int32(B, "sequences"), _int32(n_rows, "rows"), _int32(page_size, "page_size"), _int32(n_pages, "pages"),
                   _int32(batch.max_rows, "max_rows"))


def _pool(model, t, pages, what):
    """Descriptor of a pool of `pages` = (pages, slots), None: any."""
    if t.dtype != model.dtype or t.dim() != 5 or not t.is_cuda or t.stride(4) != 1:
        raise KVCommError(EINVAL, f"{what}: expected a 5-d {model.dtype} device tensor [L, Hkv, pages, slots, D] with contiguous channels")
    shape = (model.n_layers, model.n_kv_heads, *(tuple(t.shape[2:4]) if pages is None else pages), model.head_dim)
    if tuple(t.shape) != shape:
        raise KVCommError(EINVAL, f"{what}: expected shape {shape}, not {tuple(t.shape)}")
    return _CPages(t.data_ptr() or None, *t.stride()[:4])


def kvcomm_place_qkv_paged(model, q, k, v, batch, pages_k, pages_v, first_pos=0, q_out=None, q_weight=None, k_weight=None, norm_eps=0.0, stream=None):
    """kvcomm_place_qkv for the new tokens of a batch: q [L,Hq,n,D] -> q_out (made if not passed, and returned), k, v [L,Hkv,n,D] -> their slots of
    the pools pages_k, pages_v [L,Hkv,pages,slots,D].  Token t of a sequence stands at position first_pos + t.  None in the place of q, or of k and its
    pool, or of v and its pool leaves it out (the batch's pages are then those of the other pool)."""
    lib = load_library()
    if q_out is None and q is not None:
        with on_stream(stream):
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            if batch.starts is not None:   # rows of no sequence stay as they were: zeros
                q_out.zero_()
    if _done(_native.place_qkv_paged(model, q, k, v, batch, pages_k, pages_v, first_pos, q_out, q_weight, k_weight, norm_eps, stream)):
        return q_out
    n = _int32(next((x.shape[2] for x in (q, k, v) if x is not None), 0), "rows")
    pool = pages_k if pages_k is not None else pages_v
    none, no_pages = _CTensor(None, 0, 0, 0), _CPages(None, 0, 0, 0, 0)
    pages = None if pool is None else tuple(pool.shape[2:4])
    if pages is not None and len(pages) != 2:
        raise KVCommError(EINVAL, "pages_k / pages_v: expected 5-d device tensors [L, Hkv, pages, slots, D]")
    cin, cpool, cout = [none] * 3, [no_pages] * 2, none
    for i, (x, y, what) in enumerate(((q, q_out, "q"), (k, pages_k, "k"), (v, pages_v, "v"))):
        if (x is None) != (y is None):
            raise KVCommError(EINVAL, f"{what} without its place" if y is None else f"a place without {what}")
        if x is None:
            continue
        shape = (model.n_layers, model.n_kv_heads if i else model.n_q_heads, n, model.head_dim)
        cin[i] = _sized(x, model.dtype, shape, what)
        if i:
            cpool[i - 1] = _pool(model, y, pages, "pages_" + what)
        else:
            cout = _sized(y, model.dtype, shape, "q_out")
    cbatch = _batch(batch, n, 16 if pages is None else pages[1], 0 if pages is None else pages[0])
    weights = _norm_weights(model, q_weight, k_weight, norm_eps)
    _check(lib.kvcomm_place_qkv_paged(ctypes.byref(model.c()), *cin, ctypes.byref(cbatch), _int32(first_pos, "first_pos"), weights[0][0], weights[1][0],
                                      weights[0][1], weights[1][1], float(norm_eps), cout, *cpool,
                                      _on_stream_of((q, k, v, q_out, pages_k, pages_v, q_weight, k_weight, batch.table, batch.lens, batch.starts), stream)))
    return q_out


def _pages_of(model, pages_k, pages_v):
    ck = _pool(model, pages_k, None, "pages_k")
    return ck, _pool(model, pages_v, tuple(pages_k.shape[2:4]), "pages_v")


def kvcomm_paged_attn_workspace(model, n_rows, page_size, n_pages, batch):
    return int(load_library().kvcomm_paged_attn_workspace(ctypes.byref(model.c()), ctypes.byref(_batch(batch, n_rows, page_size, n_pages))))


def kvcomm_paged_attn_prefix_workspace(model, n_prefix, n_rows, page_size, n_pages, batch):
    return int(load_library().kvcomm_paged_attn_prefix_workspace(ctypes.byref(model.c()), _int32(n_prefix, "n_prefix"),
                                                                 ctypes.byref(_batch(batch, n_rows, page_size, n_pages))))


def _paged_attn(model, q, prefix_k, prefix_v, pages_k, pages_v, batch, softmax_scale, out, lse_out, want_lse, stream, workspace):
    """Both attention calls; prefix_k None: without a prefix."""
    lib = load_library()
    if out is None or (want_lse and lse_out is None):
        made = out is None, lse_out is None
        out, lse_out = _attn_outputs(q, out, lse_out, want_lse, stream)
        if batch.starts is not None:   # rows of no sequence stay as they were: zeros
            with on_stream(stream):
                for t, new in zip((out, lse_out), made):
                    if new and t is not None:
                        t.zero_()
    need = 0   # bytes of scratch to be made here; None: the native module has declined the call
    if workspace is None:
        need = _native.paged_attn_workspace(model, q, prefix_k, prefix_v, pages_k, pages_v, batch)
        workspace = _attn_scratch(need, q.device, stream) if need else None
    if need is not None and _done(_native.paged_attn(model, q, prefix_k, prefix_v, pages_k, pages_v, batch, softmax_scale, out, lse_out, workspace, stream)):
        return (out, lse_out) if want_lse else out
    ck, cv = _pages_of(model, pages_k, pages_v)
    n = _int32(q.shape[2], "rows")
    cbatch, cmodel = _batch(batch, n, pages_k.shape[3], pages_k.shape[2]), model.c()
    prefix = ()
    if prefix_k is not None:
        shape = (model.n_layers, model.n_kv_heads, prefix_k.shape[2], model.head_dim)
        prefix = (_sized(prefix_k, model.dtype, shape, "prefix_k"), _sized(prefix_v, model.dtype, shape, "prefix_v"), _int32(shape[2], "n_prefix"))
    if workspace is None:
        need = (lib.kvcomm_paged_attn_prefix_workspace(ctypes.byref(cmodel), prefix[2], ctypes.byref(cbatch)) if prefix else
                lib.kvcomm_paged_attn_workspace(ctypes.byref(cmodel), ctypes.byref(cbatch)))
        workspace = _attn_scratch(need, q.device, stream) if need else None
    cq, cout, lse, ws = _attn_checked(model, q, out, lse_out, workspace)
    call = lib.kvcomm_paged_attn_prefix if prefix else lib.kvcomm_paged_attn
    _check(call(ctypes.byref(cmodel), cq, *prefix, ck, cv, ctypes.byref(cbatch), float(softmax_scale), cout, lse, *ws,
                _on_stream_of((q, prefix_k, prefix_v, pages_k, pages_v, out, lse_out, workspace, batch.table, batch.lens, batch.starts), stream)))
    return (out, lse_out) if want_lse else out


def kvcomm_paged_attn(model, q, pages_k, pages_v, batch, softmax_scale=0.0, out=None, lse_out=None, want_lse=False, stream=None, workspace=None):
    """Causal attention of a batch's new tokens q [L,Hq,n,D] over their sequences' pages, pools [L,Hkv,pages,slots,D].

    workspace: kvcomm_paged_attn_workspace() bytes on the device (made here if not given)."""
    return _paged_attn(model, q, None, None, pages_k, pages_v, batch, softmax_scale, out, lse_out, want_lse, stream, workspace)


def kvcomm_paged_attn_prefix(model, q, prefix_k, prefix_v, pages_k, pages_v, batch, softmax_scale=0.0, out=None, lse_out=None, want_lse=False,
                             stream=None, workspace=None):
    """kvcomm_paged_attn of sequences that all continue the tokens prefix_k, prefix_v [L,Hkv,n_prefix,D], which every row sees.

    workspace: kvcomm_paged_attn_prefix_workspace() bytes on the device (made here if not given)."""
    if prefix_k is None or prefix_v is None:
        raise KVCommError(EINVAL, "prefix_k, prefix_v: a batch without a prefix goes through kvcomm_paged_attn")
    return _paged_attn(model, q, prefix_k, prefix_v, pages_k, pages_v, batch, softmax_scale, out, lse_out, want_lse, stream, workspace)
