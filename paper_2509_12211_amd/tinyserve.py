"""Thin ctypes binding over libtinyserve_hip.so (C ABI in include/tinyserve.h).

Argument marshalling only: every step of the decode path runs in the HIP
kernels.  Tensors are torch CUDA(ROCm) tensors used purely as device buffers;
the launch goes to torch's current stream.  There is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtinyserve_hip.so")

TS_OK = 0
TS_ERR_NULL = -1
TS_ERR_SHAPE = -2
TS_ERR_UNSUPPORTED = -3
TS_ERR_WORKSPACE = -4
TS_ERR_LAUNCH = -5
TS_ERR_DEVICE = -6
TS_OUT_F32 = 0
TS_OUT_BF16 = 1
TS_KV_BF16 = 0
TS_KV_INT8 = 1
TS_KV_FP16 = 2
TS_KV_FP4 = 3
TS_LENS_KEEP = 0
TS_LENS_ADVANCE = 1
TS_LENS_AFTER = 2
MAX_AXES = 4

EXPORTS = [
    "ts_build_page_meta", "ts_append_token_meta", "ts_score_pages", "ts_select_topk_pages",
    "ts_sparse_decode_attention", "ts_query_aware_decode", "ts_append_and_decode",
    "ts_append_and_decode_launches", "ts_dense_workspace_bytes", "ts_dense_decode_attention", "ts_workspace_bytes",
    "ts_workspace_init", "ts_workspace_status", "ts_set_tuning", "ts_strerror", "ts_version",
    "ts_debug_xcc_ids", "ts_query_aware_decode_static", "ts_rotate_rows", "ts_append_rows",
]


class TsLayout(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32),
        ("num_phys_pages", ctypes.c_int32), ("kv_tile_stride", ctypes.c_int32),
        ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
        ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("page_min", ctypes.c_void_p), ("page_max", ctypes.c_void_p),
        ("keep_first_pages", ctypes.c_int32), ("keep_last_pages", ctypes.c_int32),
        ("out_format", ctypes.c_int32), ("kv_format", ctypes.c_int32),
        ("cluster_size", ctypes.c_int32), ("wait_limit", ctypes.c_int32),
        ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
    ]


class TsRotary(ctypes.Structure):
    _fields_ = [
        ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
        ("num_axes", ctypes.c_int32), ("num_positions", ctypes.c_int32),
        ("cos_sin", ctypes.c_void_p), ("positions", ctypes.c_void_p),
        ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p),
        ("norm_eps", ctypes.c_float), ("axis_of_pair", ctypes.c_uint8 * 64),
    ]


class TsRows(ctypes.Structure):
    _fields_ = [
        ("num_tokens", ctypes.c_int32), ("format", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
        ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64),
    ]


class TinyServeError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


_lib = None


def lib():
    """The loaded C-ABI library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it first "
                "(python -c 'import __graft_entry__ as g; g.build()'); there is no CPU fallback")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
        lp = ctypes.POINTER(TsLayout)
        L.ts_build_page_meta.argtypes = [lp, vp]
        L.ts_append_token_meta.argtypes = [lp, vp, vp, ctypes.c_int, vp]
        L.ts_score_pages.argtypes = [lp, vp, vp, vp]
        L.ts_select_topk_pages.argtypes = [lp, vp, i32, vp, i32, vp, vp, vp]
        L.ts_sparse_decode_attention.argtypes = [lp, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp]
        L.ts_query_aware_decode.argtypes = [lp, vp, i32, vp, i32, f32, vp, vp, vp, vp, vp, sz, vp]
        L.ts_query_aware_decode_static.argtypes = [lp, vp, i32, vp, i32, f32, vp, vp, vp, vp, vp]
        L.ts_append_and_decode.argtypes = [lp, vp, vp, vp, i32, vp, i32, f32, vp, vp, vp, vp, vp, sz, vp]
        L.ts_append_and_decode_launches.argtypes = [lp, i32]
        L.ts_dense_workspace_bytes.argtypes = [lp]
        L.ts_dense_workspace_bytes.restype = sz
        L.ts_dense_decode_attention.argtypes = [lp, vp, f32, vp, vp, vp, sz, vp]
        L.ts_workspace_bytes.argtypes = [lp, i32]
        L.ts_workspace_bytes.restype = sz
        L.ts_workspace_init.argtypes = [vp, sz, vp]
        L.ts_workspace_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
        rows = ctypes.c_char_p      # (a packed TsRows)
        L.ts_rotate_rows.argtypes = [ctypes.POINTER(TsRotary), rows, i32, i32, i32, vp]
        L.ts_append_rows.argtypes = [lp, ctypes.POINTER(TsRotary), rows, vp, i32, vp]
        L.ts_set_tuning.argtypes = [i32, i32, i32]
        L.ts_debug_xcc_ids.argtypes = [vp, i32, vp]
        L.ts_strerror.argtypes = [ctypes.c_int]
        L.ts_strerror.restype = ctypes.c_char_p
        L.ts_version.restype = ctypes.c_int
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().ts_strerror(int(status)).decode()


# What stands between a decode step and its launch is paid on every call, and the smallest
# kernels behind these calls take 5 us: pointers are handed to ctypes as plain integers (the
# argtypes convert them; a c_void_p object each took 0.1 us), and the stream comes from the
# raw-handle query instead of a torch.cuda.Stream object (0.1 against 2.9 us a call).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream_on(device, where):
    """The current stream, of the device that the tensors are on."""
    if device < 0 or device != torch._C._cuda_getDevice():
        raise TinyServeError(TS_ERR_DEVICE, where)
    return torch._C._cuda_getCurrentRawStream(device)


def _check(status, where):
    if status != TS_OK:
        raise TinyServeError(status, where)


def make_layout(B, Hq, Hkv, d, S, P_max, k_pool, v_pool, block_table, seq_lens, page_min,
                page_max, keep_first_pages=0, keep_last_pages=0, out_format=TS_OUT_F32,
                k_scale=None, v_scale=None, cluster_size=0, wait_limit=0) -> TsLayout:
    """Fill the C struct; tensors must stay alive while calls using it are in flight.
    int8 pools (with k_scale / v_scale) select the INT8 cache format, float16 pools the
    FP16 one (q, new tokens and metadata must then be float16 too), a uint8 k_pool
    [n_phys][Hkv][S * (d + 4) bytes or more] with v_pool None the 4-bit one (new_fp4_pool)."""
    n_phys = 0 if k_pool is None else k_pool.shape[0]
    tile_stride = 0
    if k_pool is not None and Hkv > 1:
        # [n_phys][Hkv][...]: distance between the tiles of two heads (S*d for dense pools,
        # 2*S*d when the K and V tiles of a page are interleaved in one allocation)
        tile_stride = int(k_pool.stride(1))
        assert k_pool.stride(0) == Hkv * tile_stride and (v_pool is None or v_pool.stride(1) == tile_stride)
    elif k_pool is not None:
        tile_stride = int(k_pool.stride(0))
    lay = TsLayout(B, Hq, Hkv, d, S, P_max, n_phys, tile_stride,
                   None if k_pool is None else k_pool.data_ptr(),
                   None if v_pool is None else v_pool.data_ptr(),
                   None if block_table is None else block_table.data_ptr(),
                   None if seq_lens is None else seq_lens.data_ptr(),
                   None if page_min is None else page_min.data_ptr(),
                   None if page_max is None else page_max.data_ptr(),
                   int(keep_first_pages), int(keep_last_pages), int(out_format),
                   (TS_KV_BF16 if k_pool is None else
                    {torch.int8: TS_KV_INT8, torch.float16: TS_KV_FP16, torch.uint8: TS_KV_FP4}.get(k_pool.dtype, TS_KV_BF16)),
                   int(cluster_size), int(wait_limit),
                   None if k_scale is None else k_scale.data_ptr(),
                   None if v_scale is None else v_scale.data_ptr())
    return lay


def fp4_block_bytes(S, d) -> int:
    """Bytes of one (page, KV head) block of the 4-bit cache."""
    return S * (d + 4)


def new_fp4_pool(num_phys_pages, Hkv, S, d, device) -> torch.Tensor:
    """An empty 4-bit cache: uint8 [num_phys_pages][Hkv][fp4_block_bytes], the k_pool of make_layout."""
    return torch.zeros((num_phys_pages, Hkv, fp4_block_bytes(S, d)), dtype=torch.uint8, device=device)


def rotary_table(num_positions, rot_dim, base=10000.0, device="cuda") -> torch.Tensor:
    """cos_sin for positions 0 .. num_positions - 1 with frequencies base ** (-2 i / rot_dim), worked
    out in 64 bits.  (Any other table, of scaled or stretched positions, serves as well.)"""
    i = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    at = torch.arange(num_positions, dtype=torch.float64, device=device)[:, None] * base ** (-2.0 * i / rot_dim)
    return torch.cat([at.cos(), at.sin()], dim=1).float().contiguous()


def make_rotary(cos_sin=None, positions=None, interleaved=False, axis_of_pair=None, q_norm=None, k_norm=None,
                norm_eps=1e-6) -> TsRotary:
    """Norm and rotation of rows.  cos_sin: fp32 [num_positions][rot_dim] (None: no rotation).
    positions: int32 [num_tokens] or [num_axes][num_tokens]; with several axes axis_of_pair says for
    each of the rot_dim / 2 pairs which one it turns by.  q_norm, k_norm: fp32 [d] (None: no norm).
    The tensors are held by the struct."""
    axes = 1 if positions is None or positions.dim() == 1 else positions.shape[0]
    rows, rot = (0, 0) if cos_sin is None else cos_sin.shape
    held = [(t, dtype) for t, dtype in ((cos_sin, torch.float32), (positions, torch.int32), (q_norm, torch.float32),
                                        (k_norm, torch.float32)) if t is not None]
    for t, dtype in held:
        if t.dtype != dtype or not t.is_contiguous():
            raise TinyServeError(TS_ERR_SHAPE, "make_rotary")
    devices = {t.get_device() for t, _ in held}
    if len(devices) > 1:
        raise TinyServeError(TS_ERR_DEVICE, "make_rotary")
    r = TsRotary(rot, int(interleaved), axes, rows, _ptr(cos_sin), _ptr(positions), _ptr(q_norm), _ptr(k_norm),
                 float(norm_eps))
    if axes > 1:
        if axis_of_pair is None or len(axis_of_pair) != rot // 2:
            raise TinyServeError(TS_ERR_SHAPE, "make_rotary")
        r.axis_of_pair[:rot // 2] = [int(a) for a in axis_of_pair]
    r.held = (cos_sin, positions, q_norm, k_norm)
    r.tokens = None if positions is None else positions.shape[-1]
    r.device = devices.pop() if devices else None
    r.norm_dim = {t.numel() for t in (q_norm, k_norm) if t is not None}
    return r


# (The calls of a decode step: a struct packed by format takes a third of what one of ctypes' own does.)
_pack_rows = struct.Struct("=ii5Q5q").pack
_ROW_FORMATS = {torch.bfloat16: TS_KV_BF16, torch.float16: TS_KV_FP16}


def _row_stride(t, shape, dtype, device, where):
    """Elements between the tokens of rows [num_tokens][heads][d], which shape, dtype and device they must have."""
    s = t.stride()
    if t.get_device() != device:
        raise TinyServeError(TS_ERR_DEVICE, where)
    if t.shape != shape or t.dtype != dtype or s[2] != 1 or (s[1] != shape[2] and shape[1] > 1):
        raise TinyServeError(TS_ERR_SHAPE, where)
    return s[0]


def _check_rotary(rotary, tokens, d, device, where):
    if rotary.device is not None and rotary.device != device:
        raise TinyServeError(TS_ERR_DEVICE, where)
    if (rotary.tokens is not None and rotary.tokens != tokens) or (rotary.norm_dim and rotary.norm_dim != {d}):
        raise TinyServeError(TS_ERR_SHAPE, where)


def rotate_rows(rotary, q, k, q_out=None, k_out=None):
    """Per-head norm and rotation of q [num_tokens][Hq][d] and k [num_tokens][Hkv][d] (either may be
    None), which may be slices of one projection's rows; in place where no output is given."""
    where = "ts_rotate_rows"
    one = q if q is not None else k
    dtype = None if one is None else one.dtype
    if dtype not in _ROW_FORMATS:
        raise TinyServeError(TS_ERR_NULL if one is None else TS_ERR_UNSUPPORTED, where)
    shape = one.shape
    if len(shape) != 3:
        raise TinyServeError(TS_ERR_SHAPE, where)
    n, _, d = shape
    device = one.get_device()
    _check_rotary(rotary, n, d, device, where)
    Hq = Hkv = qs = ks = qos = kos = qp = kp = qop = kop = 0
    if q is not None:
        Hq, qp = shape[1], q.data_ptr()
        qs = qos = _row_stride(q, shape, dtype, device, where)
        qop = qp
        if q_out is not None:
            qos, qop = _row_stride(q_out, shape, dtype, device, where), q_out.data_ptr()
    if k is not None:
        shape = k.shape
        if len(shape) != 3 or shape[0] != n or shape[2] != d:
            raise TinyServeError(TS_ERR_SHAPE, where)
        Hkv, kp = shape[1], k.data_ptr()
        ks = kos = _row_stride(k, shape, dtype, device, where)
        kop = kp
        if k_out is not None:
            kos, kop = _row_stride(k_out, shape, dtype, device, where), k_out.data_ptr()
    if n == 0:        # (rows of no tokens have no address)
        return
    rows = _pack_rows(n, _ROW_FORMATS[dtype], qp, kp, 0, qop, kop, qs, ks, 0, qos, kos)
    _check(lib().ts_rotate_rows(ctypes.byref(rotary), rows, Hq, Hkv, d, _stream_on(device, where)), where)


def append_rows(layout, k, v, rotary=None, q=None, q_out=None, cu_tokens=None, advance_seq_lens=True,
                lens_include_new=False):
    """Append k, v [num_tokens][Hkv][d] to the cache, normed and rotated on the way (rotary), one token
    for each sequence or, with cu_tokens (int32 [num_seqs + 1], on the device), any number; q
    [num_tokens][Hq][d] is normed and rotated into q_out (in place if none is given) in the same
    launch.  lens_include_new: the layout's lengths count the new tokens already."""
    where = "ts_append_rows"
    dtype, shape = k.dtype, k.shape
    if dtype != (torch.float16 if layout.kv_format == TS_KV_FP16 else torch.bfloat16):
        raise TinyServeError(TS_ERR_UNSUPPORTED, where)
    if len(shape) != 3 or shape[1] != layout.num_kv_heads or shape[2] != layout.head_dim or (
            shape[0] != layout.num_seqs if cu_tokens is None else
            cu_tokens.get_device() != k.get_device() or cu_tokens.dtype != torch.int32 or cu_tokens.numel() != layout.num_seqs + 1 or not cu_tokens.is_contiguous()):
        raise TinyServeError(TS_ERR_SHAPE, where)
    n, _, d = shape
    device, ref = k.get_device(), None
    if rotary is not None:
        _check_rotary(rotary, n, d, device, where)
        ref = ctypes.byref(rotary)
    ks, vs = _row_stride(k, shape, dtype, device, where), _row_stride(v, shape, dtype, device, where)
    qs = qos = qp = qop = 0
    if q is not None:
        shape = (n, layout.num_q_heads, d)
        qp = qop = q.data_ptr()
        qs = qos = _row_stride(q, shape, dtype, device, where)
        if q_out is not None:
            qos, qop = _row_stride(q_out, shape, dtype, device, where), q_out.data_ptr()
    if n == 0:
        return
    lens = TS_LENS_AFTER if lens_include_new else TS_LENS_ADVANCE if advance_seq_lens else TS_LENS_KEEP
    rows = _pack_rows(n, 0, qp, k.data_ptr(), v.data_ptr(), qop, 0, qs, ks, vs, qos, 0)
    _check(lib().ts_append_rows(ctypes.byref(layout), ref, rows, None if cu_tokens is None else cu_tokens.data_ptr(),
                                lens, _stream_on(device, where)), where)


def build_page_meta(layout):
    _check(lib().ts_build_page_meta(ctypes.byref(layout), _stream()), "ts_build_page_meta")


def append_token_meta(layout, k_new, v_new=None, advance_seq_lens=True):
    _check(lib().ts_append_token_meta(ctypes.byref(layout), _ptr(k_new), _ptr(v_new),
                                      1 if advance_seq_lens else 0, _stream()),
           "ts_append_token_meta")


def score_pages(layout, q, scores):
    _check(lib().ts_score_pages(ctypes.byref(layout), _ptr(q), _ptr(scores), _stream()),
           "ts_score_pages")


def select_topk_pages(layout, scores, topk, max_topk, sel, sel_count, topk_per_seq=None):
    _check(lib().ts_select_topk_pages(ctypes.byref(layout), _ptr(scores), int(topk),
                                      _ptr(topk_per_seq), int(max_topk), _ptr(sel),
                                      _ptr(sel_count), _stream()), "ts_select_topk_pages")


def workspace_bytes(layout, max_topk) -> int:
    return int(lib().ts_workspace_bytes(ctypes.byref(layout), int(max_topk)))


def workspace_init(workspace):
    _check(lib().ts_workspace_init(_ptr(workspace), workspace.nbytes,
                                   _stream()), "ts_workspace_init")


def workspace_status(workspace) -> int:
    v = ctypes.c_int32(0)
    _check(lib().ts_workspace_status(_ptr(workspace), ctypes.byref(v)), "ts_workspace_status")
    return int(v.value)


def new_workspace(layout, max_topk, device) -> torch.Tensor:
    """Allocate (with torch) and initialise a workspace for this layout."""
    n = workspace_bytes(layout, max_topk)
    if n == 0:
        raise TinyServeError(TS_ERR_SHAPE, "ts_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    workspace_init(ws)
    return ws


def sparse_decode_attention(layout, q, sel, sel_count, max_topk, softmax_scale, out, workspace,
                            lse_out=None):
    _check(lib().ts_sparse_decode_attention(
        ctypes.byref(layout), _ptr(q), _ptr(sel), _ptr(sel_count), int(max_topk),
        float(softmax_scale), _ptr(out), _ptr(lse_out), _ptr(workspace), workspace.nbytes,
        _stream()), "ts_sparse_decode_attention")


def query_aware_decode(layout, q, topk, max_topk, softmax_scale, out, workspace,
                       topk_per_seq=None, scores_out=None, sel_out=None, sel_count_out=None):
    _check(lib().ts_query_aware_decode(
        ctypes.byref(layout), _ptr(q), int(topk), _ptr(topk_per_seq), int(max_topk),
        float(softmax_scale), _ptr(out), _ptr(scores_out), _ptr(sel_out), _ptr(sel_count_out),
        _ptr(workspace), workspace.nbytes, _stream()),
        "ts_query_aware_decode")


STATIC_WORKSPACE_BYTES = 4 << 20


def query_aware_decode_static(layout, q, topk, max_topk, softmax_scale, out, topk_per_seq=None,
                              scores_out=None, sel_out=None, sel_count_out=None):
    """ts_query_aware_decode on the library's own fixed workspace (allocates nothing)."""
    _check(lib().ts_query_aware_decode_static(
        ctypes.byref(layout), _ptr(q), int(topk), _ptr(topk_per_seq), int(max_topk),
        float(softmax_scale), _ptr(out), _ptr(scores_out), _ptr(sel_out), _ptr(sel_count_out),
        _stream()), "ts_query_aware_decode_static")


def append_and_decode(layout, k_new, v_new, q, topk, max_topk, softmax_scale, out, workspace,
                      topk_per_seq=None, scores_out=None, sel_out=None, sel_count_out=None):
    _check(lib().ts_append_and_decode(
        ctypes.byref(layout), _ptr(k_new), _ptr(v_new), _ptr(q), int(topk), _ptr(topk_per_seq),
        int(max_topk), float(softmax_scale), _ptr(out), _ptr(scores_out), _ptr(sel_out),
        _ptr(sel_count_out), _ptr(workspace), workspace.nbytes,
        _stream()), "ts_append_and_decode")


def new_dense_workspace(layout, device) -> torch.Tensor:
    n = int(lib().ts_dense_workspace_bytes(ctypes.byref(layout)))
    if n == 0:
        raise TinyServeError(TS_ERR_SHAPE, "ts_dense_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    workspace_init(ws)
    return ws


def dense_decode_attention(layout, q, softmax_scale, out, workspace, lse_out=None):
    _check(lib().ts_dense_decode_attention(
        ctypes.byref(layout), _ptr(q), float(softmax_scale), _ptr(out), _ptr(lse_out),
        _ptr(workspace),
        workspace.nbytes, _stream()), "ts_dense_decode_attention")


def append_and_decode_launches(layout, max_topk) -> int:
    n = int(lib().ts_append_and_decode_launches(ctypes.byref(layout), int(max_topk)))
    if n < 0:
        raise TinyServeError(n, "ts_append_and_decode_launches")
    return n


def debug_xcc_ids(num_workgroups, device) -> torch.Tensor:
    """int32 [num_workgroups]: the XCD each workgroup of a probe launch ran on."""
    ids = torch.full((int(num_workgroups),), -1, dtype=torch.int32, device=device)
    _check(lib().ts_debug_xcc_ids(_ptr(ids), int(num_workgroups), _stream()), "ts_debug_xcc_ids")
    return ids


def set_tuning(reserved=0, num_splits=0, workgroups_per_cu=0):
    _check(lib().ts_set_tuning(int(reserved), int(num_splits),
                               int(workgroups_per_cu)), "ts_set_tuning")
