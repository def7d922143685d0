"""Thin ctypes binding over libhexi_attn.so (the C ABI of include/hexi_attn.h).

Argument marshalling only: every step of the attention path runs in the library's HIP kernels.
Tensors are torch tensors used as device-memory handles (``data_ptr()``); the stream is torch's
current HIP stream unless given.  There is no CPU fallback: if the library has not been built,
loading raises.
"""
import ctypes
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

HEXI_OK = 0
HEXI_EINVAL, HEXI_EUNSUPPORTED, HEXI_EALIGN, HEXI_EWORKSPACE, HEXI_EHIP, HEXI_EINFEASIBLE = -1, -2, -3, -4, -5, -6
HEXI_BF16, HEXI_F32 = 0, 1
HEXI_ACCUMULATE, HEXI_COMPUTE_DELTA, HEXI_SKIP_DQ, HEXI_SKIP_DKDV = 1, 2, 4, 8
HEXI_TILE_EMPTY, HEXI_TILE_FULL, HEXI_TILE_PARTIAL = 0, 1, 2
HEXI_MAX_SEGS = 16
HEXI_ROPE_HALF, HEXI_ROPE_ADJACENT, HEXI_ROPE_INVERSE = 0, 1, 16

EXPORTS = ("hexi_shard_mask", "hexi_attn_fwd_chunk", "hexi_attn_merge_lse", "hexi_attn_bwd_chunk",
           "hexi_attn_win_workspace_bytes", "hexi_attn_win_fwd_chunk", "hexi_attn_win_bwd_workspace_bytes", "hexi_attn_win_bwd_chunk", "hexi_rope", "hexi_rope_a2a_pack", "hexi_rope_a2a_unpack",
           "hexi_a2a_pack", "hexi_a2a_unpack", "hexi_sched_cost", "hexi_sched_solve", "hexi_set_dkdv_run_len", "hexi_workspace_bytes", "hexi_last_error", "hexi_version")

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhexi_attn.so")
PROBE_LIB_PATH = os.path.join(_HERE, "libhexi_probe.so")     # include/hexi_probe.h: the benchmark's MFMA rate probe
PROBE_EXPORTS = ("hexi_mfma_probe",)
_lib = None
_probe_lib = None


class HexiError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"hexi error {code}: {msg}")
        self.code = code


class hexi_seg(ctypes.Structure):
    _fields_ = [("start", ctypes.c_int64), ("len", ctypes.c_int64)]


class hexi_range(ctypes.Structure):
    _fields_ = [("n_segs", ctypes.c_int32), ("segs", ctypes.POINTER(hexi_seg))]


class hexi_attn_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("kv_of_q", ctypes.POINTER(ctypes.c_int32)), ("softmax_scale", ctypes.c_float),
                ("q_stride_tok", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("kv_stride_tok", ctypes.c_int64), ("kv_stride_head", ctypes.c_int64)]


class hexi_window(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int64), ("n_sink", ctypes.c_int64)]


class hexi_rope_desc(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("pairing", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("inv_freq", ctypes.POINTER(ctypes.c_double)), ("axis_of_pair", ctypes.POINTER(ctypes.c_int8))]


class hexi_rope_tensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("n_heads", ctypes.c_int32),
                ("x_stride_tok", ctypes.c_int64), ("x_stride_head", ctypes.c_int64), ("y_stride_tok", ctypes.c_int64), ("y_stride_head", ctypes.c_int64)]


def load():
    """Loads the in-tree library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_07569_amd.build` "
                           "(hipcc, gfx950); there is no CPU fallback")
    import torch  # noqa: F401  (loads the HIP runtime the library binds to)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    rp, dp = ctypes.POINTER(hexi_range), ctypes.POINTER(hexi_attn_desc)
    lib.hexi_shard_mask.argtypes = [rp, rp, i32, i32, vp, vp, vp, ctypes.POINTER(i64)]
    lib.hexi_shard_mask.restype = ctypes.c_int
    lib.hexi_attn_fwd_chunk.argtypes = [dp, rp, rp, vp, vp, vp, vp, vp, u32, vp, ctypes.c_size_t, vp]
    lib.hexi_attn_fwd_chunk.restype = ctypes.c_int
    lib.hexi_attn_merge_lse.argtypes = [i64, i32, i32, vp, vp, vp, vp, vp, i32, vp]
    lib.hexi_attn_merge_lse.restype = ctypes.c_int
    lib.hexi_attn_bwd_chunk.argtypes = [dp, rp, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, u32, vp, ctypes.c_size_t, vp]
    lib.hexi_attn_bwd_chunk.restype = ctypes.c_int
    wp = ctypes.POINTER(hexi_window)
    lib.hexi_attn_win_workspace_bytes.argtypes = [dp, wp, i64, i64]
    lib.hexi_attn_win_workspace_bytes.restype = ctypes.c_size_t
    lib.hexi_attn_win_fwd_chunk.argtypes = [dp, wp, rp, rp, vp, vp, vp, vp, i32, vp, u32, vp, ctypes.c_size_t, vp]
    lib.hexi_attn_win_fwd_chunk.restype = ctypes.c_int
    lib.hexi_attn_win_bwd_chunk.argtypes = [dp, wp, rp, rp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, u32, vp, ctypes.c_size_t, vp]
    lib.hexi_attn_win_bwd_workspace_bytes.argtypes = [dp, wp, i64, i64]
    lib.hexi_attn_win_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.hexi_attn_win_bwd_chunk.restype = ctypes.c_int
    i32p = ctypes.POINTER(i32)
    op = ctypes.POINTER(hexi_rope_desc)
    lib.hexi_rope.argtypes = [op, rp, vp, i64, ctypes.POINTER(hexi_rope_tensor), i32, i32, i32, u32, vp]
    lib.hexi_rope.restype = ctypes.c_int
    for fn in (lib.hexi_rope_a2a_pack, lib.hexi_rope_a2a_unpack):
        fn.argtypes = [op, rp, vp, i64, vp, vp, i32, i32, i64, i32, i32p, i32p, ctypes.POINTER(ctypes.c_uint8), u32, vp]
        fn.restype = ctypes.c_int
    lib.hexi_a2a_pack.argtypes = [vp, vp, i64, i32, i32, i32, i64, i32, i32p, i32p, vp]
    lib.hexi_a2a_pack.restype = ctypes.c_int
    lib.hexi_a2a_unpack.argtypes = [vp, vp, i64, i32, i32, i32, i64, i32, i32p, i32p, vp]
    lib.hexi_a2a_unpack.restype = ctypes.c_int
    lib.hexi_sched_cost.argtypes = [vp, vp, vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)]
    lib.hexi_sched_cost.restype = ctypes.c_int
    lib.hexi_sched_solve.argtypes = [vp, vp, vp, vp, ctypes.POINTER(ctypes.c_double)]
    lib.hexi_sched_solve.restype = ctypes.c_int
    lib.hexi_set_dkdv_run_len.argtypes = [i32]
    lib.hexi_set_dkdv_run_len.restype = i32
    lib.hexi_workspace_bytes.argtypes = [dp, i64, i64]
    lib.hexi_workspace_bytes.restype = ctypes.c_size_t
    lib.hexi_last_error.restype = ctypes.c_char_p
    lib.hexi_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def load_probe():
    """Loads the benchmark's measurement-aid library (not part of the attention interface)."""
    global _probe_lib
    if _probe_lib is None:
        if not os.path.exists(PROBE_LIB_PATH):
            raise RuntimeError(f"{PROBE_LIB_PATH} is missing: build it with `python -m paper_2605_07569_amd.build`")
        import torch  # noqa: F401
        lib = ctypes.CDLL(PROBE_LIB_PATH)
        lib.hexi_mfma_probe.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p]
        lib.hexi_mfma_probe.restype = ctypes.c_int
        _probe_lib = lib
    return _probe_lib


def _check(rc):
    if rc != HEXI_OK:
        raise HexiError(rc, load().hexi_last_error().decode())


def make_range(segs: Sequence[Tuple[int, int]]):
    """[(start, len), ...] -> (hexi_range, keepalive).  A hexi_range made here is passed through: the calls below that take a
    segment list take one in its place (building it is most of a small call's host time: 3.5 us of about 11)."""
    if isinstance(segs, hexi_range):
        return segs, segs
    arr = (hexi_seg * max(1, len(segs)))(*[(int(s), int(n)) for s, n in segs])
    r = hexi_range(len(segs), arr)
    r._keep = arr
    return r, arr


def _with_rows(segs):
    """A range and its rows (whatever is wrong with a range the library says)."""
    r = segs if isinstance(segs, hexi_range) else make_range(segs)[0]
    n = r.n_segs
    if n == 1:
        return r, r.segs[0].len
    return r, sum(r.segs[i].len for i in range(max(0, min(n, HEXI_MAX_SEGS))))


def make_desc(dtype, head_dim, n_q_heads, n_kv_heads, softmax_scale, q_strides, kv_strides, kv_of_q=None):
    """q_strides / kv_strides: (token stride, head stride) in elements."""
    keep = None
    ptr = ctypes.POINTER(ctypes.c_int32)()
    if kv_of_q is not None:
        keep = (ctypes.c_int32 * len(kv_of_q))(*[int(x) for x in kv_of_q])
        ptr = ctypes.cast(keep, ctypes.POINTER(ctypes.c_int32))
    d = hexi_attn_desc(int(dtype), int(head_dim), int(n_q_heads), int(n_kv_heads), ptr, float(softmax_scale),
                       int(q_strides[0]), int(q_strides[1]), int(kv_strides[0]), int(kv_strides[1]))
    d._keep = keep
    return d


def desc_for(q, k, softmax_scale, kv_of_q=None):
    """Descriptor for torch tensors q [Lq, nq, d] and k [Lc, nkv, d] (d contiguous)."""
    import torch
    assert q.dim() == 3 and k.dim() == 3 and q.stride(2) == 1 and k.stride(2) == 1
    dt = {torch.bfloat16: HEXI_BF16, torch.float32: HEXI_F32}[q.dtype]
    return make_desc(dt, q.shape[2], q.shape[1], k.shape[1], softmax_scale,
                     (q.stride(0), q.stride(1)), (k.stride(0), k.stride(1)), kv_of_q)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    """The stream's handle.  Asked of torch's C++ side directly: the Stream object of torch.cuda.current_stream() costs as much as the
    launch itself."""
    if stream is None:
        import torch
        if not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream)


def hexi_version():
    return load().hexi_version().decode()


def hexi_last_error():
    return load().hexi_last_error().decode()


def hexi_shard_mask(q_segs, kv_segs, tile_m=0, tile_n=0, want_pos=True, want_classes=True):
    """Host bookkeeping -> dict(q_pos, kv_pos (int32 numpy), tile_class (uint8 [nm, nn]), n_pairs)."""
    lib = load()
    qr, _k1 = make_range(q_segs)
    kr, _k2 = make_range(kv_segs)
    lq, lc = (sum(r.segs[i].len for i in range(r.n_segs)) for r in (qr, kr))
    q_pos = np.empty(max(lq, 0), dtype=np.int32) if want_pos else None
    kv_pos = np.empty(max(lc, 0), dtype=np.int32) if want_pos else None
    cls = None
    if want_classes and tile_m > 0 and tile_n > 0:
        cls = np.empty((-(-lq // tile_m), -(-lc // tile_n)), dtype=np.uint8)
    n_pairs = ctypes.c_int64(0)
    rc = lib.hexi_shard_mask(ctypes.byref(qr), ctypes.byref(kr), tile_m, tile_n,
                             None if q_pos is None else q_pos.ctypes.data_as(ctypes.c_void_p),
                             None if kv_pos is None else kv_pos.ctypes.data_as(ctypes.c_void_p),
                             None if cls is None else cls.ctypes.data_as(ctypes.c_void_p),
                             ctypes.byref(n_pairs))
    _check(rc)
    return dict(q_pos=q_pos, kv_pos=kv_pos, tile_class=cls, n_pairs=int(n_pairs.value))


def hexi_attn_fwd_chunk(desc, q_segs, kv_segs, q, k, v, o, lse, flags=0, workspace=None, stream=None):
    qr = q_segs if isinstance(q_segs, hexi_range) else make_range(q_segs)[0]
    kr = kv_segs if isinstance(kv_segs, hexi_range) else make_range(kv_segs)[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = (_lib or load()).hexi_attn_fwd_chunk(desc, qr, kr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), flags,
                                              _ptr(workspace), ws_bytes, _stream(stream))
    if rc:
        _check(rc)


def hexi_attn_merge_lse(o_acc, lse_acc, o_part, lse_part, o_final=None, stream=None):
    import torch
    n_rows, nq, d = o_acc.shape
    fdt = HEXI_F32
    if o_final is not None:
        fdt = {torch.bfloat16: HEXI_BF16, torch.float32: HEXI_F32}[o_final.dtype]
    _check(load().hexi_attn_merge_lse(n_rows, nq, d, _ptr(o_acc), _ptr(lse_acc), _ptr(o_part), _ptr(lse_part),
                                      _ptr(o_final), fdt, _stream(stream)))


def hexi_attn_bwd_chunk(desc, q_segs, kv_segs, q, k, v, o, d_o, lse, delta, dq_acc, dk, dv, flags=0,
                        workspace=None, stream=None):
    qr = q_segs if isinstance(q_segs, hexi_range) else make_range(q_segs)[0]
    kr = kv_segs if isinstance(kv_segs, hexi_range) else make_range(kv_segs)[0]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = (_lib or load()).hexi_attn_bwd_chunk(desc, qr, kr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(delta),
                                              _ptr(dq_acc), _ptr(dk), _ptr(dv), flags, _ptr(workspace), ws_bytes, _stream(stream))
    if rc:
        _check(rc)


def hexi_workspace_bytes(desc, lq, lc):
    return int(load().hexi_workspace_bytes(ctypes.byref(desc), lq, lc))


def make_window(window, n_sink=0):
    """Sliding window (the row's own token counts; >= 1) and the number of first tokens that stay visible."""
    return hexi_window(int(window), int(n_sink))


def _refuse(msg):
    raise HexiError(HEXI_EINVAL, msg)


_DTYPES = {}
_torch = None


def _types():
    """torch, and its element types by the library's codes and the other way round, at the first use."""
    global _torch
    import torch
    _DTYPES.update({torch.bfloat16: HEXI_BF16, torch.float32: HEXI_F32, HEXI_BF16: torch.bfloat16, HEXI_F32: torch.float32})
    _torch = torch


def _dtype(t):
    if _torch is None:
        _types()
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise HexiError(HEXI_EUNSUPPORTED, f"element type {t.dtype} (bf16 or fp32)")
    return code


def _current_device():
    """Index of the GPU whose stream the calls use; no tensor is on -2, where none is initialised."""
    if _torch is None:
        _types()
    return _torch._C._cuda_getDevice() if _torch.cuda.is_initialized() else -2


def _fits(name, t, shape, dtype, dev, strides=None):
    """Refuses a tensor that is not of this shape and element type (a code of the library), on the current GPU, dense or with these strides."""
    if t.shape == shape and t.dtype is _DTYPES.get(dtype) and t.get_device() == dev and (t.is_contiguous() if strides is None else t.stride() == strides):
        return
    if tuple(t.shape) != shape or _dtype(t) != dtype:
        _refuse(f"{name}: {shape} elements of type {dtype} are needed, not {tuple(t.shape)} {t.dtype}")
    if not t.is_contiguous() if strides is None else any(s != w and n > 1 for s, w, n in zip(t.stride(), strides, shape)):
        _refuse(f"{name}: strides {t.stride()}; {'a contiguous tensor is needed' if strides is None else f'the descriptor says {strides}'}")
    if t.get_device() != dev:
        _refuse(f"{name} is on {t.device}, not on the current GPU")


def _win_inputs(desc, q_segs, kv_segs, q, k, v, lse, d_o=None):
    """Ranges, rows, keys, device and sizes (head_dim, q heads, kv heads) of a windowed call, its inputs checked."""
    qr, lq = _with_rows(q_segs)
    kr, lc = _with_rows(kv_segs)
    dev = _current_device()
    dt, d, nq, nkv = desc.dtype, desc.head_dim, desc.n_q_heads, desc.n_kv_heads
    q_strides, kv_strides = (desc.q_stride_tok, desc.q_stride_head, 1), (desc.kv_stride_tok, desc.kv_stride_head, 1)
    shape = (lq, nq, d)
    _fits("q", q, shape, dt, dev, q_strides)
    if d_o is not None:
        _fits("d_o", d_o, shape, dt, dev, q_strides)
    shape = (lc, nkv, d)
    _fits("k", k, shape, dt, dev, kv_strides)
    _fits("v", v, shape, dt, dev, kv_strides)
    _fits("lse", lse, (nq, lq), HEXI_F32, dev)
    return qr, kr, lq, lc, dev, d, nq, nkv


def _bytes_of(workspace, dev):
    """Bytes of a workspace from its first element on."""
    if workspace.get_device() != dev:
        _refuse(f"workspace is on {workspace.device}, not on the current GPU")
    if not workspace.is_contiguous():
        _refuse(f"workspace: strides {workspace.stride()}; a contiguous tensor is needed")
    return workspace.numel() * workspace.element_size()


def hexi_attn_win_workspace_bytes(desc, window, lq, lc):
    return int(load().hexi_attn_win_workspace_bytes(ctypes.byref(desc), ctypes.byref(window), lq, lc))


def hexi_attn_win_bwd_workspace_bytes(desc, window, lq, lc):
    return int(load().hexi_attn_win_bwd_workspace_bytes(ctypes.byref(desc), ctypes.byref(window), lq, lc))


def hexi_attn_win_fwd_chunk(desc, window, q_segs, kv_segs, q, k, v, o, lse, flags=0, workspace=None, stream=None):
    """Windowed forward; o's element type (fp32 or bf16) is the result's.  workspace: a tensor of at least hexi_attn_win_workspace_bytes, where that is not 0."""
    qr, kr, lq, lc, dev, d, nq, nkv = _win_inputs(desc, q_segs, kv_segs, q, k, v, lse)
    o_type = _dtype(o)
    _fits("o", o, (lq, nq, d), o_type, dev)
    ws_bytes = 0 if workspace is None else _bytes_of(workspace, dev)
    rc = (_lib or load()).hexi_attn_win_fwd_chunk(desc, window, qr, kr, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), o_type, lse.data_ptr(), flags,
                                                  _ptr(workspace), ws_bytes, _stream(stream))
    if rc:
        _check(rc)


def hexi_attn_win_bwd_chunk(desc, window, q_segs, kv_segs, q, k, v, o, d_o, lse, delta, dq, dk, dv, flags=0, workspace=None, stream=None):
    """Windowed backward; the element type of dq, dk and dv (one for all; None for the half that is skipped) is the gradients'.  workspace: a tensor of at least
    hexi_attn_win_bwd_workspace_bytes; None takes one from torch for the call where one is of use (none, and a slower call whose sums have another order, on a stream given by
    hand that is being captured by other means than torch.cuda.graph)."""
    qr, kr, lq, lc, dev, d, nq, nkv = _win_inputs(desc, q_segs, kv_segs, q, k, v, lse, d_o)
    _fits("delta", delta, (nq, lq), HEXI_F32, dev)
    o_type = grad = HEXI_F32
    if o is not None:
        o_type = _dtype(o)
        _fits("o", o, (lq, nq, d), o_type, dev)
    for t in (dv, dk, dq):
        if t is not None:
            grad = _dtype(t)
    for name, t, shape in (("dq", dq, (lq, nq, d)), ("dk", dk, (lc, nkv, d)), ("dv", dv, (lc, nkv, d))):
        if t is not None:
            _fits(name, t, shape, grad, dev)
    lib, ws_bytes = _lib or load(), 0
    if workspace is not None:
        ws_bytes = _bytes_of(workspace, dev)
    elif not flags & HEXI_SKIP_DKDV:
        ws_bytes = lib.hexi_attn_win_bwd_workspace_bytes(desc, window, lq, lc)
        if ws_bytes and stream is None:
            workspace = _torch.empty(ws_bytes, dtype=_torch.uint8, device=q.device)
    space, handle = _ptr(workspace), _stream(stream)
    taken = _take(lib, ws_bytes, dev, handle) if ws_bytes and space is None else None
    try:
        rc = lib.hexi_attn_win_bwd_chunk(desc, window, qr, kr, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(o), o_type, d_o.data_ptr(), lse.data_ptr(),
                                         delta.data_ptr(), _ptr(dq), _ptr(dk), _ptr(dv), grad, flags, taken if space is None else space, ws_bytes, handle)
    finally:
        if taken is not None:
            _torch.cuda.caching_allocator_delete(taken)
    if rc:
        _check(rc)


def _take(lib, n, dev, handle):
    """n bytes from torch's allocator that belong to the stream of this handle: given back, they serve what follows on it.  None on a stream that is being captured while
    torch's current one is not: torch does not know of that graph, and would hand the bytes out again while it lives."""
    status = ctypes.c_int(0)
    if (lib.hipStreamIsCapturing(ctypes.c_void_p(handle), ctypes.byref(status)) != 0 or status.value != 0) and not _torch.cuda.is_current_stream_capturing():
        return None
    return _torch.cuda.caching_allocator_alloc(n, dev, handle)


def make_rope(head_dim, inv_freq, axis_of_pair=None, pairing="half", n_axes=None):
    """Descriptor of a rotation: a frequency per pair (rot_dim = 2 len(inv_freq)), the axis of every pair (None: axis 0), "half" or "adjacent" pairs."""
    if pairing not in ("half", "adjacent"):
        _refuse(f"pairing {pairing!r}")
    if axis_of_pair is not None and len(axis_of_pair) != len(inv_freq):
        _refuse(f"{len(axis_of_pair)} axes for {len(inv_freq)} pairs")
    freq = (ctypes.c_double * max(1, len(inv_freq)))(*[float(f) for f in inv_freq])
    axes = None if axis_of_pair is None else (ctypes.c_int8 * max(1, len(axis_of_pair)))(*[int(a) for a in axis_of_pair])
    if n_axes is None:
        n_axes = 1 if axis_of_pair is None else max(1, 1 + max([int(a) for a in axis_of_pair], default=0))
    d = hexi_rope_desc(int(head_dim), 2 * len(inv_freq), HEXI_ROPE_HALF if pairing == "half" else HEXI_ROPE_ADJACENT, int(n_axes), freq,
                       ctypes.cast(axes, ctypes.POINTER(ctypes.c_int8)) if axes is not None else ctypes.POINTER(ctypes.c_int8)())
    d._keep = (freq, axes)
    return d


def _rope_positions(rope, positions, rows, dev):
    if positions is None:
        return None, 0
    import torch
    n = rope.n_axes
    if positions.dtype != torch.int32 or tuple(positions.shape) != (n, rows) or (rows > 1 and positions.stride(1) != 1) or (n > 1 and positions.stride(0) < rows):
        _refuse(f"positions: an int32 [{n}][{rows}] tensor is needed, not {tuple(positions.shape)} {positions.dtype} with strides {positions.stride()}")
    if positions.get_device() != dev:
        _refuse(f"positions are on {positions.device}, not on the current GPU")
    return positions.data_ptr(), positions.stride(0) if n > 1 else rows


def hexi_rope(rope, segs, tensors, positions=None, inverse=False, stream=None):
    """Rotates the tensors of a shard in one launch.  tensors: [(x, y), ...], x and y [rows, heads, head_dim] with contiguous columns, y may be x; all x
    of one element type, all y of one.  positions: int32 [n_axes, rows] on the device, or None for the rows' global positions."""
    r, rows = _with_rows(segs)
    if not tensors:
        _refuse("no tensors")
    dev, d = _current_device(), rope.head_dim
    pos, pos_stride = _rope_positions(rope, positions, rows, dev)
    x_type, y_type = _dtype(tensors[0][0]), _dtype(tensors[0][1])
    arr = (hexi_rope_tensor * len(tensors))()
    for i, (x, y) in enumerate(tensors):
        shape, xs, ys = x.shape, x.stride(), y.stride()
        if len(shape) != 3 or y.shape != shape or shape[0] != rows or shape[2] != d or xs[2] != 1 or ys[2] != 1 or _dtype(x) != x_type or _dtype(y) != y_type:
            _refuse(f"a tensor pair of [{rows}, heads, {d}] and one type a side is needed, not {tuple(shape)} {x.dtype} -> {tuple(y.shape)} {y.dtype}")
        if x.get_device() != dev or y.get_device() != dev:
            _refuse(f"a tensor is on {x.device} or {y.device}, not on the current GPU")
        h = shape[1]
        if rows == 1:         # the stride of an axis of one element is any
            xs, ys = (h * d, xs[1]), (h * d, ys[1])
        if h == 1:
            xs, ys = (xs[0], d), (ys[0], d)
        arr[i] = (x.data_ptr(), y.data_ptr(), h, xs[0], xs[1], ys[0], ys[1])
    rc = (_lib or load()).hexi_rope(rope, r, pos, pos_stride, arr, len(tensors), x_type, y_type, HEXI_ROPE_INVERSE if inverse else 0, _stream(stream))
    if rc:
        _check(rc)


def _rope_a2a(fn, rope, segs, whole, packed, src, dst, head_lists, rotate, positions, inverse, stream):
    r, rows = _with_rows(segs)
    d, shape, strides = rope.head_dim, whole.shape, whole.stride()
    if len(shape) != 3 or shape[0] != rows or shape[2] != d or strides[2] != 1 or (shape[1] > 1 and strides[1] != d):
        _refuse(f"a [{rows}, heads, {d}] tensor with packed heads is needed, not {tuple(shape)} with strides {strides}")
    n, dev = shape[1], _current_device()
    if packed.dtype != whole.dtype or not packed.is_contiguous() or packed.numel() < sum(len(h) for h in head_lists) * rows * d or len(rotate) != n:
        _refuse(f"packed: {packed.numel()} elements of {packed.dtype}; rotate: {len(rotate)} entries for {n} heads")
    if whole.get_device() != dev or packed.get_device() != dev:
        _refuse(f"a tensor is on {whole.device} or {packed.device}, not on the current GPU")
    pos, pos_stride = _rope_positions(rope, positions, rows, dev)
    counts, heads = _head_tables(head_lists)
    flags = (ctypes.c_uint8 * max(1, n))(*[1 if x else 0 for x in rotate])
    rc = fn(rope, r, pos, pos_stride, src.data_ptr(), dst.data_ptr(), n, _dtype(whole), strides[0] if rows > 1 else n * d, len(head_lists), counts, heads, flags,
            HEXI_ROPE_INVERSE if inverse else 0, _stream(stream))
    if rc:
        _check(rc)


def hexi_rope_a2a_pack(rope, segs, x, packed, head_lists, rotate, positions=None, inverse=False, stream=None):
    """hexi_a2a_pack of a fused shard with the heads h of x that have rotate[h] rotated on the way."""
    _rope_a2a((_lib or load()).hexi_rope_a2a_pack, rope, segs, x, packed, x, packed, head_lists, rotate, positions, inverse, stream)


def hexi_rope_a2a_unpack(rope, segs, packed, y, head_lists, rotate, positions=None, inverse=False, stream=None):
    """hexi_a2a_unpack with the inverse rotation on the way (the gradients'; inverse=True: the rotation itself)."""
    _rope_a2a((_lib or load()).hexi_rope_a2a_unpack, rope, segs, y, packed, packed, y, head_lists, rotate, positions, inverse, stream)


def _head_tables(head_lists):
    counts = (ctypes.c_int32 * max(1, len(head_lists)))(*[len(h) for h in head_lists])
    flat = [int(h) for heads in head_lists for h in heads]
    heads = (ctypes.c_int32 * max(1, len(flat)))(*flat)
    return counts, heads


def hexi_a2a_pack(x, packed, head_lists, stream=None):
    """x: [s, n_heads_total, d] (token stride may exceed a token); packed: contiguous 1-D buffer of the same
    dtype with sum(len(l)) * s * d elements; head_lists: one list of head indices per destination rank."""
    s, n, d = x.shape
    counts, heads = _head_tables(head_lists)
    _check(load().hexi_a2a_pack(_ptr(x), _ptr(packed), s, n, d, x.element_size(), x.stride(0), len(head_lists), counts, heads,
                                _stream(stream)))


def hexi_a2a_unpack(packed, y, head_lists, stream=None):
    """Inverse of hexi_a2a_pack: scatters the per-rank parts of `packed` into y [s, n_heads_total, d]."""
    s, n, d = y.shape
    counts, heads = _head_tables(head_lists)
    _check(load().hexi_a2a_unpack(_ptr(packed), _ptr(y), s, n, d, y.element_size(), y.stride(0), len(head_lists), counts, heads,
                                  _stream(stream)))


class _Cluster(ctypes.Structure):
    _fields_ = [("n_devices", ctypes.c_int32)] + [(k, ctypes.POINTER(ctypes.c_double)) for k in ("c", "b", "m", "m_static", "alpha", "bw")]


class _Model(ctypes.Structure):
    _fields_ = [("l_tot", ctypes.c_int64), ("batch", ctypes.c_int32), ("hidden", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("dtype_bytes", ctypes.c_int32), ("gamma_act", ctypes.c_double)]


class _SchedOpts(ctypes.Structure):
    _fields_ = [("m1", ctypes.c_int32), ("m2", ctypes.c_int32), ("i_max", ctypes.c_int32), ("token_quantum", ctypes.c_int32),
                ("gap_ratio", ctypes.c_double), ("perturb", ctypes.c_double), ("move_tokens", ctypes.c_int64)]


class _Schedule(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("group_of", ctypes.POINTER(ctypes.c_int32)), ("l_group", ctypes.POINTER(ctypes.c_int64)),
                ("s_pre", ctypes.POINTER(ctypes.c_int64)), ("n_heads", ctypes.POINTER(ctypes.c_int32))]


def _cluster_struct(c, b, m, m_static, alpha, bw):
    n = len(c)
    arrs = [np.ascontiguousarray(a, dtype=np.float64) for a in (c, b, m, m_static, np.asarray(alpha).reshape(-1), np.asarray(bw).reshape(-1))]
    st = _Cluster(n, *[a.ctypes.data_as(ctypes.POINTER(ctypes.c_double)) for a in arrs])
    return st, arrs


def _model_struct(l_tot, batch, hidden, head_dim, n_heads, dtype_bytes, gamma_act=2.0):
    return _Model(l_tot, batch, hidden, head_dim, n_heads, dtype_bytes, gamma_act)


def hexi_sched_cost(cluster, model, groups, l_group, s_pre, n_heads):
    """cluster: dict(c, b, m, m_static, alpha, bw); model: dict(l_tot, batch, hidden, head_dim, n_heads, dtype_bytes[, gamma_act]);
    groups: list of device lists in ring order.  Returns (T_blk, max T_nonattn, max T_A2A, sum T_step, feasible)."""
    cs, keep = _cluster_struct(**cluster)
    ms = _model_struct(**model)
    n = cs.n_devices
    group_of = np.full(n, -1, dtype=np.int32)
    for k, g in enumerate(groups):
        for d in g:
            group_of[d] = k
    lg = np.zeros(n, dtype=np.int64)
    lg[:len(groups)] = l_group
    sp, nh = np.ascontiguousarray(s_pre, dtype=np.int64), np.ascontiguousarray(n_heads, dtype=np.int32)
    sch = _Schedule(len(groups), group_of.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), lg.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                    sp.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), nh.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
    terms = (ctypes.c_double * 4)()
    feas = ctypes.c_int32(0)
    _check(load().hexi_sched_cost(ctypes.byref(cs), ctypes.byref(ms), ctypes.byref(sch), terms, ctypes.byref(feas)))
    return terms[0], terms[1], terms[2], terms[3], bool(feas.value)


def hexi_sched_solve(cluster, model, **opts):
    """Returns dict(groups, l_group, s_pre, n_heads, cost).  opts: m1, m2, i_max, token_quantum, gap_ratio, perturb, move_tokens."""
    cs, keep = _cluster_struct(**cluster)
    ms = _model_struct(**model)
    n = cs.n_devices
    o = _SchedOpts(opts.get("m1", 0), opts.get("m2", 0), opts.get("i_max", 0), opts.get("token_quantum", 0),
                   opts.get("gap_ratio", 0.0), opts.get("perturb", 0.0), opts.get("move_tokens", 0))
    group_of, lg = np.zeros(n, dtype=np.int32), np.zeros(n, dtype=np.int64)
    sp, nh = np.zeros(n, dtype=np.int64), np.zeros(n, dtype=np.int32)
    sch = _Schedule(0, group_of.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), lg.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                    sp.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), nh.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
    cost = ctypes.c_double(0.0)
    _check(load().hexi_sched_solve(ctypes.byref(cs), ctypes.byref(ms), ctypes.byref(o), ctypes.byref(sch), ctypes.byref(cost)))
    groups = [[d for d in range(n) if group_of[d] == k] for k in range(sch.n_groups)]
    return dict(groups=groups, l_group=[int(x) for x in lg[:sch.n_groups]], s_pre=[int(x) for x in sp], n_heads=[int(x) for x in nh],
                cost=cost.value)


def hexi_set_dkdv_run_len(run_len):
    """0: the library chooses per call; n >= 1: at most n q heads per dK/dV workgroup run.  Returns the previous value."""
    return int(load().hexi_set_dkdv_run_len(int(run_len)))


def hexi_mfma_probe(operands, sink, iters, stream=None):
    """operands: 65536 bytes of bf16 on the device; sink: float32[256 * 512] on the device."""
    rc = load_probe().hexi_mfma_probe(_ptr(operands), _ptr(sink), int(iters), _stream(stream))
    if rc != 0:
        raise HexiError(rc, "hexi_mfma_probe refused its arguments or the launch")

