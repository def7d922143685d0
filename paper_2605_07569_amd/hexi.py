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
           "hexi_attn_win_workspace_bytes", "hexi_attn_win_fwd_chunk", "hexi_attn_win_bwd_chunk", "hexi_rope", "hexi_rope_a2a_pack", "hexi_rope_a2a_unpack",
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
    lib.hexi_attn_win_bwd_chunk.argtypes = [dp, wp, rp, rp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, u32, vp]
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


_DTYPES = None


def _dtype(t):
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.bfloat16: HEXI_BF16, torch.float32: HEXI_F32}
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise HexiError(HEXI_EUNSUPPORTED, f"element type {t.dtype} (bf16 or fp32)")
    return code


def _on_device(*tensors):
    """Tensors that the current device's stream may use."""
    import torch
    dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else None
    for t in tensors:
        if t is not None and (not t.is_cuda or (dev is not None and t.get_device() != dev)):
            _refuse(f"a tensor is on {t.device}, not on the current GPU")


def _dense(name, t, shape, dtype=None):
    if tuple(t.shape) != shape or not t.is_contiguous() or (dtype is not None and t.dtype != dtype):
        _refuse(f"{name}: a contiguous {shape} tensor{'' if dtype is None else f' of {dtype}'} is needed, not {tuple(t.shape)} {t.dtype}")


def _win_ranges(desc, q_segs, kv_segs, q, k, v, lse, d_o=None):
    """Ranges of a windowed call, with what the binding can check of the tensors checked: element types, shapes, strides, device."""
    import torch
    qr = q_segs if isinstance(q_segs, hexi_range) else make_range(q_segs)[0]
    kr = kv_segs if isinstance(kv_segs, hexi_range) else make_range(kv_segs)[0]
    # (whatever else is wrong with a range the library refuses)
    lq = sum(qr.segs[i].len for i in range(max(0, min(qr.n_segs, HEXI_MAX_SEGS))))
    lc = sum(kr.segs[i].len for i in range(max(0, min(kr.n_segs, HEXI_MAX_SEGS))))
    d, nq, nkv = desc.head_dim, desc.n_q_heads, desc.n_kv_heads
    for name, t, shape, strides in (("q", q, (lq, nq, d), (desc.q_stride_tok, desc.q_stride_head, 1)), ("d_o", d_o, (lq, nq, d), (desc.q_stride_tok, desc.q_stride_head, 1)),
                                    ("k", k, (lc, nkv, d), (desc.kv_stride_tok, desc.kv_stride_head, 1)), ("v", v, (lc, nkv, d), (desc.kv_stride_tok, desc.kv_stride_head, 1))):
        if t is None:
            continue
        if tuple(t.shape) != shape or _dtype(t) != desc.dtype or any(s != w and n > 1 for s, w, n in zip(t.stride(), strides, shape)):
            _refuse(f"{name} is {tuple(t.shape)} with strides {t.stride()}, {t.dtype}; the descriptor and the ranges say {shape} with strides {strides}")
    _dense("lse", lse, (nq, lq), torch.float32)
    return qr, kr, lq, lc


def hexi_attn_win_workspace_bytes(desc, window, lq, lc):
    return int(load().hexi_attn_win_workspace_bytes(ctypes.byref(desc), ctypes.byref(window), lq, lc))


def hexi_attn_win_fwd_chunk(desc, window, q_segs, kv_segs, q, k, v, o, lse, flags=0, workspace=None, stream=None):
    """Windowed forward; o's element type (fp32 or bf16) is the result's."""
    lib = _lib or load()
    qr, kr, lq, lc = _win_ranges(desc, q_segs, kv_segs, q, k, v, lse)
    _dense("o", o, (lq, desc.n_q_heads, desc.head_dim))
    _on_device(q, k, v, o, lse, workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib.hexi_attn_win_fwd_chunk(desc, window, qr, kr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _dtype(o), _ptr(lse), flags, _ptr(workspace), ws_bytes,
                                     _stream(stream))
    if rc:
        _check(rc)


def hexi_attn_win_bwd_chunk(desc, window, q_segs, kv_segs, q, k, v, o, d_o, lse, delta, dq, dk, dv, flags=0, stream=None):
    """Windowed backward; the element type of dq, dk and dv (one for all; None for the half that is skipped) is the gradients'."""
    import torch
    lib = _lib or load()
    qr, kr, lq, lc = _win_ranges(desc, q_segs, kv_segs, q, k, v, lse, d_o)
    nq, nkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    _dense("delta", delta, (nq, lq), torch.float32)
    if o is not None:
        _dense("o", o, (lq, nq, d))
    grads = [t for t in (dq, dk, dv) if t is not None]
    for name, t, shape in (("dq", dq, (lq, nq, d)), ("dk", dk, (lc, nkv, d)), ("dv", dv, (lc, nkv, d))):
        if t is not None:
            _dense(name, t, shape, grads[0].dtype)
    _on_device(q, k, v, o, d_o, lse, delta, *grads)
    rc = lib.hexi_attn_win_bwd_chunk(desc, window, qr, kr, _ptr(q), _ptr(k), _ptr(v), _ptr(o), HEXI_F32 if o is None else _dtype(o), _ptr(d_o), _ptr(lse),
                                     _ptr(delta), _ptr(dq), _ptr(dk), _ptr(dv), _dtype(grads[0]) if grads else HEXI_F32, flags, _stream(stream))
    if rc:
        _check(rc)


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


def _rope_positions(rope, positions, rows):
    if positions is None:
        return None, 0
    import torch
    if positions.dtype != torch.int32 or positions.dim() != 2 or tuple(positions.shape) != (rope.n_axes, rows) or (rows > 1 and positions.stride(1) != 1):
        _refuse(f"positions: an int32 [{rope.n_axes}][{rows}] tensor is needed, not {tuple(positions.shape)} {positions.dtype}")
    return positions.data_ptr(), positions.stride(0) if rope.n_axes > 1 else max(1, rows)


def _rope_rows(segs):
    r = segs if isinstance(segs, hexi_range) else make_range(segs)[0]
    return r, sum(r.segs[i].len for i in range(max(0, min(r.n_segs, HEXI_MAX_SEGS))))


def hexi_rope(rope, segs, tensors, positions=None, inverse=False, stream=None):
    """Rotates the tensors of a shard in one launch.  tensors: [(x, y), ...], x and y [rows, heads, head_dim] with contiguous columns, y may be x; all x
    of one element type, all y of one.  positions: int32 [n_axes, rows] on the device, or None for the rows' global positions."""
    lib = _lib or load()
    r, rows = _rope_rows(segs)
    if not tensors:
        _refuse("no tensors")
    pos, pos_stride = _rope_positions(rope, positions, rows)
    arr = (hexi_rope_tensor * len(tensors))()
    x0, y0 = tensors[0]
    for a, (x, y) in zip(arr, tensors):
        if x.dim() != 3 or x.shape != y.shape or x.shape[0] != rows or x.shape[2] != rope.head_dim or x.stride(2) != 1 or y.stride(2) != 1 or \
                x.dtype != x0.dtype or y.dtype != y0.dtype:
            _refuse(f"a tensor pair of [{rows}, heads, {rope.head_dim}] and one type a side is needed, not {tuple(x.shape)} {x.dtype} -> {tuple(y.shape)} {y.dtype}")
        # (the stride of an axis of one element is any)
        d = rope.head_dim
        st = [t.stride(i) if t.shape[i] > 1 else d * (t.shape[1] if i == 0 else 1) for t in (x, y) for i in (0, 1)]
        a.x, a.y, a.n_heads = x.data_ptr(), y.data_ptr(), x.shape[1]
        a.x_stride_tok, a.x_stride_head, a.y_stride_tok, a.y_stride_head = st
        _on_device(x, y, positions)
    rc = lib.hexi_rope(rope, r, pos, pos_stride, arr, len(tensors), _dtype(x0), _dtype(y0), HEXI_ROPE_INVERSE if inverse else 0, _stream(stream))
    if rc:
        _check(rc)


def _rope_a2a(fn, rope, segs, whole, packed, src, dst, head_lists, rotate, positions, inverse, stream):
    r, rows = _rope_rows(segs)
    if whole.dim() != 3 or whole.shape[0] != rows or whole.shape[2] != rope.head_dim or whole.stride(2) != 1 or (whole.shape[1] > 1 and whole.stride(1) != rope.head_dim):
        _refuse(f"a [{rows}, heads, {rope.head_dim}] tensor with packed heads is needed, not {tuple(whole.shape)} with strides {whole.stride()}")
    n = whole.shape[1]
    if packed.dtype != whole.dtype or not packed.is_contiguous() or packed.numel() < sum(len(h) for h in head_lists) * rows * rope.head_dim or len(rotate) != n:
        _refuse(f"packed: {packed.numel()} elements of {packed.dtype}; rotate: {len(rotate)} entries for {n} heads")
    pos, pos_stride = _rope_positions(rope, positions, rows)
    _on_device(whole, packed, positions)
    counts, heads = _head_tables(head_lists)
    flags = (ctypes.c_uint8 * max(1, n))(*[1 if x else 0 for x in rotate])
    _check(fn(rope, r, pos, pos_stride, src.data_ptr(), dst.data_ptr(), n, _dtype(whole), whole.stride(0) if rows > 1 else n * rope.head_dim, len(head_lists), counts, heads, flags,
              HEXI_ROPE_INVERSE if inverse else 0, _stream(stream)))


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

