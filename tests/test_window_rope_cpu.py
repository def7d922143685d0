"""Windowed attention and rotary positions without a GPU: the window's geometry against its definition, and every refusal of the entry points, before anything is launched."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import window_util as wu
from paper_2605_07569_amd import hexi, workloads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF = float("inf")


@pytest.fixture(scope="module")
def window_binary(tmp_path_factory):
    hipcc = "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("window") / "window_check")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2605_07569_amd", "csrc"),
                           os.path.join(ROOT, "tests", "host", "window_check.cpp"), "-o", exe])
    return exe


def _random_case(rng):
    def segs(n, far):
        out, cur = [], rng.randrange(far)
        for _ in range(n):
            ln = rng.randint(1, 40)
            out.append((cur, ln))
            cur += ln + rng.randrange(60)
        return out
    far = rng.choice([1, 50, 400, 2 ** 31 - 3000])
    return wu.Case("", segs(rng.randint(1, 6), far), segs(rng.randint(1, 6), rng.choice([1, far])), rng.choice([1, 2, 17, 64, 200, 5000, 2 ** 31 - 1]),
                   rng.choice([0, 1, 5, 64, 300, 2 ** 31 - 1]))


def test_window_geometry_is_the_definition(window_binary):
    rng = random.Random(5)
    cases = [wu.Case(c.name, c.q_segs, c.kv_segs, min(c.window, 2 ** 31 - 1), min(c.n_sink, 2 ** 31 - 1)) for c in wu.CASES] + [_random_case(rng) for _ in range(150)]
    text = lambda segs: f"{len(segs)} " + " ".join(f"{s} {n}" for s, n in segs)
    out = subprocess.run([window_binary], input="\n".join(f"{c.window} {c.n_sink} {text(c.q_segs)} {text(c.kv_segs)}" for c in cases) + "\n", capture_output=True,
                         text=True, check=True).stdout.strip("\n").split("\n")
    assert len(out) == len(cases)
    for c, line in zip(cases, out):
        seen = wu.visible(c)
        left, right = line.split("|")
        for row, item in zip(seen, left.split()):
            sink, lo, hi = map(int, item.split(":"))
            want = torch.zeros(c.lc, dtype=torch.bool)
            want[:sink] = True
            want[lo:hi] = True
            assert 0 <= sink <= lo <= hi <= c.lc and torch.equal(row, want), (c, item)
        for col, item in zip(seen.T, right.split()):
            first, end = map(int, item.split(":"))
            want = torch.zeros(c.lq, dtype=torch.bool)
            want[first:end] = True
            assert torch.equal(col, want), (c, item)


def test_which_workgroups_the_steps_take(window_binary):
    """The GPU tests' steps, that every shape is among them."""
    text = lambda segs: f"{len(segs)} " + " ".join(f"{s} {n}" for s, n in segs)
    ask = lambda cases, d: subprocess.run([window_binary], input="\n".join(f"large {c.nq} {c.nkv} {d} {min(c.window, 2 ** 31 - 1)} {min(c.n_sink, 2 ** 31 - 1)} {text(c.q_segs)} {text(c.kv_segs)}"
                                                                           for c in cases) + "\n", capture_output=True, text=True, check=True).stdout.split()
    assert [x[0] for x in ask(wu.LARGE, 128)] == ["1"] * len(wu.LARGE) and [x[0] for x in ask(wu.LARGE, 64)] == ["0"] * len(wu.LARGE)
    for d in (64, 128):
        assert [x[:2] for x in ask(wu.CASES, d)] == ["01"] * len(wu.CASES)
        assert [x[1] for x in ask(wu.MANY, d)] == ["0"] * len(wu.MANY)
        assert [[p != "1" for p in x.split(":")[1:]] for x in ask(wu.PARTS, d)] == [[True, False], [True, False], [False, True], [True, True], [True, False], [True, True], [True, False]]
        assert [x[1] for x in ask(wu.PARTS, d)] == ["1"] * len(wu.PARTS)
        many = ask([wu.MANY_PARTS], d)[0]
        assert many[1] == "0" and int(many.split(":")[1]) > 1


def _codes(call, good, bad):
    """Every entry of bad = (code, changes) is refused with that code."""
    for code, changes in bad:
        args = dict(good)
        args.update(changes)
        assert call(**args) == code, (changes, hexi.hexi_last_error())
        assert hexi.hexi_last_error()


DESC = dict(dtype=hexi.HEXI_BF16, d=128, nq=8, nkv=2, scale=0.1, qs=(1024, 128), ks=(256, 128), kv_of_q=None)
BAD_DESCS = [(hexi.HEXI_EUNSUPPORTED, dict(d=96, qs=(768, 96), ks=(192, 96))), (hexi.HEXI_EUNSUPPORTED, dict(dtype=5)), (hexi.HEXI_EINVAL, dict(nkv=3)),
             (hexi.HEXI_EINVAL, dict(scale=INF)), (hexi.HEXI_EINVAL, dict(nq=129)), (hexi.HEXI_EALIGN, dict(ks=(257, 128))), (hexi.HEXI_EINVAL, dict(kv_of_q=[0] * 7 + [2])),
             (hexi.HEXI_EINVAL, dict(q_segs=[(3, 0)])), (hexi.HEXI_EINVAL, dict(kv_segs=[(0, 4), (2, 4)])), (hexi.HEXI_EUNSUPPORTED, dict(kv_segs=[(2 ** 31 - 4, 8)])),
             (hexi.HEXI_EINVAL, dict(window=0)), (hexi.HEXI_EINVAL, dict(window=-1)), (hexi.HEXI_EINVAL, dict(n_sink=-1)), (hexi.HEXI_EINVAL, dict(no_window=True))]


def _common(dtype, d, nq, nkv, scale, qs, ks, kv_of_q, q_segs, kv_segs, window, n_sink, no_window):
    desc = hexi.make_desc(dtype, d, nq, nkv, scale, qs, ks, kv_of_q)
    return desc, None if no_window else ctypes.byref(hexi.make_window(window, n_sink)), hexi.make_range(q_segs)[0], hexi.make_range(kv_segs)[0]


def test_windowed_forward_refusals():
    lib = hexi.load()

    def call(q=16, k=16, v=16, o=16, lse=16, o_dtype=hexi.HEXI_BF16, flags=0, **kw):
        desc, win, qr, kr = _common(**kw)
        return lib.hexi_attn_win_fwd_chunk(ctypes.byref(desc), win, ctypes.byref(qr), ctypes.byref(kr), q, k, v, o, o_dtype, lse, flags, None, 0, None)

    good = dict(DESC, q_segs=[(4, 4)], kv_segs=[(0, 8)], window=3, n_sink=1, no_window=False)
    _codes(call, good, BAD_DESCS + [(hexi.HEXI_EINVAL, {n: None}) for n in ("q", "k", "v", "o", "lse")] + [(hexi.HEXI_EALIGN, {n: 24}) for n in ("q", "k", "v", "o", "lse")] +
           [(hexi.HEXI_EUNSUPPORTED, dict(o_dtype=2)), (hexi.HEXI_EINVAL, dict(flags=2)), (hexi.HEXI_EINVAL, dict(flags=hexi.HEXI_ACCUMULATE))])
    assert lib.hexi_attn_win_fwd_chunk(None, None, None, None, 16, 16, 16, 16, 0, 16, 0, None, 0, None) == hexi.HEXI_EINVAL
    assert lib.hexi_attn_win_workspace_bytes(None, None, 5, 5) == 0
    # few rows and long windows need a workspace; it is asked for by the lengths alone
    desc, win, long = hexi.make_desc(hexi.HEXI_BF16, 128, 8, 2, 0.1, (1024, 128), (256, 128)), hexi.make_window(4096, 4), 100000
    need = hexi.hexi_attn_win_workspace_bytes(desc, win, 1, long)
    assert need > 0 and hexi.hexi_attn_win_workspace_bytes(desc, win, 4096, long) == 0 and hexi.hexi_attn_win_workspace_bytes(desc, win, 1, 60) == 0
    assert hexi.hexi_attn_win_workspace_bytes(desc, hexi.make_window(0), 1, long) == 0 and hexi.hexi_attn_win_workspace_bytes(desc, win, 0, long) == 0
    qr, kr = hexi.make_range([(long, 1)])[0], hexi.make_range([(1, long)])[0]
    for ws, n, code in ((None, 0, hexi.HEXI_EWORKSPACE), (16, need - 1, hexi.HEXI_EWORKSPACE), (None, need, hexi.HEXI_EWORKSPACE), (24, need, hexi.HEXI_EALIGN)):
        assert lib.hexi_attn_win_fwd_chunk(desc, win, qr, kr, 16, 16, 16, 16, hexi.HEXI_BF16, 16, 0, ws, n, None) == code


def test_windowed_backward_refusals():
    lib = hexi.load()

    def call(q=16, k=16, v=16, o=16, d_o=16, lse=16, delta=16, dq=16, dk=16, dv=16, o_dtype=hexi.HEXI_F32, grad=hexi.HEXI_BF16, flags=hexi.HEXI_COMPUTE_DELTA, **kw):
        desc, win, qr, kr = _common(**kw)
        return lib.hexi_attn_win_bwd_chunk(ctypes.byref(desc), win, ctypes.byref(qr), ctypes.byref(kr), q, k, v, o, o_dtype, d_o, lse, delta, dq, dk, dv, grad, flags, None, 0, None)

    good = dict(DESC, q_segs=[(4, 4)], kv_segs=[(0, 8)], window=3, n_sink=1, no_window=False)
    names = ("q", "k", "v", "o", "d_o", "lse", "delta", "dq", "dk", "dv")
    _codes(call, good, BAD_DESCS + [(hexi.HEXI_EINVAL, {n: None}) for n in names] + [(hexi.HEXI_EALIGN, {n: 24}) for n in names] +
           [(hexi.HEXI_EUNSUPPORTED, dict(o_dtype=2)), (hexi.HEXI_EUNSUPPORTED, dict(grad=3)), (hexi.HEXI_EINVAL, dict(flags=32)), (hexi.HEXI_EINVAL, dict(flags=hexi.HEXI_ACCUMULATE)),
            (hexi.HEXI_EINVAL, dict(flags=hexi.HEXI_SKIP_DQ | hexi.HEXI_SKIP_DKDV)), (hexi.HEXI_EINVAL, dict(flags=hexi.HEXI_SKIP_DQ, dk=None)),
            (hexi.HEXI_EINVAL, dict(flags=hexi.HEXI_SKIP_DKDV, dq=None))])
    # many rows behind sinks are of use in parts; the workspace is asked for by the lengths alone, and may be left out
    desc, win = hexi.make_desc(hexi.HEXI_BF16, 128, 8, 1, 0.1, (1024, 128), (128, 128)), hexi.make_window(1024, 4)
    size = hexi.hexi_attn_win_bwd_workspace_bytes
    need = size(desc, win, 16384, 17408)
    assert need > 0 and size(desc, win, 512, 17408) == 0 and size(desc, hexi.make_window(1024), 16384, 17408) == 0
    assert size(desc, hexi.make_window(0, 4), 16384, 17408) == 0 and size(desc, win, 0, 17408) == 0 and lib.hexi_attn_win_bwd_workspace_bytes(None, None, 5, 5) == 0
    qr, kr = hexi.make_range([(1024, 16384)])[0], hexi.make_range([(0, 17408)])[0]
    for ws, n, code in ((16, need - 1, hexi.HEXI_EWORKSPACE), (24, need, hexi.HEXI_EALIGN)):
        assert lib.hexi_attn_win_bwd_chunk(desc, win, qr, kr, 16, 16, 16, 16, hexi.HEXI_BF16, 16, 16, 16, 16, 16, 16, hexi.HEXI_BF16, 0, ws, n, None) == code


def test_rope_refusals():
    lib = hexi.load()

    def tensors(n, **kw):
        t = dict(x=16, y=32, n_heads=2, xt=256, xh=128, yt=256, yh=128)
        t.update(kw)
        return (hexi.hexi_rope_tensor * max(1, n))(*[hexi.hexi_rope_tensor(t["x"], t["y"], t["n_heads"], t["xt"], t["xh"], t["yt"], t["yh"])] * n)

    def rope(d=128, freq=(1.0,) * 64, axes=None, n_axes=1, pairing=0, null=False, rot=None):
        r = hexi.make_rope(d, freq, axes, n_axes=n_axes)
        r.pairing = pairing
        if rot is not None:
            r.rot_dim = rot
        if null:
            r.inv_freq = ctypes.POINTER(ctypes.c_double)()
        return r

    def call(rope_args=None, segs=((5, 4),), pos=None, pos_stride=0, tensor_args=None, n=1, n_given=None, xd=0, yd=0, flags=0, no_desc=False):
        r = rope(**(rope_args or {}))
        arr = tensors(n, **(tensor_args or {}))
        return lib.hexi_rope(None if no_desc else ctypes.byref(r), ctypes.byref(hexi.make_range(list(segs))[0]), pos, pos_stride, arr, n if n_given is None else n_given, xd, yd, flags, None)

    E, S, A = hexi.HEXI_EINVAL, hexi.HEXI_EUNSUPPORTED, hexi.HEXI_EALIGN
    _codes(call, {}, [(E, dict(no_desc=True)), (S, dict(rope_args=dict(d=120))), (S, dict(rope_args=dict(d=272))), (S, dict(rope_args=dict(freq=(1.0,) * 4))),
                      (S, dict(rope_args=dict(freq=(1.0,) * 72))), (S, dict(rope_args=dict(rot=20))), (S, dict(rope_args=dict(rot=0))), (S, dict(rope_args=dict(rot=-16))),
                      (E, dict(rope_args=dict(pairing=2))), (E, dict(rope_args=dict(n_axes=0))), (E, dict(rope_args=dict(n_axes=5))),
                      (E, dict(rope_args=dict(axes=[0] * 63 + [2], n_axes=2))), (E, dict(rope_args=dict(axes=[-1] + [0] * 63, n_axes=2))), (E, dict(rope_args=dict(null=True))),
                      (E, dict(rope_args=dict(freq=(1.0,) * 63 + (INF,)))), (E, dict(rope_args=dict(freq=(float("nan"),) * 64))), (E, dict(rope_args=dict(freq=(2e6,) * 64))),
                      (E, dict(segs=())), (E, dict(segs=((5, 0),))), (E, dict(pos=16, pos_stride=3)), (A, dict(pos=18, pos_stride=4)), (E, dict(flags=1)),
                      (S, dict(xd=2)), (S, dict(yd=-1)), (E, dict(n_given=0)), (E, dict(n=5)), (E, dict(tensor_args=dict(x=None))), (E, dict(tensor_args=dict(y=None))),
                      (E, dict(tensor_args=dict(n_heads=0))), (E, dict(tensor_args=dict(xt=120))), (E, dict(tensor_args=dict(yh=64))), (S, dict(tensor_args=dict(xt=2 ** 40))),
                      (S, dict(tensor_args=dict(yh=2 ** 62))), (E, dict(tensor_args=dict(y=16), yd=1)), (E, dict(tensor_args=dict(y=16, yt=512))),
                      (A, dict(tensor_args=dict(x=24))), (A, dict(tensor_args=dict(y=40))), (A, dict(tensor_args=dict(xt=260))), (A, dict(tensor_args=dict(yh=132)))])


def test_rope_redistribution_refusals():
    lib = hexi.load()
    i32 = ctypes.c_int32

    def call(fn, n=6, d=128, dtype=0, stride=None, counts=(2, 1), heads=(0, 5, 3), ptr=16, rotate=True, flags=0, segs=((0, 4),), pos=None):
        r = hexi.make_rope(d, (1.0,) * (d // 2))
        c, h = (i32 * max(1, len(counts)))(*counts), (i32 * max(1, len(heads)))(*heads)
        rot = (ctypes.c_uint8 * n)(*[1] * n) if rotate else None
        return fn(ctypes.byref(r), ctypes.byref(hexi.make_range(list(segs))[0]), pos, 0, ptr, ptr, n, dtype, n * d if stride is None else stride, len(counts), c, h, rot, flags, None)

    E, S, A = hexi.HEXI_EINVAL, hexi.HEXI_EUNSUPPORTED, hexi.HEXI_EALIGN
    for fn in (lib.hexi_rope_a2a_pack, lib.hexi_rope_a2a_unpack):
        _codes(call, dict(fn=fn), [(E, dict(heads=(0, 6, 3))), (E, dict(heads=(0, -1, 3))), (E, dict(counts=(2, -1))), (S, dict(dtype=2)), (S, dict(d=24)),
                                   (E, dict(stride=6 * 128 - 8)), (A, dict(stride=6 * 128 + 4)), (A, dict(ptr=8)), (E, dict(ptr=None)), (E, dict(rotate=False)), (E, dict(flags=2)),
                                   (E, dict(segs=())), (E, dict(pos=16)), (S, dict(n=300, counts=(257,), heads=tuple(range(257)))), (S, dict(stride=2 ** 40))])
        assert call(fn, counts=(), heads=()) == hexi.HEXI_OK      # no heads listed: nothing to move
    assert call(lib.hexi_rope_a2a_unpack, heads=(0, 5, 0)) == E


def test_binding_refuses_what_does_not_fit_before_the_library_is_asked():
    """Shapes, element types, strides and devices that the C ABI cannot see."""
    q, k = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    desc, win = hexi.desc_for(q, k, 0.1), hexi.make_window(3, 1)
    o, lse = torch.zeros(4, 8, 128), torch.zeros(8, 4)

    def fwd(**kw):
        a = dict(q_segs=[(4, 4)], kv_segs=[(0, 8)], q=q, k=k, v=k, o=o, lse=lse)
        a.update(kw)
        hexi.hexi_attn_win_fwd_chunk(desc, win, a["q_segs"], a["kv_segs"], a["q"], a["k"], a["v"], a["o"], a["lse"])

    def refused(f, *args, **kw):
        with pytest.raises(hexi.HexiError) as e:
            f(*args, **kw)
        return e.value.code

    E, S = hexi.HEXI_EINVAL, hexi.HEXI_EUNSUPPORTED
    assert refused(fwd) == E                                              # tensors on the CPU
    for kw in (dict(q=q[:3]), dict(q=q[:, :7]), dict(v=k[:7]), dict(q=q.float()), dict(o=o[:3]), dict(o=o[:, :, ::2]), dict(lse=lse[:, :3]), dict(lse=lse.double()),
               dict(q_segs=[(4, 5)]), dict(kv_segs=[(0, 9)]), dict(q=torch.zeros(4, 9, 128, dtype=torch.bfloat16)[:, :8])):
        assert refused(fwd, **kw) == E
    assert refused(fwd, q=q.half()) == S

    def bwd(**kw):
        a = dict(d_o=q, delta=lse, dq=o, dk=torch.zeros(8, 2, 128), dv=torch.zeros(8, 2, 128), o=o)
        a.update(kw)
        hexi.hexi_attn_win_bwd_chunk(desc, win, [(4, 4)], [(0, 8)], q, k, k, a["o"], a["d_o"], lse, a["delta"], a["dq"], a["dk"], a["dv"])

    for kw in ({}, dict(d_o=q[:3]), dict(delta=lse[:7]), dict(dq=o.bfloat16()), dict(dk=torch.zeros(7, 2, 128)), dict(o=o[:3])):
        assert refused(bwd, **kw) == E
    rope = hexi.make_rope(128, [1.0] * 64)
    x = torch.zeros(4, 2, 128)
    R = hexi.hexi_rope
    assert refused(R, rope, [(0, 4)], [(x, x)]) == E and refused(R, rope, [(0, 4)], []) == E and refused(R, rope, [(0, 5)], [(x, x)]) == E
    assert refused(R, rope, [(0, 4)], [(x, x[:, :1])]) == E and refused(R, rope, [(0, 4)], [(x, x.bfloat16()), (x, x)]) == E and refused(R, rope, [(0, 4)], [(x[..., :64], x[..., :64])]) == E
    assert refused(R, rope, [(0, 4)], [(x, x)], positions=torch.zeros(1, 4)) == E and refused(R, rope, [(0, 4)], [(x, x)], positions=torch.zeros(2, 4, dtype=torch.int32)) == E
    assert refused(hexi.make_rope, 128, [1.0] * 64, [0] * 63) == E and refused(hexi.make_rope, 128, [1.0] * 64, pairing="other") == E
    P, U = hexi.hexi_rope_a2a_pack, hexi.hexi_rope_a2a_unpack
    flat = torch.zeros(4 * 2 * 128)
    assert refused(P, rope, [(0, 4)], x, flat, [[0, 1]], [1, 1]) == E                            # on the CPU
    assert refused(P, rope, [(0, 4)], x, flat[1:], [[0, 1]], [1, 1]) == E and refused(P, rope, [(0, 4)], x, flat, [[0, 1]], [1]) == E
    assert refused(U, rope, [(0, 4)], flat.bfloat16(), x, [[0, 1]], [1, 1]) == E and refused(U, rope, [(0, 3)], flat, x, [[0, 1]], [1, 1]) == E


@pytest.mark.parametrize("q_segs,window,n_sink", [([(0, 5)], 1, 0), ([(7, 3), (12, 1), (30, 4)], 3, 0), ([(7, 3), (12, 1), (30, 4)], 21, 2), ([(7, 3), (30, 4)], 10 ** 12, 0),
                                                  ([(7, 3), (30, 4)], 5, 10 ** 12), ([(50, 3)], 10, 41), ([(50, 3)], 10, 42), ([(50, 3)], 10, 4), ([], 4, 4)])
def test_window_segs_are_the_keys_that_rows_see(q_segs, window, n_sink):
    rows = [p for s, n in q_segs for p in range(s, s + n)]
    last = max(rows, default=-1)
    need = {j for p in rows for j in range(p + 1) if p - j < window or j < n_sink}
    segs = workloads.window_segs(q_segs, window, n_sink)
    held = [j for s, n in segs for j in range(s, s + n)]
    assert held == sorted(set(held)) and all(b[0] > a[0] + a[1] for a, b in zip(segs, segs[1:]))
    assert set(held) == need and (not held or held[-1] == last)
