"""GPU parity of attention under a sliding window with sinks (hexi_attn_win_fwd_chunk, hexi_attn_win_bwd_chunk) against its definition in float64."""
import pytest
import torch

import window_util as wu
from paper_2605_07569_amd import hexi
from window_util import CASES, Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
# relative L2 allowed: P and dS are rounded to bf16 at random (2^-9 / sqrt(3) of each rms, twice for dS), the result once more: under 5e-3; fp32: 1e-5
REL = {BF16: 5e-3, F32: 1e-5}


def guarded(shape, dtype, fill):
    """A dense tensor inside a longer buffer of canaries."""
    n = 1
    for s in shape:
        n *= s
    flat = torch.full((n + 128,), 77.0, dtype=dtype, device=DEV)
    flat[64:64 + n] = fill
    return flat, flat[64:64 + n].view(shape)


def untouched(*flats):
    for f in flats:
        assert torch.all(f[:64] == 77.0) and torch.all(f[-64:] == 77.0), "wrote outside of its tensor"


def setup(c, dtype, d, seed=0):
    x = wu.inputs(c, dtype, d, seed)
    dev = {n: wu.strided(t, c.pad, DEV) for n, t in x.items()}
    desc = hexi.desc_for(dev["q"], dev["k"], d ** -0.5, c.kv_of_q)
    return x, dev, desc, hexi.make_window(c.window, c.n_sink)


def workspace(desc, window, c):
    n = hexi.hexi_attn_win_workspace_bytes(desc, window, c.lq, c.lc)
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", CASES, ids=lambda c: c.name)
def test_forward(c, dtype, d):
    x, dev, desc, window = setup(c, dtype, d)
    for out in (F32, BF16):
        print(f"\n  {c.name}: {dtype} d={d} -> {out}", flush=True)
        o_flat, o = guarded((c.lq, c.nq, d), out, float("nan"))
        l_flat, lse = guarded((c.nq, c.lq), F32, float("nan"))
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse, workspace=workspace(desc, window, c))
        torch.cuda.synchronize()
        ro, rl, bo, bl = wu.forward(c, x, out)
        wu.within("lse", lse, rl, bl)
        wu.within("o", o, ro, bo, max(REL[dtype], 0 if out == F32 else REL[BF16]))
        untouched(o_flat, l_flat)


@pytest.mark.parametrize("c", wu.LARGE, ids=lambda c: c.name)
def test_forward_in_256_row_workgroups(c):
    x, dev, desc, window = setup(c, BF16, 128, 11)
    heads = [0, 1, c.nq // 2, c.nq - 1]
    sub = Case(c.name, c.q_segs, c.kv_segs, c.window, c.n_sink, len(heads), c.nkv, [h // (c.nq // c.nkv) for h in heads])
    some = dict(x, q=x["q"][:, heads])
    for out in (F32, BF16):
        print(f"\n  {c.name} -> {out}", flush=True)
        o_flat, o = guarded((c.lq, c.nq, 128), out, float("nan"))
        l_flat, lse = guarded((c.nq, c.lq), F32, float("nan"))
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse)
        torch.cuda.synchronize()
        ro, rl, bo, bl = wu.forward(sub, some, out)
        wu.within("lse", lse[heads], rl, bl)
        wu.within("o", o[:, heads], ro, bo, REL[BF16])
        assert torch.isfinite(o.float()).all() and not lse.isnan().any()
        untouched(o_flat, l_flat)
    # merged into a running result
    old = torch.randn(c.lq, c.nq, 128, generator=torch.Generator().manual_seed(5))
    o, lse = old.to(DEV), torch.zeros(c.nq, c.lq, device=DEV)
    hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse, flags=hexi.HEXI_ACCUMULATE)
    ro, rl, bo, bl = wu.forward(sub, some, F32)
    total = torch.logaddexp(rl, torch.zeros_like(rl))
    w = torch.exp(rl - total).T[..., None]
    old = old[:, heads].double()
    # (a weight is off by the LSE's error, and the merge rounds a few times more)
    wu.within("merged lse", lse[heads], total, bl.nan_to_num(0) + 8 * wu.U * (1 + total.abs()))
    wu.within("merged o", o[:, heads], w * ro + (1 - w) * old, bo + (bl.T[..., None].nan_to_num(0) + 16 * wu.U) * (ro.abs() + old.abs()) + 1e-6)
    # a value that is not finite
    bad, at = x["v"].clone(), c.lc // 2
    bad[at, :, 17] = float("nan")
    hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], bad.to(DEV), o, lse)
    ro = ro.clone()
    ro[wu.visible(sub)[:, at], :, 17] = float("nan")
    wu.within("o", o[:, heads], ro, bo)


def test_forward_in_256_row_workgroups_with_drifting_scores():
    """Scores that rise by far more than 2^60 along a row's keys: the workgroup's second pass with a running maximum."""
    c = Case("drift", [(600, 512)], [(0, 1112)], 500, 40, nq=128, nkv=1)
    x = wu.inputs(c, BF16, 128, 12)
    x["k"] = (x["k"].float() * torch.linspace(0.1, 40, c.lc)[:, None, None]).to(BF16)
    dev = {n: t.to(DEV) for n, t in x.items()}
    desc, window = hexi.desc_for(dev["q"], dev["k"], 128 ** -0.5), hexi.make_window(c.window, c.n_sink)
    o, lse = torch.empty(c.lq, c.nq, 128, device=DEV), torch.empty(c.nq, c.lq, device=DEV)
    hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse)
    heads = [0, 100]
    sub = Case(c.name, c.q_segs, c.kv_segs, c.window, c.n_sink, 2, 1)
    ro, rl, bo, bl = wu.forward(sub, dict(x, q=x["q"][:, heads]), F32)
    wu.within("lse", lse[heads], rl, bl)
    wu.within("o", o[:, heads], ro, bo, REL[BF16])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", CASES, ids=lambda c: c.name)
def test_backward(c, dtype, d):
    x, dev, desc, window = setup(c, dtype, d, 1)
    ro, rl, _, _ = wu.forward(c, x, dtype)
    lse = rl.float()
    for grad, o_type in ((F32, F32), (BF16, BF16)):
        print(f"\n  {c.name}: {dtype} d={d} -> {grad}", flush=True)
        o = ro.to(o_type)
        ref = wu.backward(c, x, o, lse, grad)
        # fp32: dq is added to what is there, dk and dv are overwritten; bf16: all are overwritten
        dq0 = 0.5 if grad == F32 else float("nan")
        f1, dq = guarded((c.lq, c.nq, d), grad, dq0)
        f2, dk = guarded((c.lc, c.nkv, d), grad, float("nan"))
        f3, dv = guarded((c.lc, c.nkv, d), grad, float("nan"))
        f4, delta = guarded((c.nq, c.lq), F32, float("nan"))
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o.to(DEV), dev["d_o"], lse.to(DEV), delta, dq, dk, dv,
                                     flags=hexi.HEXI_COMPUTE_DELTA)
        torch.cuda.synchronize()
        rel = max(REL[dtype], 0 if grad == F32 else REL[BF16])
        wu.within("delta", delta, *ref["delta"])
        add = 0.5 if grad == F32 else 0.0
        wu.within("dq", dq, ref["dq"][0] + add, ref["dq"][1] + 2 * wu.U * add)
        wu.within("dk", dk, *ref["dk"], _rel_of(ref["dk"], rel))
        wu.within("dv", dv, *ref["dv"], rel)
        untouched(f1, f2, f3, f4)
        # the halves by themselves
        dq2, dk2, dv2 = torch.zeros_like(dq) + (0.5 if grad == F32 else 0), torch.empty_like(dk), torch.empty_like(dv)
        args = (desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], None, dev["d_o"], lse.to(DEV), delta)
        hexi.hexi_attn_win_bwd_chunk(*args, dq2, None, None, flags=hexi.HEXI_SKIP_DKDV)
        hexi.hexi_attn_win_bwd_chunk(*args, None, dk2, dv2, flags=hexi.HEXI_SKIP_DQ)
        torch.cuda.synchronize()
        wu.within("dq alone", dq2, ref["dq"][0] + add, ref["dq"][1] + 2 * wu.U * add)
        wu.within("dk alone", dk2, *ref["dk"])
        wu.within("dv alone", dv2, *ref["dv"])


def _rel_of(pair, rel):
    """dS is a difference: where its terms cancel (rows of one key), relative L2 says nothing and the elementwise bound alone holds."""
    want, bound = pair
    return rel if float(bound.norm()) < 0.05 * float(want.norm()) else None


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", wu.PARTS, ids=lambda c: c.name)
def test_backward_in_parts(c, dtype, d):
    """With the workspace that a call takes by itself, with one given, and with none; a value that is not finite; the sums added to what is there."""
    x, dev, desc, window = setup(c, dtype, d, 15)
    ro, rl, _, _ = wu.forward(c, x, F32)
    lse, o = rl.float(), ro.float()
    need = hexi.hexi_attn_win_bwd_workspace_bytes(desc, window, c.lq, c.lc)
    assert need > 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    delta = torch.empty(c.nq, c.lq, device=DEV)
    lib, (qr, kr) = hexi.load(), (hexi.make_range(c.q_segs)[0], hexi.make_range(c.kv_segs)[0])

    def run(grad, inputs=dev, how=None, fill=float("nan"), flags=0):
        f1, dq = guarded((c.lq, c.nq, d), grad, 0.0)
        f2, dk = guarded((c.lc, c.nkv, d), grad, fill)
        f3, dv = guarded((c.lc, c.nkv, d), grad, fill)
        flags |= hexi.HEXI_COMPUTE_DELTA
        if how == "none":
            code = hexi.HEXI_BF16 if grad == BF16 else hexi.HEXI_F32
            assert lib.hexi_attn_win_bwd_chunk(desc, window, qr, kr, *(inputs[n].data_ptr() for n in ("q", "k", "v")), o_dev.data_ptr(), hexi.HEXI_F32, inputs["d_o"].data_ptr(),
                                               lse_dev.data_ptr(), delta.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), code, flags, None, 0,
                                               torch.cuda.current_stream().cuda_stream) == hexi.HEXI_OK
        else:
            hexi.hexi_attn_win_bwd_chunk(desc, window, qr, kr, inputs["q"], inputs["k"], inputs["v"], o_dev, inputs["d_o"], lse_dev, delta, dq, dk, dv, flags=flags,
                                         workspace=ws[:need] if how == "given" else None)
        torch.cuda.synchronize()
        untouched(f1, f2, f3)
        assert torch.all(ws[need:] == 255)
        return dict(dq=dq, dk=dk, dv=dv)

    o_dev, lse_dev = o.to(DEV), lse.to(DEV)
    for grad in (F32, BF16):
        print(f"\n  {c.name}: {dtype} d={d} -> {grad}", flush=True)
        ref = wu.backward(c, x, o, lse, grad)
        rel = max(REL[dtype], 0 if grad == F32 else REL[BF16])
        got = run(grad)
        again, none = run(grad, how="given"), run(grad, how="none")
        for name in got:
            wu.within(name, got[name], *ref[name], rel)
            wu.within(name + " without a workspace", none[name], *ref[name], rel)
            assert torch.equal(got[name], again[name])
    ref = wu.backward(c, x, o, lse, F32)
    got = run(F32, fill=0.25, flags=hexi.HEXI_ACCUMULATE)
    for name in ("dk", "dv"):
        wu.within("added " + name, got[name] - 0.25, ref[name][0], ref[name][1] + 2.0 ** -23 + 2 * wu.U * ref[name][0].abs())
    seen = wu.visible(c)
    for where, at in (("q", c.lq // 2), ("d_o", c.lq - 1), ("k", 1)):
        bad = x[where].clone()
        bad[at, 0, 5] = float("inf")
        got = run(F32, dict(dev, **{where: wu.strided(bad, c.pad, DEV)}))
        rows, keys = (seen[:, at], torch.arange(c.lc) == at) if where == "k" else (torch.arange(c.lq) == at, seen[at])
        for name, hit in (("dq", rows), ("dk", keys), ("dv", keys)):
            wu.within(name + " of the others", got[name].cpu()[~hit], ref[name][0][~hit], ref[name][1][~hit])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("c", wu.MANY + [wu.MANY_PARTS], ids=lambda c: c.name)
def test_backward_in_64_row_workgroups(c, d):
    """All heads at once, two kv heads looked at; rows whose LSE is infinite, and then a value that is not finite in one of each input."""
    x, dev, desc, window = setup(c, BF16, d, 13)
    group, kv = c.nq // c.nkv, [0, min(33, c.nkv - 1)]
    heads = [h * group + i for h in kv for i in range(group)]
    sub = Case(c.name, c.q_segs, c.kv_segs, c.window, c.n_sink, len(heads), len(kv))
    some = dict(q=x["q"][:, heads], k=x["k"][:, kv], v=x["v"][:, kv], d_o=x["d_o"][:, heads])
    ro, rl, _, _ = wu.forward(sub, some, F32)
    lse = rl.float()
    lse[0, c.lq // 2], lse[1, c.lq - 1], lse[2, 3] = float("-inf"), float("inf"), float("-inf")
    all_o, all_lse = torch.zeros(c.lq, c.nq, d), torch.zeros(c.nq, c.lq)
    all_lse += 20.0
    all_o[:, heads], all_lse[heads] = ro.float(), lse
    seen = wu.visible(c)

    def run(grad, inputs):
        dq0 = 0.5 if grad == F32 else float("nan")
        f1, dq = guarded((c.lq, c.nq, d), grad, dq0)
        f2, dk = guarded((c.lc, c.nkv, d), grad, float("nan"))
        f3, dv = guarded((c.lc, c.nkv, d), grad, float("nan"))
        delta = torch.empty(c.nq, c.lq, device=DEV)
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, inputs["q"], inputs["k"], inputs["v"], all_o.to(grad).to(DEV), inputs["d_o"], all_lse.to(DEV), delta,
                                     dq, dk, dv, flags=hexi.HEXI_COMPUTE_DELTA)
        torch.cuda.synchronize()
        untouched(f1, f2, f3)
        return dict(dq=dq[:, heads].float().cpu() - (0.5 if grad == F32 else 0.0), dk=dk[:, kv].cpu(), dv=dv[:, kv].cpu()), dq, dk, dv

    for grad in (F32, BF16):
        print(f"\n  {c.name}: d={d} -> {grad}", flush=True)
        ref = wu.backward(sub, some, ro.float().to(grad), lse, grad)
        got, *whole = run(grad, dev)
        # (0.5 was added to and taken from dq again: 2^-23)
        for name in ("dq", "dk", "dv"):
            wu.within(name, got[name], ref[name][0], ref[name][1] + (2.0 ** -22 if name == "dq" else 0.0), REL[BF16])
        assert all(torch.isfinite(t.float()).all() for t in whole)
    ref = wu.backward(sub, some, ro.float(), lse, F32)
    for where, at, head in (("k", c.lc // 2, kv[-1]), ("v", c.lc - 1, 0), ("q", c.lq // 3, heads[-1]), ("d_o", c.lq - 2, 0)):
        bad = x[where].clone()
        bad[at, head, 5] = float("nan")
        got, *_ = run(F32, dict(dev, **{where: wu.strided(bad, c.pad, DEV)}))
        if where in ("k", "v"):
            rows, keys = seen[:, at], torch.arange(c.lc) == at
            of_q, of_kv = [h // group == head for h in heads], [h == head for h in kv]
        else:
            rows, keys = torch.arange(c.lq) == at, seen[at]
            of_q, of_kv = [h == head for h in heads], [h == head // group for h in kv]
        hit = {"dq": rows[:, None] & torch.tensor(of_q), "dk": keys[:, None] & torch.tensor(of_kv)}
        hit["dv"] = hit["dk"]
        for name in ("dq", "dk", "dv"):
            keep = ~hit[name]
            wu.within(f"{name} of the others", got[name][keep], ref[name][0][keep], ref[name][1][keep] + (2.0 ** -22 if name == "dq" else 0.0))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_accumulation_over_chunks_is_the_whole(dtype, d):
    """Keys in three uneven chunks, forward and backward, against one call over all of them."""
    c = Case("chunks", [(150, 180), (700, 90)], [(0, 790)], 140, 9, nq=4, nkv=2)
    _chunks(c, [[(0, 100)], [(100, 333)], [(433, 7), (440, 350)]], dtype, d)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_accumulation_of_split_units(dtype, d):
    """Few rows, long chunks: the units' runs of keys are split over workgroups, and joined with what is there."""
    for rows in (3, 70):
        _split_chunks(Case("split chunks", [(6000, rows)], [(0, 6000 + rows)], 5500, 40, nq=3, nkv=1), [[(0, 3100)], [(3100, 2900 + rows)]], dtype, d)


def _split_chunks(c, parts, dtype, d):
    window = hexi.make_window(c.window, c.n_sink)
    for part in parts:
        q, k = torch.empty(c.lq, c.nq, d, dtype=dtype), torch.empty(sum(n for _, n in part), c.nkv, d, dtype=dtype)
        assert hexi.hexi_attn_win_workspace_bytes(hexi.desc_for(q, k, 1.0), window, c.lq, k.shape[0]) > 0
    _chunks(c, parts, dtype, d)


def _chunks(c, parts, dtype, d):
    x, dev, desc, window = setup(c, dtype, d, 2)
    z = lambda *s: torch.zeros(s, device=DEV)
    o, lse = z(c.lq, c.nq, d), torch.full((c.nq, c.lq), float("-inf"), device=DEV)
    ro, rl, bo, bl = wu.forward(c, x, F32)
    at = 0
    for part in parts:
        n = sum(m for _, m in part)
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, part, dev["q"], dev["k"][at:at + n], dev["v"][at:at + n], o, lse, flags=hexi.HEXI_ACCUMULATE,
                                     workspace=workspace(desc, window, Case("", c.q_segs, part, c.window, c.n_sink)))
        at += n
    # every merge rounds o and lse again: three more half steps, and the weights' exponentials
    wu.within("lse", lse, rl, 4 * bl)
    wu.within("o", o, ro, 4 * bo, REL[dtype])
    ref = wu.backward(c, x, ro.float(), rl.float(), F32)
    delta, dq, dk, dv = z(c.nq, c.lq), z(c.lq, c.nq, d), z(c.lc, c.nkv, d) + 1.0, z(c.lc, c.nkv, d) + 1.0
    at, flags = 0, hexi.HEXI_COMPUTE_DELTA
    for part in parts:
        n = sum(m for _, m in part)
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, part, dev["q"], dev["k"][at:at + n], dev["v"][at:at + n], ro.float().to(DEV), dev["d_o"],
                                     rl.float().to(DEV), delta, dq, dk[at:at + n], dv[at:at + n], flags=flags | hexi.HEXI_ACCUMULATE)
        flags = 0
        at += n
    wu.within("dq", dq, ref["dq"][0], ref["dq"][1] + 4 * wu.U * ref["dq"][0].abs(), REL[dtype])
    for name, got in (("dk", dk), ("dv", dv)):
        wu.within(name, got, ref[name][0] + 1.0, ref[name][1] + 2 * wu.U * (1 + ref[name][0].abs()))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_window_past_everything_is_causal_attention(dtype):
    c = Case("causal", [(100, 333)], [(0, 433)], 10 ** 9, 0, nq=4, nkv=2)
    x, dev, desc, window = setup(c, dtype, 128, 3)
    o, lse = torch.empty(c.lq, c.nq, 128, device=DEV), torch.empty(c.nq, c.lq, device=DEV)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse)
    hexi.hexi_attn_fwd_chunk(desc, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o2, lse2)
    _, _, bo, bl = wu.forward(c, x, F32)
    wu.within("o", o, o2.double().cpu(), 2 * bo)
    wu.within("lse", lse, lse2.double().cpu(), 2 * bl)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, d, bad):
    """One bad value of v in a key: rows that see the key have it in that column, no other row or column is touched; one bad key: the rows that see it are
    NaN or as without it (a score of -inf), no other is touched.  Backward: the same for dq, and dk and dv of bad rows of q and dO."""
    c = Case("bad", [(100, 190)], [(0, 5), (61, 229)], 40, 5, nq=2, nkv=1)
    few = Case("bad, few rows", [(3000, 9)], [(0, 5), (500, 2509)], 2400, 5, nq=2, nkv=1)
    split = Case("bad, split", [(3000, 65)], [(0, 5), (500, 2565)], 2400, 5, nq=2, nkv=1)
    for c, where, key, col in ((c, "v", 3, 7), (c, "v", 90, 50), (c, "v", 233, 0), (c, "k", 2, 9), (c, "k", 120, 33), (c, "k", 233, 63),
                               (few, "v", 2, 3), (few, "v", 108, 9), (few, "v", 2513, 60), (few, "k", 110, 4), (few, "k", 2513, 5), (split, "v", 1, 3), (split, "v", 140, 9), (split, "v", 2540, 63), (split, "k", 150, 4), (split, "k", 2569, 5)):
        print(f"\n  {where}[{key}, {col}] = {bad}", flush=True)
        x = wu.inputs(c, dtype, d, 4)
        clean = {n: t.clone() for n, t in x.items()}
        x[where][key, 0, col] = bad
        dev = {n: t.to(DEV) for n, t in x.items()}
        desc, window = hexi.desc_for(dev["q"], dev["k"], d ** -0.5), hexi.make_window(c.window, c.n_sink)
        o, lse = torch.empty(c.lq, c.nq, d, device=DEV), torch.empty(c.nq, c.lq, device=DEV)
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, lse, workspace=workspace(desc, window, c))
        sees = wu.visible(c)[:, key]
        ro, rl, bo, bl = wu.forward(c, clean, F32)
        if where == "v":
            ro[sees, :, col] = bad
            wu.within("lse", lse, rl, bl)
            wu.within("o", o, ro, bo)
        else:
            o, lse = o.cpu().double(), lse.cpu().double()
            wu.within("o of the others", o[~sees], ro[~sees], bo[~sees])
            wu.within("lse of the others", lse[:, ~sees], rl[:, ~sees], bl[:, ~sees])
            for h in range(c.nq):
                hit = sees if bad != bad else sees & (clean["q"][:, h, col].float() * bad > 0)
                assert o[hit, h].isnan().all() and lse[h, hit].isnan().all()
                assert torch.isfinite(o[sees & ~hit, h]).all()
    c = Case("bad", [(100, 190)], [(0, 5), (61, 229)], 40, 5, nq=2, nkv=1)
    ro, rl, _, _ = wu.forward(c, wu.inputs(c, dtype, d, 4), F32)
    for where, at, col in (("v", 90, 50), ("k", 120, 33), ("k", 2, 3), ("q", 77, 5), ("d_o", 130, 11), ("d_o", 0, 1)):
        print(f"\n  backward {where}[{at}, {col}] = {bad}", flush=True)
        x = wu.inputs(c, dtype, d, 4)
        ref = wu.backward(c, x, ro.float(), rl.float(), F32)
        x[where][at, 0, col] = bad
        dev = {n: t.to(DEV) for n, t in x.items()}
        desc, window = hexi.desc_for(dev["q"], dev["k"], d ** -0.5), hexi.make_window(c.window, c.n_sink)
        delta = (ro * wu.inputs(c, dtype, d, 4)["d_o"].double()).sum(2).T.float().contiguous().to(DEV)
        dq, dk, dv = torch.zeros(c.lq, c.nq, d, device=DEV), torch.empty(c.lc, 1, d, device=DEV), torch.empty(c.lc, 1, d, device=DEV)
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], None, dev["d_o"], rl.float().to(DEV), delta, dq, dk, dv)
        if where in ("k", "v"):      # what the rows and keys that it touches get is not looked at
            rows, hit_keys = wu.visible(c)[:, at], torch.arange(c.lc) == at
        else:
            rows, hit_keys = torch.arange(c.lq) == at, wu.visible(c)[at]
        assert torch.isfinite(dq.cpu()[~rows]).all()
        wu.within("dq of the others", dq.cpu()[~rows], ref["dq"][0][~rows], ref["dq"][1][~rows])
        for name, got in (("dk", dk), ("dv", dv)):
            wu.within(name + " of the others", got.cpu()[~hit_keys], ref[name][0][~hit_keys], ref[name][1][~hit_keys])
        assert not torch.isfinite(dk.cpu()[hit_keys]).all()


def test_padding_rows_of_a_wider_buffer_may_hold_anything():
    """Rows behind the shard's and behind the chunk's in the same buffers are NaN, before and behind."""
    c = Case("inside", [(90, 77)], [(40, 127)], 33, 0, nq=2, nkv=1)
    for dtype in (BF16, F32):
        x = wu.inputs(c, dtype, 128, 5)
        wide = {}
        for n, t in x.items():
            w = torch.full((t.shape[0] + 200,) + t.shape[1:], float("nan"), dtype=dtype, device=DEV)
            w[100:100 + t.shape[0]] = t.to(DEV)
            wide[n] = w[100:100 + t.shape[0]]
        desc, window = hexi.desc_for(wide["q"], wide["k"], 128 ** -0.5), hexi.make_window(c.window)
        o, lse = torch.empty(c.lq, c.nq, 128, device=DEV), torch.empty(c.nq, c.lq, device=DEV)
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, wide["q"], wide["k"], wide["v"], o, lse)
        ro, rl, bo, bl = wu.forward(c, x, F32)
        wu.within("o", o, ro, bo)
        wu.within("lse", lse, rl, bl)


def test_infinite_lse_rows_have_no_gradient():
    c = Case("dead", [(50, 100)], [(0, 150)], 60, 2, nq=2, nkv=1)
    for dtype in (BF16, F32):
        x, dev, desc, window = setup(c, dtype, 64, 6)
        ro, rl, _, _ = wu.forward(c, x, F32)
        lse = rl.float()
        lse[0, 10], lse[1, 99], lse[0, 64] = float("-inf"), float("inf"), float("-inf")
        ref = wu.backward(c, x, ro.float(), lse, F32)
        delta, dq = torch.empty(c.nq, c.lq, device=DEV), torch.zeros(c.lq, c.nq, 64, device=DEV)
        dk, dv = torch.empty(c.lc, 1, 64, device=DEV), torch.empty(c.lc, 1, 64, device=DEV)
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], ro.float().to(DEV), dev["d_o"], lse.to(DEV), delta, dq, dk, dv,
                                     flags=hexi.HEXI_COMPUTE_DELTA)
        for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
            wu.within(name, got, *ref[name])


def test_gradients_against_differences():
    """<gradient, direction> against a central difference of the float64 definition along it, fp32 kernels."""
    c = Case("differences", [(40, 60)], [(0, 100)], 25, 3, nq=2, nkv=1)
    d = 64
    x, dev, desc, window = setup(c, F32, d, 7)
    ro, rl, _, _ = wu.forward(c, x, F32)
    delta, dq = torch.empty(c.nq, c.lq, device=DEV), torch.zeros(c.lq, c.nq, d, device=DEV)
    dk, dv = torch.empty(c.lc, 1, d, device=DEV), torch.empty(c.lc, 1, d, device=DEV)
    hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], ro.float().to(DEV), dev["d_o"], rl.float().to(DEV), delta, dq, dk, dv,
                                 flags=hexi.HEXI_COMPUTE_DELTA)
    for name, grad in (("q", dq), ("k", dk), ("v", dv)):
        g = torch.Generator().manual_seed(11)
        step = torch.randn(x[name].shape, generator=g, dtype=torch.float64)
        f = []
        for sign in (1, -1):
            y = {n: t.double() for n, t in x.items()}
            y[name] = y[name] + sign * 1e-4 * step
            f.append(float((wu.forward(c, y, F32)[0] * x["d_o"].double()).sum()))
        want, got = (f[0] - f[1]) / 2e-4, float((grad.double().cpu() * step).sum())
        # a central difference is off by a third derivative times 1e-8 / 6; the sum of |terms| times 1e-5 covers it and the kernels' 1e-5
        assert abs(got - want) <= 2e-5 * float((grad.double().cpu() * step).abs().sum()), (name, got, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streams_graphs_and_repeats(dtype):
    """On a side stream; captured and replayed among eager work; twice with the same bits."""
    c = Case("graph", [(300, 200)], [(0, 3), (201, 299)], 100, 3, nq=4, nkv=2)
    d = 128
    x, dev, desc, window = setup(c, dtype, d, 8)
    ws = workspace(desc, window, c)
    qr, kr = hexi.make_range(c.q_segs)[0], hexi.make_range(c.kv_segs)[0]

    def buffers():
        return dict(o=torch.empty(c.lq, c.nq, d, dtype=dtype, device=DEV), lse=torch.empty(c.nq, c.lq, device=DEV), delta=torch.empty(c.nq, c.lq, device=DEV),
                    dq=torch.zeros(c.lq, c.nq, d, dtype=dtype, device=DEV), dk=torch.empty(c.lc, c.nkv, d, dtype=dtype, device=DEV), dv=torch.empty(c.lc, c.nkv, d, dtype=dtype, device=DEV))

    def step(b):
        b["dq"].zero_()
        hexi.hexi_attn_win_fwd_chunk(desc, window, qr, kr, dev["q"], dev["k"], dev["v"], b["o"], b["lse"], workspace=ws)
        hexi.hexi_attn_win_bwd_chunk(desc, window, qr, kr, dev["q"], dev["k"], dev["v"], b["o"], dev["d_o"], b["lse"], b["delta"], b["dq"], b["dk"], b["dv"],
                                     flags=hexi.HEXI_COMPUTE_DELTA)

    want = buffers()
    step(want)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), buffers()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(got)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    for i in range(4):
        for t in got.values():
            t.fill_(float("nan"))
        eager = buffers()
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) and torch.equal(eager[n], want[n]) for n in want), i
    # new inputs in the same places
    y = wu.inputs(c, dtype, d, 9)
    for n in y:
        dev[n].copy_(y[n])
    graph.replay()
    step(eager)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], eager[n]) for n in got) and not torch.equal(got["o"], want["o"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_parts_on_streams_and_in_graphs(dtype):
    """A backward that takes a workspace by itself: on two streams at once, captured and replayed among eager calls, on a stream given by hand (without one)."""
    c, d = wu.PARTS[0], 64
    x, dev, desc, window = setup(c, dtype, d, 17)
    ro, rl, _, _ = wu.forward(c, x, F32)
    o, lse = ro.float().to(DEV), rl.float().to(DEV)
    ref = wu.backward(c, x, ro.float(), rl.float(), dtype)
    assert hexi.hexi_attn_win_bwd_workspace_bytes(desc, window, c.lq, c.lc) > 0

    def buffers():
        e = lambda *s, t=dtype: torch.zeros(s, dtype=t, device=DEV)
        return dict(delta=e(c.nq, c.lq, t=F32), dq=e(c.lq, c.nq, d), dk=e(c.lc, c.nkv, d), dv=e(c.lc, c.nkv, d))

    def run(b, **kw):
        b["dq"].zero_()
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, dev["q"], dev["k"], dev["v"], o, dev["d_o"], lse, b["delta"], b["dq"], b["dk"], b["dv"],
                                     flags=hexi.HEXI_COMPUTE_DELTA, **kw)

    want = buffers()
    run(want)
    torch.cuda.synchronize()
    same = lambda b: all(torch.equal(b[n], want[n]) for n in want)
    two, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, stream in zip(two, streams):
            with torch.cuda.stream(stream):
                run(b)
    torch.cuda.synchronize()
    assert same(two[0]) and same(two[1])
    captured, eager = buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(captured)
    for _ in range(4):
        captured["dk"].fill_(float("nan"))
        captured["dv"].fill_(float("nan"))
        graph.replay()
        run(eager)
        torch.cuda.synchronize()
        assert same(captured) and same(eager)
    b = buffers()
    torch.cuda.synchronize()
    run(b, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for name in ("dq", "dk", "dv"):
        wu.within(name, b[name], *ref[name], max(REL[dtype], 0 if dtype == F32 else REL[BF16]))
