"""GPU parity of the windowed kernels in 64-row units against the definition in float64 (tests/test_window_units_cpu.py says that these steps take them)."""
import pytest
import torch

import window_util as wu
from paper_2605_07569_amd import hexi
from test_gpu_window import BF16, DEV, F32, REL, guarded, setup, untouched, workspace
from window_util import Case

pytestmark = pytest.mark.gpu


def some_heads(c, x, heads):
    """The case and the inputs of these q heads alone."""
    return Case(c.name, c.q_segs, c.kv_segs, c.window, c.n_sink, len(heads), c.nkv, [c.heads[h] for h in heads]), dict(x, q=x["q"][:, heads])


def forward_with_merges_and_bad_values(c, dtype, d):
    x, dev, desc, window = setup(c, dtype, d, 21)
    heads = sorted({0, 1, c.nq // 2, c.nq - 1})
    sub, some = some_heads(c, x, heads)
    need = hexi.hexi_attn_win_workspace_bytes(desc, window, c.lq, c.lc)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)

    def run(inputs, o, lse, flags=0):
        hexi.hexi_attn_win_fwd_chunk(desc, window, c.q_segs, c.kv_segs, inputs["q"], inputs["k"], inputs["v"], o, lse, flags=flags, workspace=ws[:need] if need else None)
        torch.cuda.synchronize()
        assert torch.all(ws[need:] == 255)

    for out in (F32, BF16):
        print(f"\n  {c.name}: {dtype} d={d} -> {out}", flush=True)
        o_flat, o = guarded((c.lq, c.nq, d), out, float("nan"))
        l_flat, lse = guarded((c.nq, c.lq), F32, float("nan"))
        run(dev, o, lse)
        ro, rl, bo, bl = wu.forward(sub, some, out)
        wu.within("lse", lse[heads], rl, bl)
        wu.within("o", o[:, heads], ro, bo, max(REL[dtype], 0 if out == F32 else REL[BF16]))
        assert torch.isfinite(o.float()).all() and not lse.isnan().any()
        untouched(o_flat, l_flat)
    ro, rl, bo, bl = wu.forward(sub, some, F32)
    # merged into a running result (a weight is off by the LSE's error, and the merge rounds a few times more)
    old = torch.randn(c.lq, c.nq, d, generator=torch.Generator().manual_seed(5))
    o, lse = old.to(DEV), torch.zeros(c.nq, c.lq, device=DEV)
    run(dev, o, lse, hexi.HEXI_ACCUMULATE)
    total = torch.logaddexp(rl, torch.zeros_like(rl))
    w = torch.exp(rl - total).T[..., None]
    old = old[:, heads].double()
    wu.within("merged lse", lse[heads], total, bl.nan_to_num(0) + 8 * wu.U * (1 + total.abs()))
    wu.within("merged o", o[:, heads], w * ro + (1 - w) * old, bo + (bl.T[..., None].nan_to_num(0) + 16 * wu.U) * (ro.abs() + old.abs()) + 1e-6)
    # values that are not finite: of v in its column of the rows that see it, of k in those rows alone
    sees = wu.visible(sub)
    for at, value in ((c.lc // 2, float("nan")), (c.lc - 1, float("inf")), (0, float("-inf"))):
        bad = x["v"].clone()
        bad[at, :, 17] = value
        run(dict(dev, v=wu.strided(bad, c.pad, DEV)), o, lse)
        want = ro.clone()
        want[sees[:, at], :, 17] = value
        wu.within("o", o[:, heads], want, bo)
        wu.within("lse", lse[heads], rl, bl)
        bad = x["k"].clone()
        bad[at, :, 40] = value
        run(dict(dev, k=wu.strided(bad, c.pad, DEV)), o, lse)
        hidden = ~sees[:, at]
        wu.within("o of the others", o[:, heads].cpu()[hidden], ro[hidden], bo[hidden])
        wu.within("lse of the others", lse[heads].cpu()[:, hidden], rl[:, hidden], bl[:, hidden])
        if value != value:
            assert o[:, heads].cpu()[~hidden].isnan().all() and lse[heads].cpu()[:, ~hidden].isnan().all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", wu.FORWARD_64, ids=lambda c: c.name)
def test_forward(c, dtype, d):
    forward_with_merges_and_bad_values(c, dtype, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("c", wu.FORWARD_64_SPLITS, ids=lambda c: c.name)
def test_forward_in_splits(c, d):
    forward_with_merges_and_bad_values(c, BF16, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("c", wu.BACKWARD_64, ids=lambda c: c.name)
def test_backward_fp32(c, d):
    """Overwritten and added to, with and without the workspace; rows whose LSE is infinite; a value that is not finite in one of each input."""
    x, dev, desc, window = setup(c, F32, d, 23)
    kv = [0, c.nkv - 1]
    heads = [h for h in range(c.nq) if c.heads[h] in kv]
    sub = Case(c.name, c.q_segs, c.kv_segs, c.window, c.n_sink, len(heads), len(kv), [kv.index(c.heads[h]) for h in heads])
    some = dict(q=x["q"][:, heads], k=x["k"][:, kv], v=x["v"][:, kv], d_o=x["d_o"][:, heads])
    ro, rl, _, _ = wu.forward(sub, some, F32)
    lse = rl.float()
    lse[0, c.lq // 2], lse[1, c.lq - 1], lse[1, 3] = float("-inf"), float("inf"), float("-inf")
    all_o, all_lse = torch.zeros(c.lq, c.nq, d), torch.full((c.nq, c.lq), 20.0)
    all_o[:, heads], all_lse[heads] = ro.float(), lse
    o_dev, lse_dev, delta = all_o.to(DEV), all_lse.to(DEV), torch.empty(c.nq, c.lq, device=DEV)
    need = hexi.hexi_attn_win_bwd_workspace_bytes(desc, window, c.lq, c.lc)
    assert (need > 0) == c.name.startswith("parts")
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    seen = wu.visible(c)

    def run(inputs, grad=F32, fill=float("nan"), flags=0, space=None):
        f1, dq = guarded((c.lq, c.nq, d), grad, 0.5 if grad == F32 else float("nan"))
        f2, dk = guarded((c.lc, c.nkv, d), grad, fill)
        f3, dv = guarded((c.lc, c.nkv, d), grad, fill)
        hexi.hexi_attn_win_bwd_chunk(desc, window, c.q_segs, c.kv_segs, inputs["q"], inputs["k"], inputs["v"], o_dev, inputs["d_o"], lse_dev, delta, dq, dk, dv,
                                     flags=flags | hexi.HEXI_COMPUTE_DELTA, workspace=space)
        torch.cuda.synchronize()
        untouched(f1, f2, f3)
        assert torch.all(ws[need:] == 255)
        return dict(dq=dq[:, heads].double().cpu() - (0.5 if grad == F32 else 0.0), dk=dk[:, kv].cpu(), dv=dv[:, kv].cpu()), (dq, dk, dv)

    for grad in (F32, BF16):
        print(f"\n  {c.name}: d={d} -> {grad}", flush=True)
        ref = wu.backward(sub, some, ro.float(), lse, grad)
        got, whole = run(dev, grad)
        # (0.5 was added to dq: half a step of what is there, |dq| + 0.5, and of the sum)
        slack = {"dq": 2 * wu.U * (0.5 + ref["dq"][0].abs()) if grad == F32 else 0.0, "dk": 0.0, "dv": 0.0}
        for name in got:
            wu.within(name, got[name], ref[name][0], ref[name][1] + slack[name], REL[grad])
        assert all(torch.isfinite(t.float()).all() for t in whole)
        if need:
            again, _ = run(dev, grad, space=ws[:need])
            assert all(torch.equal(got[name], again[name]) for name in got)
    ref = wu.backward(sub, some, ro.float(), lse, F32)
    got, _ = run(dev, fill=0.25, flags=hexi.HEXI_ACCUMULATE)
    for name in ("dk", "dv"):
        wu.within("added " + name, got[name] - 0.25, ref[name][0], ref[name][1] + 2.0 ** -23 + 2 * wu.U * ref[name][0].abs())
    for where, at, head in (("k", c.lc // 2, kv[-1]), ("v", c.lc - 1, 0), ("q", c.lq // 3, heads[-1]), ("d_o", c.lq - 2, 0)):
        for value in (float("nan"), float("inf")):
            bad = x[where].clone()
            bad[at, head, 5] = value
            got, _ = run(dict(dev, **{where: wu.strided(bad, c.pad, DEV)}))
            if where in ("k", "v"):
                rows, keys = seen[:, at], torch.arange(c.lc) == at
                of_q, of_kv = [c.heads[h] == head for h in heads], [h == head for h in kv]
            else:
                rows, keys = torch.arange(c.lq) == at, seen[at]
                of_q, of_kv = [h == head for h in heads], [h == c.heads[head] for h in kv]
            hit = {"dq": rows[:, None] & torch.tensor(of_q), "dk": keys[:, None] & torch.tensor(of_kv)}
            hit["dv"] = hit["dk"]
            slack = {"dq": 2 * wu.U * (0.5 + ref["dq"][0].abs()), "dk": torch.zeros_like(ref["dk"][0]), "dv": torch.zeros_like(ref["dv"][0])}
            for name in got:
                keep = ~hit[name]
                wu.within(f"{name} of the others", got[name][keep], ref[name][0][keep], (ref[name][1] + slack[name])[keep])
