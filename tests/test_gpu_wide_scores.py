"""Scores that are finite but further apart than the largest fp32 value: the key with the largest one has all the weight.

fp32 calls, and windowed bf16 calls of few rows, subtract the reference from a score first.  The other bf16 kernels form s log2(e) scale minus a rounded reference in one fma: the
reference is off by up to half its step, which from 2^31 on is 128 and more, so an exponential of it says nothing, and no bound holds for them here (below 2^24 it is under 1, and cancels
between the weights and their sum)."""
import pytest
import torch

from paper_2605_07569_amd import hexi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d,scale", [(128, 128 ** -0.5), (64, 0.125), (64, 0.1), (128, 0.3)])
@pytest.mark.parametrize("windowed,rows,dtype", [(w, n, torch.float32) for w in (True, False) for n in (1, 8, 40, 300)] + [(True, 1, torch.bfloat16), (True, 8, torch.bfloat16)])
def test_one_key_has_all_the_weight(windowed, rows, dtype, d, scale):
    """Keys of every 16-key part of a block but one score -2.5e38, one key 2.5e38: their difference is not finite, the exact result is that key's v."""
    nq, nkv, first, at = 4, 1, 100, 5
    lc = first + rows
    g = torch.Generator().manual_seed(rows)
    q, k = torch.zeros(rows, nq, d), torch.zeros(lc, nkv, d)
    q[..., 3], k[..., 3] = 1.6e19, -1.6e19
    k[at, :, 3] = 1.6e19
    q, k, v = q.to(dtype), k.to(dtype), torch.randn(lc, nkv, d, generator=g).to(dtype)
    score = float(q[0, 0, 3].double() * k[at, 0, 3].double())
    assert 2.4e38 < score < 3.4e38
    desc = hexi.desc_for(q, k, scale)
    o, lse = torch.full((rows, nq, d), float("nan"), device=DEV), torch.full((nq, rows), float("nan"), device=DEV)
    dev = [t.to(DEV) for t in (q, k, v)]
    if windowed:
        window = hexi.make_window(10 ** 9)
        n = hexi.hexi_attn_win_workspace_bytes(desc, window, rows, lc)
        hexi.hexi_attn_win_fwd_chunk(desc, window, [(first, rows)], [(0, lc)], *dev, o, lse, workspace=torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
    else:
        n = hexi.hexi_workspace_bytes(desc, rows, lc)
        hexi.hexi_attn_fwd_chunk(desc, [(first, rows)], [(0, lc)], *dev, o, lse, workspace=torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
    # a weight of one and products with it: one rounding of each; the LSE is a score (two products' roundings in the score, one with the scale, or with log2 e and back)
    want = v[at, 0].double().expand(rows, nq, d)
    assert bool(((o.double().cpu() - want).abs() <= 2.0 ** -22 * want.abs()).all()), o.isnan().sum()
    assert bool(((lse.double().cpu() - score * scale).abs() <= 8 * 2.0 ** -24 * score * scale).all())
