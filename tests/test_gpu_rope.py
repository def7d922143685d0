"""GPU parity of the rotary positions (hexi_rope) and of the rotation inside the head redistribution against their definition in float64."""
import math

import numpy as np
import pytest
import torch

from oracle import a2a
from paper_2605_07569_amd import hexi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def freqs(rot, axes, base=10000.0):
    n = rot // 2
    return [base ** (-i / n) for i in range(n)], [i * axes // n for i in range(n)]


def turned(x, pos, freq, axis, adjacent, inverse):
    """x [rows, heads, d] in float64, pos [axes, rows]: rotated, and a bound of the fp32 arithmetic.  An angle is held to 2^-25 of a quarter turn and a
    few roundings of sine and cosine: 4 half steps of fp32 each, one more per product and for the sum: 8 u (|a| + |b|)."""
    n, r = len(freq), 2 * len(freq)
    a = pos.double()[axis].T * torch.tensor(freq, dtype=torch.float64) * (-1 if inverse else 1)
    c, s = a.cos()[:, None], a.sin()[:, None]
    i, j = (slice(0, r, 2), slice(1, r, 2)) if adjacent else (slice(0, n), slice(n, r))
    y, bound = x.clone(), torch.zeros_like(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    bound[..., i] = bound[..., j] = 8 * 2.0 ** -24 * (x[..., i].abs() + x[..., j].abs())
    return y, bound


def close(got, want, bound, out):
    half = 2.0 ** -8 if out == BF16 else 0.0
    err = (got.double().cpu() - want).abs()
    limit = bound + 1.01 * half * want.abs()
    assert bool((err <= limit).all()), f"{int((err > limit).sum())} of {err.numel()} over the bound, worst {float((err / (limit + 1e-30)).max()):.2f}"


def table(axes, rows, seed, big=100000):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-big, big, (axes, rows), generator=g, dtype=torch.int32)


@pytest.mark.parametrize("adjacent", [False, True], ids=["half", "adjacent"])
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 64), (64, 16), (80, 80), (96, 32), (128, 112), (16, 16), (256, 256)])
def test_rope_shapes(d, rot, x_type, y_type, adjacent):
    for rows, heads, axes, use_table, inverse in ((1, (1, 1), 1, False, False), (7, (3, 2), 3, True, False), (65, (5, 1), 2, True, True), (300, (6, 2), 1, False, True)):
        print(f"\n  rows={rows} heads={heads} d={d} rot={rot} axes={axes} {x_type} -> {y_type} inverse={inverse}", flush=True)
        g = torch.Generator().manual_seed(rows)
        freq, axis = freqs(rot, axes)
        half = rows // 2
        segs = [(1000, rows)] if half == 0 else [(1000, half), (900000, rows - half)]
        pos = table(axes, rows, 5) if use_table else torch.cat([torch.arange(s, s + n) for s, n in segs])[None].expand(axes, -1)
        rope = hexi.make_rope(d, freq, axis, pairing="adjacent" if adjacent else "half", n_axes=axes)
        xs = [torch.randn(rows, h, d, generator=g).to(x_type) for h in heads]
        ys = [torch.full((rows * h * d + 64,), 77.0, dtype=y_type, device=DEV) for h in heads]
        pairs = [(x.to(DEV), y[:-64].view(rows, h, d)) for x, y, h in zip(xs, ys, heads)]
        hexi.hexi_rope(rope, segs, pairs, positions=pos.to(DEV) if use_table else None, inverse=inverse)
        torch.cuda.synchronize()
        for x, y, (_, got) in zip(xs, ys, pairs):
            close(got, *turned(x.double(), pos, freq, axis, adjacent, inverse), y_type)
            assert torch.all(y[-64:] == 77.0)
            if y_type == F32 or x_type == BF16:      # columns that are not rotated are copied
                assert torch.equal(got[..., rot:].cpu().to(F32), x[..., rot:].to(y_type).to(F32))


def test_rope_far_positions_and_signs():
    """Positions up to the ends of int32, high frequencies: the angle loses nothing."""
    d = 64
    freq = [1.0, 0.5, math.pi, 1e-9, 123.456, 1000.1] + [0.9 ** i for i in range(26)]
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1048575, -777777777, 2 ** 30]], dtype=torch.int32)
    rope = hexi.make_rope(d, freq)
    x = torch.randn(8, 2, d, generator=torch.Generator().manual_seed(1))
    y = torch.empty(8, 2, d, device=DEV)
    hexi.hexi_rope(rope, [(0, 8)], [(x.to(DEV), y)], positions=pos.to(DEV))
    # the float64 products of the definition would be off by 2^-53 of an angle of up to 2e12: long double here
    a = np.multiply.outer(pos[0].numpy().astype(np.longdouble), np.array(freq, dtype=np.longdouble))
    c, s = torch.from_numpy(np.cos(a).astype(np.float64))[:, None], torch.from_numpy(np.sin(a).astype(np.float64))[:, None]
    lo, hi = x.double()[..., :32], x.double()[..., 32:]
    want = torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    # (an 80-bit angle of 2e12 is itself held to 2^-64 x 2e12 = 1.1e-7)
    limit = (8 * 2.0 ** -24 + 2.0 ** -64 * torch.from_numpy(np.abs(a).astype(np.float64)))[:, None] * (lo.abs() + hi.abs())
    assert bool(((y.double().cpu() - want).abs() <= torch.cat([limit, limit], -1)).all())
    assert torch.equal(y[0].cpu(), x[0])


def test_rope_in_place_in_a_fused_buffer_and_back():
    """q and k rotated in place inside a fused q / k / v buffer with padding; the rest stays; the inverse brings them back to two roundings."""
    rows, nq, nkv, d = 133, 6, 2, 128
    for dtype, half in ((BF16, 2.0 ** -8), (F32, 2.0 ** -24)):
        wide = torch.randn(rows, nq + 2 * nkv + 1, d, generator=torch.Generator().manual_seed(3)).to(dtype)
        buf = wide.to(DEV)
        q, k = buf[:, :nq], buf[:, nq:nq + nkv]
        freq, axis = freqs(d, 1)
        rope = hexi.make_rope(d, freq, axis)
        hexi.hexi_rope(rope, [(50000, rows)], [(q, q), (k, k)])
        pos = (torch.arange(rows) + 50000)[None]
        close(buf[:, :nq + nkv], *turned(wide[:, :nq + nkv].double(), pos, freq, axis, False, False), dtype)
        assert torch.equal(buf[:, nq + nkv:].cpu(), wide[:, nq + nkv:])
        hexi.hexi_rope(rope, [(50000, rows)], [(q, q), (k, k)], inverse=True)
        x = wide[:, :nq + nkv].double()
        pair = x[..., :64].abs() + x[..., 64:].abs()
        limit = (2.1 * half * 1.5 + 16 * 2.0 ** -24) * torch.cat([pair, pair], -1)      # each rotation rounds both of a pair: at most sqrt(2) half (|a| + |b|) comes back per rounding
        assert bool(((buf[:, :nq + nkv].double().cpu() - x).abs() <= limit).all())


def test_rope_head_major_strides_and_padding_rows():
    """[heads][rows][d] storage; rows behind the shard's stay as they are."""
    rows, h, d = 40, 3, 64
    x = torch.randn(h, rows + 9, d, generator=torch.Generator().manual_seed(4)).to(DEV)
    y = torch.full((h, rows + 5, d), 77.0, device=DEV)
    freq, axis = freqs(64, 2)
    pos = table(2, rows, 6)
    hexi.hexi_rope(hexi.make_rope(d, freq, axis), [(0, rows)], [(x.transpose(0, 1)[:rows], y.transpose(0, 1)[:rows])], positions=pos.to(DEV))
    close(y.transpose(0, 1)[:rows], *turned(x.transpose(0, 1)[:rows].double().cpu(), pos, freq, axis, False, False), F32)
    assert torch.all(y[:, rows:] == 77.0)


def test_rope_copies_and_rotates_what_is_not_finite():
    """Unrotated columns keep infinities, NaN and -0; a bad value of a pair stays in its pair."""
    rows, d, rot = 5, 64, 32
    x = torch.randn(rows, 1, d, generator=torch.Generator().manual_seed(5))
    x[1, 0, 40], x[2, 0, 41], x[3, 0, 63], x[4, 0, 3] = float("inf"), float("nan"), -0.0, float("inf")
    freq, axis = freqs(rot, 1)
    y = torch.empty_like(x, device=DEV)
    hexi.hexi_rope(hexi.make_rope(d, freq, axis), [(10, rows)], [(x.to(DEV), y)])
    y = y.cpu()
    assert y[1, 0, 40] == float("inf") and y[2, 0, 41].isnan() and math.copysign(1.0, float(y[3, 0, 63])) == -1.0
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[4, 0, 3] = bad[4, 0, 19] = bad[1, 0, 40] = bad[2, 0, 41] = True
    assert torch.isfinite(y[~bad]).all() and not torch.isfinite(y[bad]).any()


def _parts(x, lists):
    return torch.from_numpy(a2a.a2a_pack(x.numpy(), lists))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,rot,adjacent,axes", [(128, 128, False, 1), (64, 32, True, 3), (64, 64, False, 2)])
def test_rope_pack_and_unpack(dtype, d, rot, adjacent, axes):
    n = 12
    rotate = [1] * 6 + [1, 0] + [0] * 4
    freq, axis = freqs(rot, axes)
    rope = hexi.make_rope(d, freq, axis, pairing="adjacent" if adjacent else "half", n_axes=axes)
    for rows, lists, pad in ((1, [[3]], 0), (33, [[11, 0, 5], [], [3], [8, 9, 1, 2, 6]], 0), (129, [[0, 7], [0, 6, 6], list(range(12))], 40), (70, [[4, 1, 7], [11, 0, 5, 2, 3]], 24)):
        print(f"\n  rows={rows} d={d} rot={rot} {dtype} lists={lists}", flush=True)
        g = torch.Generator().manual_seed(rows)
        x = torch.randn(rows, n, d, generator=g).to(dtype)
        wide = torch.zeros(rows, n * d + pad, dtype=dtype)
        wide[:, :n * d] = x.view(rows, -1)
        xd = torch.as_strided(wide.to(DEV), (rows, n, d), (n * d + pad, d, 1))
        pos = table(axes, rows, 7, 1000) if axes > 1 else (torch.arange(rows) + 4000)[None]
        segs = [(4000, rows)]
        total = sum(len(h) for h in lists) * rows * d
        packed = torch.full((total + 64,), 77.0, dtype=dtype, device=DEV)
        posd = pos.to(DEV) if axes > 1 else None
        hexi.hexi_rope_a2a_pack(rope, segs, xd, packed, lists, rotate, positions=posd)
        keep = torch.tensor(rotate)[None, :, None] == 0

        def want_of(t, inverse):
            y, b = turned(t.double(), pos, freq, axis, adjacent, inverse)
            return torch.where(keep, t.double(), y), torch.where(keep, torch.zeros_like(b), b)

        y, b = want_of(x, False)
        close(packed[:total], _parts(y, lists), _parts(b, lists), dtype)
        assert torch.all(packed[total:] == 77.0)
        # inverse pack, and heads that are not rotated are exact copies
        hexi.hexi_rope_a2a_pack(rope, segs, xd, packed, lists, [0] * n, positions=posd, inverse=True)
        assert torch.equal(packed[:total].cpu().float(), _parts(x.float(), lists))
        flat = [h for heads in lists for h in heads]
        if len(set(flat)) < len(flat):
            with pytest.raises(hexi.HexiError):
                hexi.hexi_rope_a2a_unpack(rope, segs, packed[:total], xd, lists, rotate, positions=posd)
            continue
        z = torch.randn(total, generator=g).to(dtype)
        y_wide = torch.full((rows, n * d + pad), 77.0, dtype=dtype, device=DEV)
        yd = torch.as_strided(y_wide, (rows, n, d), (n * d + pad, d, 1))
        for inverse in (False, True):
            hexi.hexi_rope_a2a_unpack(rope, segs, z.to(DEV), yd, lists, rotate, positions=posd, inverse=inverse)
            back = torch.from_numpy(a2a.a2a_unpack(z.double().numpy(), rows, n, d, lists, y=np.full((rows, n, d), 77.0)))
            w, b = want_of(back, not inverse)
            listed = torch.zeros(n, dtype=torch.bool)
            listed[flat] = True
            close(yd[:, listed], w[:, listed], b[:, listed], dtype)
            assert torch.all(yd[:, ~listed] == 77.0) and torch.all(y_wide[:, n * d:] == 77.0)


def test_rope_gradient_is_the_inverse_rotation():
    """<rope(x), y> = <x, inverse(y)>, and against differences of the definition."""
    rows, h, d = 20, 2, 64
    g = torch.Generator().manual_seed(8)
    x, y = torch.randn(rows, h, d, generator=g), torch.randn(rows, h, d, generator=g)
    freq, axis = freqs(64, 3)
    pos = table(3, rows, 9, 500)
    rope = hexi.make_rope(d, freq, axis)
    a, b = torch.empty_like(x, device=DEV), torch.empty_like(x, device=DEV)
    hexi.hexi_rope(rope, [(0, rows)], [(x.to(DEV), a)], positions=pos.to(DEV))
    hexi.hexi_rope(rope, [(0, rows)], [(y.to(DEV), b)], positions=pos.to(DEV), inverse=True)
    lhs, rhs = float((a.cpu().double() * y.double()).sum()), float((x.double() * b.cpu().double()).sum())
    assert abs(lhs - rhs) <= 16 * 2.0 ** -24 * 2 * float((x.double().abs() * y.double().abs()).sum() + x.norm() * y.norm())
    step = torch.randn(x.shape, generator=g, dtype=torch.float64)
    f = [float((turned(x.double() + e * step, pos, freq, axis, False, False)[0] * y.double()).sum()) for e in (0.5, -0.5)]
    got = float((b.cpu().double() * step).sum())      # the rotation is linear: a difference is exact
    assert abs((f[0] - f[1]) - got) <= 1e-6 * float((b.cpu().double() * step).abs().sum())


def test_rope_streams_and_graphs():
    rows, d = 77, 128
    freq, axis = freqs(d, 1)
    rope = hexi.make_rope(d, freq, axis)
    x = torch.randn(rows, 4, d, device=DEV).to(BF16)
    y, z, want = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    lists, rotate = [[0, 2], [1, 3]], [1, 1, 0, 1]
    p1, p2 = (torch.empty(x.numel(), dtype=BF16, device=DEV) for _ in range(2))
    hexi.hexi_rope(rope, [(9, rows)], [(x, want)])
    hexi.hexi_rope_a2a_pack(rope, [(9, rows)], x, p1, lists, rotate)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        hexi.hexi_rope(rope, [(9, rows)], [(x, y)])
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hexi.hexi_rope(rope, [(9, rows)], [(x, z)])
        hexi.hexi_rope_a2a_pack(rope, [(9, rows)], x, p2, lists, rotate)
    for _ in range(4):
        z.fill_(float("nan")); p2.fill_(float("nan"))
        graph.replay()
        hexi.hexi_rope(rope, [(9, rows)], [(x, y)])
        torch.cuda.synchronize()
        assert torch.equal(z, want) and torch.equal(p2, p1) and torch.equal(y, want)
