"""Rotary positions on long shards, alone and inside the head redistribution: workgroups of several tokens, the last one with fewer, and tokens of more pieces than a
workgroup takes in one pass."""
import numpy as np
import pytest
import torch

from oracle import a2a
from paper_2605_07569_amd import hexi
from test_gpu_rope import BF16, DEV, F32, _parts, close, freqs, table, turned

pytestmark = pytest.mark.gpu

# rows, heads of the tensors, d, rot, axes: a workgroup of 256 threads takes 896 / pieces tokens (bf16 pieces of 16 columns, fp32 ones of 8) or a 1024th of the rows, if that is less
SHAPES = [
    (2050, (5, 1), 64, 64, 2),          # bf16: 3 tokens, one in the last workgroup
    (5003, (3, 2), 128, 32, 3),         # 5 tokens, 3 in the last one
    (5003, (36, 4), 128, 128, 1),       # bf16: 2 tokens of 320 pieces, 1 in the last one; fp32: 1
    (3001, (7,), 256, 112, 2),
    (917505, (1,), 16, 16, 1),          # 896 tokens of one piece (bf16): most LDS; one in the last workgroup
    (70, (64, 8), 128, 128, 1),         # fp32: 1152 pieces a token, two passes
    (1500, (120, 30), 128, 96, 2),      # bf16: 1200 pieces a token
]


def positions_of(rows, axes, use_table, seed):
    half = rows // 3
    segs = [(777, half), (5000000, rows - half)]
    pos = table(axes, rows, seed) if use_table else torch.cat([torch.arange(s, s + n) for s, n in segs])[None].expand(axes, -1)
    return segs, pos


@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rope(shape, x_type, y_type):
    rows, heads, d, rot, axes = shape
    freq, axis = freqs(rot, axes)
    for adjacent, use_table, inverse in ((False, False, False), (True, True, True)):
        print(f"\n  {shape} {x_type} -> {y_type} adjacent={adjacent} table={use_table}", flush=True)
        g = torch.Generator().manual_seed(rows)
        segs, pos = positions_of(rows, axes, use_table, 3)
        wide_pos = torch.full((axes, rows + 5), -12345, dtype=torch.int32)      # entries behind a row of the table are another tensor's
        wide_pos[:, :rows] = pos
        rope = hexi.make_rope(d, freq, axis, pairing="adjacent" if adjacent else "half", n_axes=axes)
        xs = [torch.randn(rows, h, d, generator=g).to(x_type) for h in heads]
        ys = [torch.full((rows * h * d + 64,), 77.0, dtype=y_type, device=DEV) for h in heads]
        pairs = [(x.to(DEV), y[:-64].view(rows, h, d)) for x, y, h in zip(xs, ys, heads)]
        hexi.hexi_rope(rope, segs, pairs, positions=wide_pos.to(DEV)[:, :rows] if use_table else None, inverse=inverse)
        torch.cuda.synchronize()
        for x, y, (_, got) in zip(xs, ys, pairs):
            close(got, *turned(x.double(), pos, freq, axis, adjacent, inverse), y_type)
            assert torch.all(y[-64:] == 77.0)
            if y_type == F32 or x_type == BF16:
                assert torch.equal(got[..., rot:].cpu().to(F32), x[..., rot:].to(y_type).to(F32))
        if x_type == y_type:      # in place: the same bits
            for x, _ in pairs:
                x_before = x.clone()
                hexi.hexi_rope(rope, segs, [(x, x)], positions=wide_pos.to(DEV)[:, :rows] if use_table else None, inverse=inverse)
                y = torch.empty_like(x)
                hexi.hexi_rope(rope, segs, [(x_before, y)], positions=wide_pos.to(DEV)[:, :rows] if use_table else None, inverse=inverse)
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n,d,rot,adjacent,axes,pad", [(2050, 6, 64, 64, False, 1, 0), (5003, 7, 64, 32, True, 3, 24), (5003, 40, 128, 128, False, 2, 0), (66, 90, 128, 112, True, 1, 8),
                                                            (1100, 200, 64, 64, False, 1, 0)])
def test_rope_pack_and_unpack(rows, n, d, rot, adjacent, axes, pad, dtype):
    freq, axis = freqs(rot, axes)
    rope = hexi.make_rope(d, freq, axis, pairing="adjacent" if adjacent else "half", n_axes=axes)
    order = [(7 * h + 3) % n for h in range(n)] if n % 7 else [(5 * h + 3) % n for h in range(n)]
    lists = [order[: n // 3], [], order[n // 3: n - 1]]      # one head goes nowhere
    rotate = [h % 3 != 1 for h in range(n)]
    g = torch.Generator().manual_seed(rows)
    segs, pos = positions_of(rows, axes, axes > 1, 4)
    posd = pos.contiguous().to(DEV) if axes > 1 else None
    x = torch.randn(rows, n, d, generator=g).to(dtype)
    wide = torch.zeros(rows, n * d + pad, dtype=dtype)
    wide[:, :n * d] = x.view(rows, -1)
    xd = torch.as_strided(wide.to(DEV), (rows, n, d), (n * d + pad, d, 1))
    total = (n - 1) * rows * d
    packed = torch.full((total + 64,), 77.0, dtype=dtype, device=DEV)
    hexi.hexi_rope_a2a_pack(rope, segs, xd, packed, lists, rotate, positions=posd)
    torch.cuda.synchronize()
    keep = ~torch.tensor(rotate)[None, :, None]

    def want_of(t, inverse):
        y, b = turned(t.double(), pos, freq, axis, adjacent, inverse)
        return torch.where(keep, t.double(), y), torch.where(keep, torch.zeros_like(b), b)

    y, b = want_of(x, False)
    close(packed[:total], _parts(y, lists), _parts(b, lists), dtype)
    assert torch.all(packed[total:] == 77.0)
    z = torch.randn(total, generator=g).to(dtype)
    y_wide = torch.full((rows, n * d + pad), 77.0, dtype=dtype, device=DEV)
    yd = torch.as_strided(y_wide, (rows, n, d), (n * d + pad, d, 1))
    hexi.hexi_rope_a2a_unpack(rope, segs, z.to(DEV), yd, lists, rotate, positions=posd)
    torch.cuda.synchronize()
    back = torch.from_numpy(a2a.a2a_unpack(z.double().numpy(), rows, n, d, lists, y=np.full((rows, n, d), 77.0)))
    w, b = want_of(back, True)
    listed = torch.ones(n, dtype=torch.bool)
    listed[order[n - 1]] = False
    close(yd[:, listed], w[:, listed], b[:, listed], dtype)
    assert torch.all(yd[:, ~listed] == 77.0) and torch.all(y_wide[:, n * d:] == 77.0)


def test_rope_on_as_many_rows_as_a_range_can_have():
    """2^31 - 1 rows of one head of 16 columns, in place (64 GiB): the first and last rows, and those around the ends of workgroups in the middle."""
    rows, d = 2 ** 31 - 1, 16
    if torch.cuda.mem_get_info()[0] < 80 * 2 ** 30:
        pytest.skip("needs 80 GiB of free device memory")
    freq, axis = freqs(d, 1)
    at = torch.tensor([0, 1, 895, 896, 2 ** 30 - 1, 2 ** 30, 1198372 * 896 - 1, 1198372 * 896, rows - 1024, rows - 2, rows - 1])
    x = torch.randn(len(at), 1, d, generator=torch.Generator().manual_seed(2)).to(BF16)
    big = torch.zeros(rows, 1, d, dtype=BF16, device=DEV)
    for i, r in enumerate(at.tolist()):
        big[r] = x[i].to(DEV)
    hexi.hexi_rope(hexi.make_rope(d, freq, axis), [(0, rows)], [(big, big)])
    torch.cuda.synchronize()
    got = torch.stack([big[r] for r in at.tolist()])
    close(got, *turned(x.double(), at[None], freq, axis, False, False), BF16)
    beside = torch.stack([big[r] for r in (2, 894, 2 ** 30 + 1, rows - 3)])
    assert torch.all(beside == 0)
    del big
    torch.cuda.empty_cache()
