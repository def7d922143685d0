"""Windowed attention by its definition in float64, with elementwise error bounds, and the cases that the tests share.

Bounds.  u = 2^-24 is half a step of fp32, h = 2^-8 half a step of bf16 (0 for fp32 inputs: nothing is rounded to fewer bits there).
A score is a sum of d products and a few more roundings: |error| <= (d + 16) u scale sum |q k| + 16 u (|s| + |m|), m the value that is
subtracted from it before the exponential (a row's LSE here: the reference of the kernels is within a few units of it).  Exponentials
and the sums' own roundings are counted as 2^-20 and n u relative.  E_ij: what that makes of P_ij, relative.  P and dS are rounded to
bf16 as operands (h each, the sum that normalises o is that of the rounded P: at most h (sum w |v| + |o|)), results to the
type they are asked for in (h or u)."""
from dataclasses import dataclass, field, replace
from typing import List, Optional

import torch

U, H = 2.0 ** -24, 2.0 ** -8


@dataclass
class Case:
    name: str
    q_segs: list
    kv_segs: list
    window: int
    n_sink: int
    nq: int = 2
    nkv: int = 1
    kv_of_q: Optional[List[int]] = None
    k_scale: float = 1.0
    pad: int = 0                     # extra columns between heads and tokens of the inputs

    @property
    def lq(self):
        return sum(n for _, n in self.q_segs)

    @property
    def lc(self):
        return sum(n for _, n in self.kv_segs)

    @property
    def heads(self):
        return self.kv_of_q or [h // (self.nq // self.nkv) for h in range(self.nq)]


BIG = 2 ** 31 - 2
CASES = [
    Case("one key", [(5, 1)], [(5, 1)], 1, 0),
    Case("one row", [(600, 1)], [(0, 3), (401, 200)], 200, 3, nq=8),
    Case("halo", [(300, 200)], [(0, 3), (264, 236)], 37, 3, nq=3),
    Case("window of one", [(10, 100)], [(0, 110)], 1, 0, nq=4, nkv=2),
    Case("zigzag", [(128, 130), (1000, 70)], [(0, 5), (100, 158), (901, 169)], 100, 5, nq=4, nkv=2),
    Case("whole sequence", [(0, 333)], [(0, 333)], 64, 33, nq=2, nkv=2, k_scale=3.0),
    Case("window ends at block edges", [(256, 128)], [(128, 256)], 128, 0),
    Case("step before the shard", [(500, 300)], [(200, 300)], 128, 210, nq=3),          # later rows see 10 sinks alone
    Case("step too far back", [(5000, 70)], [(1000, 90)], 128, 0),                       # nothing is seen
    Case("step in the future", [(100, 70)], [(170, 65)], 128, 400),
    Case("sinks alone", [(9000, 65)], [(0, 40)], 16, 33),
    Case("sinks reach the window", [(150, 100)], [(0, 250)], 60, 120),
    Case("sinks past the rows", [(10, 150)], [(0, 300)], 8, 1000),
    Case("window past everything", [(40, 260)], [(0, 300)], 10 ** 12, 0, nq=5, nkv=2, kv_of_q=[0, 1, 1, 0, 1]),
    Case("gaps", [(7 + 50 * i, 1 + 2 * i) for i in range(16)], [(40 * i, 3 + 2 * i) for i in range(16)], 45, 50, nq=3, nkv=1),
    Case("rows without keys", [(0, 70), (500, 70)], [(30, 20), (490, 30)], 25, 0),
    Case("far positions", [(BIG - 199, 200)], [(0, 4), (BIG - 260, 261)], 50, 4),
    Case("huge window at far positions", [(BIG - 99, 100)], [(0, 4), (BIG - 160, 161)], 2 ** 40, 2 ** 40),
    Case("strides", [(70, 90)], [(20, 140)], 33, 0, nq=3, nkv=3, pad=16),
    Case("long", [(3000, 520)], [(0, 17), (1977, 1543)], 1024, 17, nq=4, nkv=1),
    Case("one token", [(60000, 1)], [(0, 4), (57000, 3001)], 2990, 4, nq=8),
    Case("one token, heads of their own", [(5000, 1)], [(0, 4), (3000, 2001)], 1990, 4, nq=3, nkv=3),
    Case("one token, a block", [(500, 1)], [(0, 4), (440, 61)], 50, 4, nq=4, nkv=2),
    Case("one token, a few blocks", [(500, 1)], [(0, 4), (300, 201)], 190, 4, nq=4, nkv=2),
    Case("two tokens, nine blocks", [(500, 2)], [(0, 502)], 511, 0, nq=4, nkv=1),
    Case("three tokens", [(900, 2), (1200, 1)], [(0, 70), (300, 901)], 700, 60, nq=5, nkv=2, kv_of_q=[1, 0, 1, 1, 1]),
    Case("few rows", [(4000, 70)], [(0, 300), (1500, 2570)], 2500, 100, nq=2, nkv=2),
    Case("long odd", [(2001, 431)], [(101, 2331)], 1901, 0, nq=2, nkv=2, k_scale=2.0),
]

# Steps whose forward takes 256-row workgroups (128 heads of up to 512 rows: 256 of them): windows within a tile and over several, sinks, rows of two places in
# one workgroup, rows that see nothing, a whole group of rows past the end, chunks whose first keys every row sees
LARGE = [
    Case("one", [(900, 511)], [(0, 3), (800, 611)], 1, 3, nq=128, nkv=2),
    Case("short", [(900, 512)], [(0, 70), (800, 612)], 70, 64, nq=128, nkv=2),
    Case("pair", [(300, 300), (5000, 201)], [(0, 130), (200, 400), (4600, 601)], 333, 128, nq=128, nkv=1),
    Case("ring step", [(700, 512)], [(100, 600)], 800, 0, nq=128, nkv=4),
    Case("odd", [(2000, 449)], [(900, 1549)], 1024, 0, nq=128, nkv=1, k_scale=3.0),
    Case("rows without keys", [(50, 60), (3000, 452)], [(300, 2500)], 10 ** 6, 0, nq=128, nkv=1),
    Case("group past the end", [(4000, 1380)], [(1001, 4379)], 3000, 0, nq=42, nkv=1),
    Case("gap", [(100, 200), (9000, 290)], [(0, 300), (8500, 64), (8600, 690)], 700, 10, nq=128, nkv=128),
    Case("everything", [(200, 500)], [(0, 640)], 10 ** 9, 0, nq=128, nkv=2),
]

# The same steps with two q heads to a kv head: their backward takes 64-row workgroups, that of CASES 32-row ones.
MANY = [replace(c, nq=128, nkv=64) for c in LARGE]

# Steps whose dK / dV units walk their rows in parts: the sinks', all, both; keys behind the sinks in their tile, sinks that only some of the chunk's rows see, sinks elsewhere, a
# step in the future of most of them.
PARTS = [
    Case("sinks", [(100, 3000)], [(0, 3100)], 50, 20, nq=2, nkv=1),
    Case("sinks of two tiles", [(40, 2100), (9000, 901)], [(0, 70), (8700, 1201)], 300, 67, nq=6, nkv=2, kv_of_q=[0, 1, 1, 0, 1, 1]),
    Case("all", [(300, 2501)], [(0, 601)], 10 ** 6, 0, nq=8, nkv=1),
    Case("all and sinks", [(0, 3333)], [(0, 400)], 700, 33, nq=8, nkv=1, k_scale=2.0),
    Case("sinks elsewhere", [(5000, 3000)], [(4900, 700)], 101, 16, nq=2, nkv=1),
    Case("mostly in the future", [(0, 3001)], [(2800, 500)], 2500, 3000, nq=4, nkv=1),
    Case("strides", [(1000, 2222)], [(3, 5), (700, 2522)], 222, 7, nq=3, nkv=1, pad=16),
]
MANY_PARTS = Case("many heads", [(500, 1333)], [(0, 40), (460, 1373)], 40, 30, nq=64, nkv=8)

# Steps whose forward takes 64-row units, whole, in bf16 and fp32 at both head_dims
FORWARD_64 = [
    Case("mid-size", [(500, 333)], [(0, 9), (380, 453)], 121, 9, nq=64, nkv=16),
    Case("ring step", [(700, 300)], [(500, 230)], 150, 0, nq=96, nkv=8),                  # later rows see nothing
    Case("rows without keys", [(50, 60), (3000, 271)], [(300, 2500), (2890, 201)], 70, 0, nq=128, nkv=4),
    Case("gaps", [(7 + 50 * i, 11 + 2 * i) for i in range(16)], [(40 * i, 9 + 2 * i) for i in range(16)], 95, 50, nq=64, nkv=8, kv_of_q=[(5 * h + h // 7) % 8 for h in range(64)]),
    Case("strides", [(2000, 257)], [(1901, 356)], 101, 0, nq=60, nkv=12, k_scale=2.0, pad=16),
    Case("sinks of the step", [(9000, 259)], [(0, 130)], 64, 100, nq=64, nkv=64),
    Case("everything", [(40, 250)], [(0, 290)], 10 ** 9, 0, nq=96, nkv=32),
]
# and, in bf16, in splits of their keys
FORWARD_64_SPLITS = [
    Case("long window", [(8000, 40)], [(0, 8040)], 7001, 0, nq=32, nkv=8),
    Case("long window, sinks", [(8000, 60)], [(0, 70), (1000, 7060)], 7001, 67, nq=16, nkv=2, kv_of_q=[1, 0, 0, 1] * 4),
]
# Steps whose fp32 backward takes 64-row dQ and 64-key dK / dV units, whole and in parts (a name says which)
BACKWARD_64 = [
    Case("whole", [(40, 700)], [(0, 820)], 20, 0, nq=32, nkv=32),
    Case("whole, ring step", [(900, 1111)], [(300, 720)], 150, 0, nq=64, nkv=64),
    Case("whole, strides", [(900, 877)], [(0, 7), (889, 888)], 11, 5, nq=24, nkv=24, pad=16),
    Case("parts", [(500, 1133)], [(0, 5), (480, 1153)], 21, 3, nq=16, nkv=16),
    Case("parts, heads", [(900, 1377)], [(0, 40), (880, 1397)], 20, 37, nq=32, nkv=16, kv_of_q=[(5 * h + h // 7) % 16 for h in range(32)]),
]


def positions(segs):
    return torch.cat([torch.arange(s, s + n, dtype=torch.int64) for s, n in segs])


def visible(c):
    p, j = positions(c.q_segs)[:, None], positions(c.kv_segs)[None]
    return (j <= p) & ((p - j < c.window) | (j < c.n_sink))


def strided(x, pad, device):
    """x [rows, heads, d] as a slice of a wider buffer."""
    if pad == 0:
        return x.to(device)
    wide = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + pad), float("nan"), dtype=x.dtype)
    wide[:, :x.shape[1], :x.shape[2]] = x
    return wide.to(device)[:, :x.shape[1], :x.shape[2]]


def inputs(c, dtype, d, seed=0):
    g = torch.Generator().manual_seed(1000 * seed + 7)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float32)
    x = dict(q=n(c.lq, c.nq, d), k=n(c.lc, c.nkv, d) * c.k_scale, v=n(c.lc, c.nkv, d), d_o=n(c.lq, c.nq, d))
    return {name: t.to(dtype) for name, t in x.items()}


def forward(c, x, out):
    """o [lq, nq, d], lse [nq, lq] in float64 and bounds of their errors."""
    q, k, v = (x[n].double() for n in ("q", "k", "v"))
    d = q.shape[2]
    scale, seen, h = d ** -0.5, visible(c), H if x["q"].dtype == torch.bfloat16 else 0.0
    o, lse = torch.zeros_like(q), torch.full((c.nq, c.lq), float("-inf"), dtype=torch.float64)
    bo, bl = torch.zeros_like(o), torch.zeros_like(lse)
    zero = torch.zeros((), dtype=torch.float64)
    for i, j in enumerate(c.heads):
        s = torch.where(seen, scale * q[:, i] @ k[:, j].T, torch.tensor(float("-inf"), dtype=torch.float64))
        z = torch.logsumexp(s, 1)
        w = torch.where(seen, torch.exp(s - z[:, None].clamp(min=-1e300)), zero)
        mag = scale * q[:, i].abs() @ k[:, j].abs().T
        fin = torch.where(seen, s.abs() + z[:, None].abs().nan_to_num(0, 0, 0), zero)
        e = torch.where(seen, (d + 16) * U * mag + 16 * U * fin, zero).amax(1) + 2.0 ** -20 + (seen.sum(1) + 16) * U
        o[:, i], lse[i] = w @ torch.where(torch.isfinite(v[:, j]), v[:, j], zero), z
        wv = w @ v[:, j].abs().nan_to_num(0, 0, 0)
        bo[:, i] = (2 * e + 1.01 * h)[:, None] * (wv + o[:, i].abs()) + (1.01 * (H if out == torch.bfloat16 else U) * o[:, i].abs())
        bl[i] = 2 * e + 4 * U * z.abs().nan_to_num(0, 0, 0)
    return o, lse, bo, bl


def backward(c, x, o, lse, out):
    """delta, dq, dk, dv in float64 from the given o and lse, and bounds."""
    q, k, v, g = (x[n].double() for n in ("q", "k", "v", "d_o"))
    o, lse = o.double(), lse.double()
    d = q.shape[2]
    scale, seen, h = d ** -0.5, visible(c), H if x["q"].dtype == torch.bfloat16 else 0.0
    ho = H if out == torch.bfloat16 else 2 * U
    delta = (g * o).sum(2).T
    b_delta = (d + 8) * U * (g * o).abs().sum(2).T
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    bq, bk, bv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    zero = torch.zeros((), dtype=torch.float64)
    for i, j in enumerate(c.heads):
        live = seen & torch.isfinite(lse[i])[:, None]
        s = scale * q[:, i] @ k[:, j].T
        p = torch.where(live, torch.exp(torch.where(live, s - lse[i][:, None], zero)), zero)
        mag = scale * q[:, i].abs() @ k[:, j].abs().T
        e = torch.where(live, (d + 16) * U * mag + 16 * U * (s.abs() + lse[i].abs().nan_to_num(0, 0, 0)[:, None]), zero) + 2.0 ** -20
        dp = g[:, i] @ v[:, j].T - delta[i][:, None]
        b_dp = (d + 16) * U * (g[:, i].abs() @ v[:, j].abs().T) + b_delta[i][:, None] + 4 * U * delta[i].abs()[:, None]
        ds = p * dp
        b_ds = ds.abs() * (e + 1.01 * h) + 1.01 * p * b_dp
        n_r, n_c = (c.lc + 16) * U, (c.lq * c.nq + 16) * U
        dq[:, i] = scale * ds @ k[:, j]
        bq[:, i] = 1.01 * scale * (b_ds + n_r * ds.abs()) @ k[:, j].abs()
        dk[:, j] += scale * ds.T @ q[:, i]
        bk[:, j] += 1.01 * scale * (b_ds + n_c * ds.abs()).T @ q[:, i].abs()
        dv[:, j] += p.T @ g[:, i]
        bv[:, j] += 1.01 * (p * (e + 1.01 * h + n_c)).T @ g[:, i].abs()
    return dict(delta=(delta, b_delta + 2 * U * delta.abs()), dq=(dq, bq + 1.01 * ho * dq.abs()), dk=(dk, bk + 1.01 * ho * dk.abs()), dv=(dv, bv + 1.01 * ho * dv.abs()))


def within(name, got, want, bound, rel=None):
    """Elementwise within the bound; not finite exactly where the reference is not; and, for more than a few elements, relative L2 `rel`."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN elsewhere"
    assert torch.equal(got[~fin & ~want.isnan()], want[~fin & ~want.isnan()]), f"{name}: infinities differ"
    err = (got - want)[fin].abs()
    over = err > bound[fin] + 1e-30
    worst = float((err / (bound[fin] + 1e-30)).max()) if err.numel() else 0.0
    norm = float(want[fin].norm())
    l2 = float(err.norm()) / norm if norm else 0.0
    print(f"    {name}: rel-L2 {l2:.2e}, {worst:.2f} of the bound", flush=True)
    assert not bool(over.any()), f"{name}: {int(over.sum())} of {err.numel()} over the bound, worst {worst:.2f}"
    if rel is not None and norm:
        assert l2 <= rel, f"{name}: relative L2 {l2:.2e} > {rel}"
