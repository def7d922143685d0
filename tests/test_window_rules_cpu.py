"""The launch rules of the windowed kernels against the timings that they were fitted to: the choice they make is, on average, within a few percent of the fastest measured one."""
import os

import pytest

from test_window_units_cpu import BF16, F32, ROOT, units  # noqa: F401 (a fixture)
from window_util import Case

TIMINGS = os.path.join(ROOT, "profiles", "windowed_rules")


def read(name):
    path = os.path.join(TIMINGS, name)
    if not os.path.exists(path):
        pytest.skip("the timings are not in this tree")
    return [[float(x) for x in line.split()] for line in open(path) if line[0] != "#"]


def step(nq, nkv, rows, window):
    """The calls that were timed: a shard behind its halo."""
    return Case("", [(int(window) + 100, int(rows))], [(101, int(rows) + int(window) - 1)], int(window), 0, int(nq), int(nkv))


def mean_loss(pairs):
    """Mean of the chosen time over the fastest one."""
    assert pairs
    return sum(chosen / min(t for t in times if t > 0) for chosen, times in pairs) / len(pairs)


def test_bf16_forward_units_and_splits(units):  # noqa: F811
    splits, losses, few = (1, 2, 4, 8, 16, 32), [], 0
    for d in (64, 128):
        rows = [r for r in read("bf16_forward.txt") if r[0] == d]
        cases = [step(*r[1:5]) for r in rows]
        taken = units(cases, BF16, d, plain=True)
        for r, (size, n) in zip(rows, taken):
            if size not in (32, 64) or n not in splits:
                few += 1
                continue
            chosen = r[5 + (6 if size == 32 else 0) + splits.index(n)]
            if chosen > 0:
                losses.append((chosen, r[5:]))
    assert len(losses) > 250 and mean_loss(losses) < 1.02, (len(losses), few, mean_loss(losses))


def test_bf16_backward_units(units):  # noqa: F811
    losses = []
    for d in (64, 128):
        rows = [r for r in read("bf16_backward.txt") if r[0] == d]
        for r, (_, dq, _) in zip(rows, units([step(*r[1:5]) for r in rows], BF16, d)):
            losses.append((r[8] if dq == 32 else r[5], (r[5], r[8])))
    assert len(losses) == 900 and mean_loss(losses) < 1.01, mean_loss(losses)


@pytest.mark.parametrize("part,at", [("forward", (5, 6)), ("dq", (8, 11)), ("dkdv", (9, 12))])
def test_fp32_units(units, part, at):  # noqa: F811
    losses = []
    for d in (64, 128):
        rows = [r for r in read("fp32.txt") if r[0] == d]
        for r, (fwd, dq, dkdv) in zip(rows, units([step(*r[1:5]) for r in rows], F32, d)):
            size = {"forward": fwd[0], "dq": dq, "dkdv": dkdv[0]}[part]
            if r[at[0]] > 0 and size in (16, 64) and not (part == "forward" and fwd[1]):
                losses.append((r[at[0] if size == 64 else at[1]], (r[at[0]], r[at[1]])))
    assert len(losses) > 100 and mean_loss(losses) < 1.02, (len(losses), mean_loss(losses))


def test_bf16_forward_in_256_row_workgroups(units):  # noqa: F811
    rows = read("bf16_forward_256.txt")
    taken = [x[0][0] for x in units([step(*r[:4]) for r in rows], BF16, 128)]
    losses = [(r[5] if size == 256 else r[4], r[4:]) for r, size in zip(rows, taken)]
    assert len(losses) == 45 and mean_loss(losses) < 1.02, mean_loss(losses)
