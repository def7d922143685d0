"""Which windowed kernels the GPU tests run, by the rules that the launchers use: every one of them, at both head_dims."""
import os
import subprocess

import pytest

import window_util as wu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32 = 0, 1


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    """units(cases, dtype, d): of every case the forward's units (rows of a unit, whether its keys are split; 0 rows: few rows), dQ's rows, and dK / dV's keys and whether
    the rows behind them are cut into parts."""
    hipcc = "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("window") / "window_shapes_check")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2605_07569_amd", "csrc"),
                           os.path.join(ROOT, "tests", "host", "window_shapes_check.cpp"), "-o", exe])
    text = lambda segs: f"{len(segs)} " + " ".join(f"{s} {n}" for s, n in segs)

    def ask(cases, dtype, d, plain=False):
        lines = [f"{dtype} {c.nq} {c.nkv} {d} {min(c.window, 2 ** 31 - 1)} {min(c.n_sink, 2 ** 31 - 1)} {text(c.q_segs)} {text(c.kv_segs)}" for c in cases]
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        if plain:      # the forward's rows of a unit and number of splits
            return [tuple(map(int, line.split()[0][3:].split(":"))) for line in out]
        split = lambda word, name: (int(word[len(name):].split(":")[0]), word.split(":")[1] != "1")
        return [(split(f, "fwd"), int(q[2:]), split(k, "dkdv")) for f, q, k in (line.split() for line in out)]

    return ask


@pytest.mark.parametrize("d", [64, 128])
def test_the_lists_take_the_units_that_they_are_made_for(units, d):
    for dtype in (BF16, F32):
        assert [x[0] for x in units(wu.FORWARD_64, dtype, d)] == [(64, False)] * len(wu.FORWARD_64)
    assert [x[0] for x in units(wu.FORWARD_64_SPLITS, BF16, d)] == [(64, True)] * len(wu.FORWARD_64_SPLITS)
    assert [x[1:] for x in units(wu.BACKWARD_64, F32, d)] == [(64, (64, c.name.startswith("parts"))) for c in wu.BACKWARD_64]


@pytest.mark.parametrize("d", [64, 128])
def test_every_kernel_is_run(units, d):
    taken = lambda lists, dtype: [x for cases in lists for x in units(cases, dtype, d)]
    fwd = lambda lists, dtype: {x[0] for x in taken(lists, dtype)}
    shared = [wu.CASES, wu.FORWARD_64, wu.FORWARD_64_SPLITS]
    both = lambda rows: {(r, cut) for r in rows for cut in (False, True)}
    assert fwd(shared + ([wu.LARGE] if d == 128 else []), BF16) == both((0, 32, 64)) | ({(256, False)} if d == 128 else set())
    assert fwd(shared, F32) == both((0, 16)) | {(64, False)}
    assert {x[2] for x in taken([wu.CASES, wu.PARTS, wu.MANY, [wu.MANY_PARTS]], BF16)} == both((32, 64))
    fp32 = taken([wu.CASES, wu.PARTS, wu.BACKWARD_64], F32)
    assert {x[1] for x in fp32} == {16, 64} and {x[2] for x in fp32} == both((16, 64))
