"""The accumulators of the windowed 64-row backward kernels in the code that is built: the check of tests/test_quad_accumulators_cpu.py on their file."""
import os
import subprocess

import pytest

from paper_2605_07569_amd import build
from test_quad_accumulators_cpu import kernels, violations

SRC = "hexi_bf16_quad_win.hip"


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if not os.path.exists(build._hipcc()):
        pytest.skip("hipcc not available")
    out = str(tmp_path_factory.mktemp("quad_win") / "quad_win.s")
    r = subprocess.run([build._hipcc()] + build.FLAGS + build.FILE_FLAGS.get(SRC, []) + ["--offload-device-only", "-S", os.path.join(build.CSRC, SRC), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    with open(out) as f:
        return f.read()


def test_nothing_touches_an_accumulator_before_it_has_settled(assembly):
    found = kernels(assembly)
    backward = {n: k for n, k in found.items() if "bwd_quad" in n}
    assert len(backward) == 2 and len(found) == 4
    for name, (ins, labels) in backward.items():
        assert sum(asm and code.startswith("v_mfma") for code, asm in ins) >= 32, name
        assert violations(ins, labels) == set(), name


def test_no_kernel_asks_the_dispatch_packet_for_its_size(assembly):
    # (it lies in host memory: a microsecond and more before anything else can start)
    assert ".amdhsa_user_sgpr_dispatch_ptr 1" not in assembly
