"""The rotation's launch for every number of rows that a range can have: all rows once, fewer than 2^32 threads, no arithmetic past 32 bits (UBSan)."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LAST = 2 ** 31 - 1


def test_the_launch_covers_the_rows(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "rope_shape_check")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-I", "/opt/rocm/include",
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2605_07569_amd", "csrc"), os.path.join(ROOT, "tests", "host", "rope_shape_check.cpp"), "-o", exe])
    rng = random.Random(1)
    rows = [1, 2, 1023, 1024, 1025, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, LAST - 1024, LAST - 1023, LAST - 1022, LAST - 895, LAST - 1, LAST] + [int(2 ** rng.uniform(0, 31)) - 1 or 1 for _ in range(60)]
    asked = [(n, p) for n in rows for p in (1, 2, 3, 8, 320, 447, 448, 449, 895, 896, 897, 8 * 65535, 4 * 16 * 65535)]
    out = subprocess.run([exe], input="".join(f"{n} {p}\n" for n, p in asked), capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    for (n, p), line in zip(asked, out.stdout.splitlines()):
        tokens, grid = map(int, line.split())
        assert tokens >= 1 and (grid - 1) * tokens < n <= grid * tokens and grid * 256 < 2 ** 32, (n, p, tokens, grid)
        # a pass of the workgroup, and a thousand workgroups, where they do not need fewer
        want = min(max(896 // p, 1), -(-n // 1024))
        assert tokens == max(want, -(-n // (2 ** 24 - 1))), (n, p, tokens)
