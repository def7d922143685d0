"""Tensors of one rotation that are written where another one is read or written: refused before anything is launched."""
import ctypes

import pytest

from paper_2605_07569_amd import hexi


@pytest.mark.parametrize("pairs", [[(16, 16), (16, 16)], [(16, 64), (32, 64)], [(16, 64), (64, 128)], [(64, 128), (16, 64)], [(16, 16), (32, 48), (64, 48)], [(16, 32), (48, 64), (80, 96), (96, 112)]])
def test_a_result_of_one_tensor_is_not_part_of_another(pairs):
    rope = hexi.make_rope(64, [1.0] * 32)
    arr = (hexi.hexi_rope_tensor * len(pairs))(*[hexi.hexi_rope_tensor(x, y, 2, 128, 64, 128, 64) for x, y in pairs])
    call = lambda n: hexi.load().hexi_rope(ctypes.byref(rope), ctypes.byref(hexi.make_range([(0, 4)])[0]), None, 0, arr, n, hexi.HEXI_F32, hexi.HEXI_F32, 0, None)
    assert call(len(pairs)) == hexi.HEXI_EINVAL and "tensor" in hexi.hexi_last_error()
