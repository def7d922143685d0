"""Workspace sizes for descriptors, windows and lengths that the calls refuse: nothing is asked for."""
import pytest

from paper_2605_07569_amd import hexi


@pytest.mark.parametrize("change", [dict(dtype=5), dict(dtype=-1), dict(head_dim=96), dict(n_q_heads=0), dict(n_q_heads=129), dict(n_kv_heads=0), dict(n_kv_heads=9), dict(n_kv_heads=-1)], ids=str)
def test_no_workspace_for_what_is_refused(change):
    sizes = lambda desc, window: (hexi.hexi_attn_win_workspace_bytes(desc, window, 1, 100000), hexi.hexi_attn_win_bwd_workspace_bytes(desc, window, 16384, 100000))
    desc, window = hexi.make_desc(hexi.HEXI_BF16, 128, 8, 1, 0.1, (1024, 128), (128, 128)), hexi.make_window(1024, 4)
    assert all(sizes(desc, window))
    for name, value in change.items():
        setattr(desc, name, value)
    assert sizes(desc, window) == (0, 0)
