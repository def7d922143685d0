"""What the binding makes of a workspace tensor, without a GPU: a library in its place records the calls."""
import pytest
import torch

from paper_2605_07569_amd import hexi


class Recorder:
    def __init__(self):
        self.calls = []

    def hexi_attn_win_bwd_workspace_bytes(self, *args):
        return 4096

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return hexi.HEXI_OK
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Recorder()
    hexi._types()
    monkeypatch.setattr(hexi, "_lib", lib)
    monkeypatch.setattr(hexi, "_current_device", lambda: -1)      # that of CPU tensors
    monkeypatch.setattr(hexi, "_stream", lambda stream: 0)
    return lib


def _calls(workspace):
    q, k = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(8, 2, 128, dtype=torch.bfloat16)
    o, lse, dk = torch.zeros(4, 8, 128), torch.zeros(8, 4), torch.zeros(8, 2, 128)
    desc, win, segs = hexi.desc_for(q, k, 0.1), hexi.make_window(3, 1), ([(4, 4)], [(0, 8)])
    yield lambda: hexi.hexi_attn_win_fwd_chunk(desc, win, *segs, q, k, k, o, lse, workspace=workspace)
    yield lambda: hexi.hexi_attn_win_bwd_chunk(desc, win, *segs, q, k, k, o, q, lse, lse.clone(), o.clone(), dk, dk.clone(), workspace=workspace)


def test_a_workspace_whose_elements_do_not_lie_side_by_side_is_refused(library):
    """numel() elements from its first one on would not all be its own."""
    for workspace in (torch.zeros(1, dtype=torch.uint8).expand(4096), torch.zeros(8192, dtype=torch.uint8)[::2], torch.zeros(64, 64).T[:, :32]):
        for call in _calls(workspace):
            with pytest.raises(hexi.HexiError) as e:
                call()
            assert e.value.code == hexi.HEXI_EINVAL
    assert not library.calls


def test_a_workspace_is_handed_on_with_its_bytes(library):
    whole = torch.zeros(64, 64)
    for workspace in (whole, whole[32:], torch.zeros(4096, dtype=torch.uint8), whole.T.T):
        for call in _calls(workspace):
            library.calls.clear()
            call()
            (_, args), = library.calls
            assert workspace.data_ptr() in args and workspace.numel() * workspace.element_size() in args
