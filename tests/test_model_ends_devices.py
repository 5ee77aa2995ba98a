"""Where the operators at the ends of a model run: on the current device, with tensors, workspace and stream of that
device; anything else is refused before a kernel is launched. Stand-ins take the place of device tensors: no GPU."""
import pytest
import torch

from paper_2609_37842_amd import eogp as E


class OnDevice:
    """What the checks ask of a tensor (or stream) of device `index`, -1 for the host."""

    def __init__(self, index):
        self.index = self.device_index = index
        self.is_cuda = index >= 0

    def get_device(self):
        return self.index


@pytest.fixture
def device_0(monkeypatch):
    monkeypatch.setattr(E, "_current_device", lambda: 0)


CALLS = {
    "embed": lambda t, **k: E.eogp_embed_tokens(t[0], t[1], **k),
    "embed_backward": lambda t, **k: E.eogp_embed_backward(t[0], t[1], 5, **k),
    "norm": lambda t, **k: E.eogp_layer_norm(t[0], t[1], **k),
    "norm_backward": lambda t, **k: E.eogp_layer_norm_backward(t[0], t[1], None, t[0], t[0], **k),
    "xent": lambda t, **k: E.eogp_softmax_xent(t[0], t[1], **k),
    "sample": lambda t, **k: E.eogp_sample_tokens(t[0], t[1], **k),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(name, device_0):
    for pair in ([OnDevice(1), OnDevice(1)], [OnDevice(0), OnDevice(1)], [OnDevice(1), OnDevice(0)]):
        with pytest.raises(ValueError, match="current device cuda:0, not cuda:1"):
            CALLS[name](pair)
    with pytest.raises(ValueError, match="device tensors"):
        CALLS[name]([OnDevice(0), OnDevice(-1)])


@pytest.mark.parametrize("name", CALLS)
def test_a_stream_of_another_device_is_refused(name, device_0):
    with pytest.raises(ValueError, match="stream must belong to the current device cuda:0, not cuda:1"):
        CALLS[name]([OnDevice(0), OnDevice(0)], stream=OnDevice(1))


@pytest.mark.parametrize("name", ["embed_backward", "norm_backward"])
def test_a_workspace_elsewhere_is_refused(name, device_0):
    for where, match in ((-1, "device tensors"), (1, "not cuda:1")):
        with pytest.raises(ValueError, match=match):
            CALLS[name]([OnDevice(0), OnDevice(0)], ws=OnDevice(where))


def test_a_workspace_is_one_piece_of_memory():
    """Expanded and strided workspaces have fewer bytes, or others, than their element count says."""
    for ws in (torch.empty(1, dtype=torch.uint8).expand(4096), torch.empty(8192, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            E._scratch(4096, ws.device, ws, None)
    with pytest.raises(ValueError, match="workspace needs 4096"):
        E._scratch(4096, torch.device("cpu"), torch.empty(4095, dtype=torch.uint8), None)
    ws = torch.empty(2048, dtype=torch.int16)
    assert E._scratch(4096, ws.device, ws, None) == (ws, 4096)
    assert E._scratch(0, ws.device, None, None) == (None, 0)
