"""Where axon_rope_table makes its table. Nothing here touches a GPU."""
import pytest

torch = pytest.importorskip("torch")
from test_kv_devices import Tensor, ax  # noqa: E402, F401


@pytest.fixture
def made(ax, monkeypatch):  # noqa: F811
    devices = []

    def empty(*shape, device, **k):
        devices.append(torch.device(device))
        return Tensor(shape, torch.float32, torch.device(device).index)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(ax, "_current_device", lambda: 1)
    monkeypatch.setattr(ax, "_raw_stream", lambda index: 0)
    return devices


@pytest.mark.parametrize("device", [None, "cuda", "cuda:1", 1, torch.device("cuda"), torch.device("cuda", 1)], ids=str)
def test_the_current_device(ax, made, device):  # noqa: F811
    ax.axon_rope_table(32, 64, 1e4, device=device)
    assert made == [torch.device("cuda", 1)] and ax._calls == ["axon_rope_table"]


@pytest.mark.parametrize("device", ["cuda:0", 0])
def test_another_device_is_refused(ax, made, device):  # noqa: F811
    with pytest.raises(ValueError):
        ax.axon_rope_table(32, 64, 1e4, device=device)
    assert not made and not ax._calls


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu")], ids=str)
def test_other_kinds_of_device_are_refused(ax, made, device):  # noqa: F811
    with pytest.raises(TypeError):
        ax.axon_rope_table(32, 64, 1e4, device=device)
    assert not made and not ax._calls
