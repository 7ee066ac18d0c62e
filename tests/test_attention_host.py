"""The layers' side of the binding, on the CPU, with tensors that only claim to be on
GPUs: what is not on the layer's GPU is refused before any launch, and launches go to
that GPU also where another one is torch's current."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1911_08076_amd import attention as A
from paper_1911_08076_amd import api

BF16 = torch.bfloat16


class Launches:
    """Stands for the binding: notes each launch and the GPU that was current."""
    current = 0

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        if name.endswith("_desc"):
            return getattr(api, name)
        if name == "ifq_kv_cache_bytes":
            return lambda desc: 4096
        if name.endswith("_workspace_bytes"):
            return lambda desc: 64
        return lambda *args, **kw: self.seen.append((name, Launches.current))


class Device:
    """Stands for torch.cuda.device."""

    def __init__(self, device):
        self.index = torch.device(device).index

    def __enter__(self):
        self.before, Launches.current = Launches.current, self.index

    def __exit__(self, *args):
        Launches.current = self.before


@pytest.fixture
def launches(monkeypatch):
    Launches.current = 0
    p = Launches()
    monkeypatch.setattr(A, "P", p)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: Launches.current)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    with FakeTensorMode():
        yield p


def layer(dev="cuda:0", dev2=None):
    w1 = torch.empty(256, 64, dtype=BF16, device=dev)
    w2 = torch.empty(64, 128, dtype=BF16, device=dev2 or dev)
    return A.AttentionLayer(w1, w2, 2, 1, 64, num_pages=4, max_pages=2, page_tokens=32, rot_dim=0)


def arguments(dev):
    return {"x": torch.empty(3, 64, dtype=BF16, device=dev),
            "offsets": torch.empty(2, dtype=torch.int32, device=dev),
            "lengths": torch.empty(1, dtype=torch.int32, device=dev),
            "pages": torch.empty(1, 2, dtype=torch.int32, device=dev),
            "out": torch.empty(3, 64, dtype=BF16, device=dev)}


@pytest.mark.parametrize("elsewhere", ["cpu", "cuda:1"])
@pytest.mark.parametrize("name", ["x", "offsets", "lengths", "pages", "out"])
def test_what_is_not_on_the_layers_gpu_is_refused(launches, name, elsewhere):
    attend = layer()
    launches.seen.clear()
    args = arguments("cuda:0")
    args[name] = args[name].to(elsewhere)
    with pytest.raises(ValueError, match="cuda:0"):
        attend(**args, max_q=3)
    assert launches.seen == []


def test_weights_off_the_gpu_or_on_two_are_refused(launches):
    for dev, dev2 in (("cpu", None), ("cuda:0", "cpu"), ("cuda:0", "cuda:1")):
        with pytest.raises(ValueError):
            layer(dev, dev2)
    assert launches.seen == []


@pytest.mark.parametrize("change", [(3, 63), (2, 64)])
def test_an_output_that_does_not_fit_is_refused_before_the_append(launches, change):
    attend = layer()
    launches.seen.clear()
    args = arguments("cuda:0")
    args["out"] = torch.empty(*change, dtype=BF16, device="cuda:0")
    with pytest.raises(ValueError):
        attend(**args, max_q=3)
    assert launches.seen == []


@pytest.mark.parametrize("dev", ["cuda:0", "cuda:1"])
def test_launches_go_to_the_layers_gpu(launches, dev):
    attend = layer(dev)
    attend(**arguments(dev), max_q=3)
    attend.qkv(torch.empty(5, 64, dtype=BF16, device=dev))
    assert [n for n, _ in launches.seen] == 2 * ["ifq_f8_quantize"] + [
        "ifq_f8_quantize", "ifq_f8_matmul", "ifq_kv_append", "ifq_kv_attention",
        "ifq_f8_quantize", "ifq_f8_matmul", "ifq_f8_quantize", "ifq_f8_matmul"]
    assert {index for _, index in launches.seen} == {torch.device(dev).index}
    assert Launches.current == 0
