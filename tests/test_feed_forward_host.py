"""The feed-forward layers' side of the binding, on the CPU, with tensors that only
claim to be on GPUs: what does not fit or is not on the layer's GPU is refused
before any launch, and launches go to that GPU also where another one is current."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1911_08076_amd import api
from paper_1911_08076_amd import feed_forward as F

BF16, F32 = torch.bfloat16, torch.float32


class Launches:
    """Stands for the binding: notes each launch and the GPU that was current."""
    current = 0

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        if name.endswith("_desc"):
            return getattr(api, name)
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
    monkeypatch.setattr(F, "P", p)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: Launches.current)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    with FakeTensorMode():
        yield p


def empty(*shape, dtype=BF16, dev="cuda:0"):
    return torch.empty(*shape, dtype=dtype, device=dev)


def test_weights_that_do_not_fit_are_refused(launches):
    for w in (empty(4, 64, dev="cpu"), empty(64), empty(8, 64).t(), empty(0, 64), empty(4, 0),
              empty(4, 64, dtype=torch.float64)):
        with pytest.raises(ValueError):
            F.F4Linear(w)
    w, down = empty(96, 64), empty(64, 96)
    for args in ((w, empty(95, 64), down), (w, w, w), (w, w, empty(64, 96, dev="cuda:1")),
                 (w, empty(96, 64, dev="cpu"), down), (w, w, down, "relu")):
        with pytest.raises(ValueError):
            F.FeedForward(*args)
    assert launches.seen == []


def test_tensors_without_dimensions_are_refused(launches):
    with pytest.raises(ValueError):
        F.F4Weight(empty(1)[0])
    with pytest.raises(ValueError):
        F.token_logprobs(empty(1)[0])
    assert launches.seen == []


def test_values_of_a_type_that_is_not_known_are_refused(launches):
    weight = F.F4Weight(empty(96, 64))
    launches.seen.clear()
    for dtype in (torch.float64, torch.int32):
        with pytest.raises(ValueError):
            weight.values(dtype)
    assert launches.seen == []
    assert weight.values(F32).dtype == F32 and weight.values(BF16).shape == (96, 64)


@pytest.mark.parametrize("x", [
    lambda: empty(3, 64, dev="cpu"), lambda: empty(3, 64, dev="cuda:1"), lambda: empty(3, 63),
    lambda: empty(3, 64, dtype=F32), lambda: empty(64, 3).t(), lambda: empty(64)])
def test_rows_that_do_not_fit_are_refused(launches, x):
    layers = (F.F4Linear(empty(96, 64)), F.FeedForward(empty(96, 64), empty(96, 64), empty(64, 96)),
              F.Classifier(empty(96, 64)))
    launches.seen.clear()
    for layer in layers:
        with pytest.raises(ValueError):
            layer(x())
    assert launches.seen == []


@pytest.mark.parametrize("out", [
    lambda n: empty(3, n, dev="cuda:1"), lambda n: empty(2, n), lambda n: empty(3, n - 1),
    lambda n: empty(n, 3).t(), lambda n: empty(3, n, dtype=torch.int32)])
def test_outputs_that_do_not_fit_are_refused(launches, out):
    for n, layer in ((96, F.F4Linear(empty(96, 64))),
                     (64, F.FeedForward(empty(96, 64), empty(96, 64), empty(64, 96)))):
        launches.seen.clear()
        with pytest.raises(ValueError):
            layer(empty(3, 64), out=out(n))
        assert launches.seen == []
    with pytest.raises(ValueError):
        layer(empty(3, 64), out=empty(3, 64, dtype=F32))     # a block gives x's type
    with pytest.raises(ValueError):
        F.F4Linear(empty(96, 64))(empty(3, 64), out=empty(3, 96), dtype=F32)


def test_an_output_over_the_input_is_refused(launches, monkeypatch):
    monkeypatch.setattr(F, "_overlap", lambda a, b: a is b)     # these have no addresses
    layer, x = F.F4Linear(empty(64, 64)), empty(3, 64)
    launches.seen.clear()
    with pytest.raises(ValueError):
        layer(x, out=x)
    assert launches.seen == []


def test_overlaps():
    rows = torch.empty(8, 64, dtype=BF16)
    assert F._overlap(rows, rows) and F._overlap(rows[:3], rows[2:5]) and F._overlap(rows[2:5], rows)
    assert not F._overlap(rows[:3], rows[3:]) and not F._overlap(rows[3:], rows[:3])
    assert not F._overlap(rows, torch.empty_like(rows)) and not F._overlap(rows[:0], rows)


def test_logits_and_tokens_that_do_not_fit_are_refused(launches):
    good = empty(3, 50, dtype=F32)
    for x in (empty(3, 50, dev="cpu"), empty(50), empty(50, 3).t(), empty(3, 50, dtype=torch.int32)):
        with pytest.raises(ValueError):
            F.token_logprobs(x)
    for t in (empty(3, dtype=torch.int64), empty(4, dtype=torch.int32),
              empty(3, dtype=torch.int32, dev="cuda:1"), empty(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            F.token_logprobs(good, t)
    assert launches.seen == []


def test_a_classifier_refuses_tokens_before_its_product(launches):
    classifier = F.Classifier(empty(50, 64))
    launches.seen.clear()
    for t in (empty(3, dtype=torch.int64), empty(4, dtype=torch.int32), empty(3, 1, dtype=torch.int32),
              empty(3, dtype=torch.int32, dev="cuda:1"), empty(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            classifier(empty(3, 64), t)
    assert launches.seen == []
    classifier(empty(3, 64), empty(3, dtype=torch.int32))
    assert [name for name, _ in launches.seen] == ["ifq_f4_matmul", "ifq_logprobs"]


@pytest.mark.parametrize("dev", ["cuda:0", "cuda:1"])
def test_launches_go_to_the_layers_gpu(launches, dev):
    feed = F.FeedForward(empty(96, 64, dev=dev), empty(96, 64, dev=dev), empty(64, 96, dev=dev),
                         "gelu")
    classifier = F.Classifier(empty(50, 64, dev=dev))
    y = feed(empty(3, 64, dev=dev))
    assert y.shape == (3, 64) and y.device == torch.device(dev) and y.dtype == BF16
    got = classifier(y, empty(3, dtype=torch.int32, dev=dev), top=4)
    assert got.logprob.shape == got.entropy.shape == (3,)
    assert got.top_logprobs.shape == got.top_tokens.shape == (3, 4)
    assert [n for n, _ in launches.seen[:7]] == 4 * ["ifq_f4_quantize"] + [
        "ifq_f4_gated", "ifq_f4_matmul", "ifq_f4_matmul"]
    assert launches.seen[7][0] == "ifq_logprobs"
    assert {index for _, index in launches.seen} == {torch.device(dev).index}
    assert Launches.current == 0


def test_no_rows_launch_no_product(launches):
    feed = F.FeedForward(empty(96, 64), empty(96, 64), empty(64, 96))
    launches.seen.clear()
    assert feed(empty(0, 64)).shape == (0, 64) and launches.seen == []
