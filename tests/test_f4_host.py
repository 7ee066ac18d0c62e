"""Host side of the products with 4-bit weights and of log probabilities, on the
CPU: every refusal comes before a launch, empty calls launch nothing, workspaces
are asked for and passed on. Device pointers here are host addresses that no call
gets far enough to use."""
import ctypes

import pytest
import torch

import paper_1911_08076_amd as P
from paper_1911_08076_amd import _ffi

EINVAL, EUNSUP, EBUF = -1, -2, -4
BF16, F16, F32 = P.IFQ_TYPE_BF16, P.IFQ_TYPE_F16, P.IFQ_TYPE_F32
X = torch.zeros(4096, dtype=torch.uint8)
X = X[(-X.data_ptr()) % 64:]                 # 64-byte aligned
ODD = X[1:]


def refused(status, call, *args, **kw):
    with pytest.raises(P.IfqError) as e:
        call(*args, stream=0, **kw)
    assert e.value.status == status, e.value


def changed(d, change):
    for k, v in change.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), EINVAL), (dict(k=-1), EINVAL), (dict(rows=2 ** 31), EINVAL),
    (dict(x_type=3), EINVAL), (dict(x_type=-1), EINVAL), (dict(reserved=1), EINVAL),
    (dict(ld_x=64), EINVAL), (dict(ld_codes=47), EINVAL), (dict(ld_codes=32), EINVAL),
    (dict(ld_codes=56), EUNSUP), (dict(ld_x=2 ** 41), EINVAL), (dict(ld_codes=2 ** 41), EINVAL),
    (dict(rows=2 ** 30, k=2 ** 14, ld_x=2 ** 14, ld_codes=2 ** 13), EUNSUP)])
def test_weights_refuse_descriptors(change, status):
    d = changed(P.f4_weights_desc(4, 65, BF16), change)
    refused(status, P.ifq_f4_quantize, d, X, X, X)
    refused(status, P.ifq_f4_dequantize, d, X, X, X)


def test_weights_refuse_pointers():
    d = P.f4_weights_desc(4, 65, BF16)
    for args in ((None, X, X), (X, None, X), (X, X, None), (ODD, X, X), (X, X[8:], X),
                 (X, X, X[2:])):
        refused(EINVAL, P.ifq_f4_quantize, d, *args)
        refused(EINVAL, P.ifq_f4_dequantize, d, args[1], args[2], args[0])
    refused(EINVAL, P.ifq_f4_quantize, P.f4_weights_desc(4, 65, F32), X[2:], X, X)


BAD = [
    (dict(m=-1), EINVAL), (dict(n=-1), EINVAL), (dict(k=0), EINVAL), (dict(n=2 ** 31), EINVAL),
    (dict(x_type=F32), EINVAL), (dict(x_type=-1), EINVAL), (dict(y_type=3), EINVAL),
    (dict(reserved=1), EINVAL), (dict(ld_x=129), EINVAL), (dict(ld_w=79), EINVAL),
    (dict(ld_w=64), EINVAL), (dict(ld_w=88), EUNSUP), (dict(ld_w=2 ** 25 + 16), EUNSUP),
    (dict(ld_y=31), EINVAL), (dict(ld_x=2 ** 41), EINVAL),
    (dict(m=2 ** 30, n=2 ** 30, ld_y=2 ** 30), EUNSUP)]


@pytest.mark.parametrize("change,status", BAD + [(dict(activation=1), EINVAL)])
def test_product_refuses_descriptors(change, status):
    d = changed(P.f4_matmul_desc(8, 32, 130, BF16), change)
    refused(status, P.ifq_f4_matmul, d, X, X, X, X)
    assert P.ifq_f4_matmul_workspace_bytes(d) == 0 and P.ifq_f4_matmul_kernel_name(d) == ""


@pytest.mark.parametrize("change,status", BAD + [(dict(activation=0), EINVAL),
                                                 (dict(activation=4), EINVAL),
                                                 (dict(activation=-1), EINVAL)])
def test_gated_refuses_descriptors(change, status):
    d = changed(P.f4_matmul_desc(8, 32, 130, BF16, activation=P.IFQ_ACT_SILU), change)
    refused(status, P.ifq_f4_gated, d, X, X, X, X, X, X)
    assert P.ifq_f4_gated_workspace_bytes(d) == 0 and P.ifq_f4_gated_kernel_name(d) == ""


def test_products_refuse_pointers():
    d = P.f4_matmul_desc(8, 32, 130, BF16, F32)
    good = [X] * 4
    for i in range(4):
        refused(EINVAL, P.ifq_f4_matmul, d, *(good[:i] + [None] + good[i + 1:]))
    for i, p in ((0, ODD), (1, X[8:]), (2, X[2:]), (3, X[2:])):
        refused(EINVAL, P.ifq_f4_matmul, d, *(good[:i] + [p] + good[i + 1:]))
    d.activation = P.IFQ_ACT_GELU
    good = [X] * 6
    for i in range(6):
        refused(EINVAL, P.ifq_f4_gated, d, *(good[:i] + [None] + good[i + 1:]))
    for i, p in ((0, ODD), (1, X[8:]), (2, X[2:]), (3, X[4:]), (4, ODD), (5, X[2:])):
        refused(EINVAL, P.ifq_f4_gated, d, *(good[:i] + [p] + good[i + 1:]))


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), EINVAL), (dict(n=0), EINVAL), (dict(rows=2 ** 31), EINVAL),
    (dict(n=2 ** 31), EINVAL), (dict(x_type=3), EINVAL), (dict(top=-1), EINVAL),
    (dict(top=65, ld_top=65), EINVAL), (dict(n=3), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(scale=2.0 ** 65), EINVAL),
    (dict(reserved=1), EINVAL), (dict(ld_x=99), EINVAL), (dict(ld_top=4), EINVAL),
    (dict(rows=2 ** 30), EUNSUP), (dict(n=2 ** 20 + 1, ld_x=2 ** 21), EUNSUP)])
def test_logprobs_refuses_descriptors(change, status):
    d = changed(P.logprobs_desc(8, 100, BF16, top=5), change)
    refused(status, P.ifq_logprobs, d, X, X, X, X, X, X)
    assert P.ifq_logprobs_workspace_bytes(d) == 0


def test_logprobs_refuses_pointers():
    d = P.logprobs_desc(8, 100, F32, top=5)
    good = [X] * 6
    for i in (0, 1, 2, 4, 5):                       # the entropy is optional
        refused(EINVAL, P.ifq_logprobs, d, *(good[:i] + [None] + good[i + 1:]))
    for i in range(6):
        refused(EINVAL, P.ifq_logprobs, d, *(good[:i] + [X[2:]] + good[i + 1:]))
    d = P.logprobs_desc(8, 100, F32)
    refused(EINVAL, P.ifq_logprobs, d, X, X, X, X, X, X)      # no top asked for


def test_calls_of_the_wrong_kind():
    d = P.f4_matmul_desc(1, 1, 16, BF16)
    with pytest.raises(ctypes.ArgumentError):
        P.ifq_f4_quantize(d, X, X, X, stream=0)
    with pytest.raises(ctypes.ArgumentError):
        P.ifq_logprobs(d, X, X, X, X, X, X, stream=0)
    with pytest.raises(ctypes.ArgumentError):
        P.ifq_f4_matmul(P.f4_weights_desc(1, 1, BF16), X, X, X, X, stream=0)
    with pytest.raises(AttributeError):
        P.ifq_f4_matmul(d, 4096, X, X, X, stream=0)


def test_empty_calls_do_nothing():
    for rows, k in ((0, 64), (4, 0)):
        P.ifq_f4_quantize(P.f4_weights_desc(rows, k, BF16), None, None, None, stream=0)
        P.ifq_f4_dequantize(P.f4_weights_desc(rows, k, BF16), None, None, None, stream=0)
    for m, n in ((0, 32), (8, 0)):
        d = P.f4_matmul_desc(m, n, 128, BF16)
        assert P.ifq_f4_matmul_workspace_bytes(d) == 0 and P.ifq_f4_matmul_kernel_name(d) == ""
        P.ifq_f4_matmul(d, None, None, None, None, stream=0)
        d.activation = P.IFQ_ACT_SILU
        assert P.ifq_f4_gated_workspace_bytes(d) == 0
        P.ifq_f4_gated(d, None, None, None, None, None, None, stream=0)
    d = P.logprobs_desc(0, 100, BF16, top=5)
    assert P.ifq_logprobs_workspace_bytes(d) == 0
    P.ifq_logprobs(d, None, None, None, None, None, None, stream=0)


class FakeCall:
    def __init__(self, need):
        self.need, self.seen = need, []

    def _any(self, d, *args):
        ws, nbytes, stream = args[-3:]
        self.seen.append((ws, nbytes, stream))
        return 0 if nbytes >= self.need else EBUF

    f4_matmul = f4_gated = logprobs = _any


@pytest.mark.parametrize("call,desc,n", [
    ("ifq_f4_matmul", P.f4_matmul_desc(1, 32, 128, BF16), 4),
    ("ifq_f4_gated", P.f4_matmul_desc(1, 32, 128, BF16, activation=1), 6),
    ("ifq_logprobs", P.logprobs_desc(8, 100, BF16, top=5), 6)])
def test_workspaces(monkeypatch, call, desc, n):
    from paper_1911_08076_amd import api
    fake = FakeCall(4096)
    monkeypatch.setattr(_ffi, "call", fake)
    monkeypatch.setattr(api, call + "_workspace_bytes", lambda d: 4096)
    monkeypatch.setattr(api, "_workspace", lambda nbytes, like, stream:
                        torch.zeros(nbytes, dtype=torch.uint8))
    getattr(P, call)(desc, *[X] * n, stream=7)
    (ws0, n0, s0), (ws1, n1, s1) = fake.seen
    assert ws0 is None and n0 == 0 and n1 == ws1.numel() == 4096 and s0 == s1 == 7
    fake.seen.clear()
    with pytest.raises(P.IfqError):                 # the caller's, too small: not retried
        getattr(P, call)(desc, *[X] * n, ws=torch.zeros(64, dtype=torch.uint8), stream=7)
    assert len(fake.seen) == 1
