"""Host side of the operators for serving language models, on the CPU: every
refusal comes before a launch, empty calls launch nothing, and workspaces are
asked for and passed on. Device pointers here are host addresses that no call
gets far enough to use."""
import ctypes

import numpy as np
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


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), EINVAL), (dict(k=-1), EINVAL), (dict(rows=2 ** 31), EINVAL),
    (dict(x_type=3), EINVAL), (dict(x_type=-1), EINVAL), (dict(block_rows=0), EINVAL),
    (dict(block_rows=64), EINVAL), (dict(ld_x=63), EINVAL), (dict(ld_codes=63), EINVAL),
    (dict(ld_codes=72), EUNSUP), (dict(ld_x=2 ** 41), EINVAL)])
def test_quantize_refuses_descriptors(change, status):
    d = P.f8_quant_desc(4, 64, BF16)
    for k, v in change.items():
        setattr(d, k, v)
    refused(status, P.ifq_f8_quantize, d, X, X, X)


def test_launches_of_too_many_workgroups_are_refused():
    refused(EUNSUP, P.ifq_f8_quantize, P.f8_quant_desc(2 ** 30, 2 ** 14, BF16), X, X, X)
    d = kv(batch=65535, total_q=2 ** 30, max_q=2 ** 20, num_pages=1)
    refused(EUNSUP, P.ifq_kv_append, d, X, X, X, None, None, X, X, X, X, X)
    refused(EUNSUP, P.ifq_kv_read, d, X, X, X, X, X, X)
    need = P.ifq_kv_attention_workspace_bytes(d)
    assert need == 0
    refused(EUNSUP, P.ifq_kv_attention, d, X, X, X, X, X, X)


def test_quantize_refuses_pointers():
    d = P.f8_quant_desc(4, 64, BF16)
    for args in ((None, X, X), (X, None, X), (X, X, None), (ODD, X, X), (X, X[4:], X),
                 (X, X, ODD)):
        refused(EINVAL, P.ifq_f8_quantize, d, *args)
    refused(EINVAL, P.ifq_f8_quantize, P.f8_quant_desc(4, 64, F32), X[2:], X, X)


@pytest.mark.parametrize("change,status", [
    (dict(m=-1), EINVAL), (dict(n=-1), EINVAL), (dict(k=0), EINVAL), (dict(n=2 ** 31), EINVAL),
    (dict(k=120), EUNSUP), (dict(ld_a=120), EINVAL), (dict(ld_a=136), EUNSUP),
    (dict(ld_w=127), EINVAL), (dict(ld_w=130), EUNSUP), (dict(ld_y=31), EINVAL),
    (dict(ld_a=2 ** 25 + 16), EUNSUP), (dict(ld_w=2 ** 26), EUNSUP),
    (dict(m=1, n=2 ** 30, ld_y=2 ** 30), EUNSUP),
    (dict(y_type=7), EINVAL), (dict(m=2 ** 30, n=2 ** 30, ld_y=2 ** 30), EUNSUP)])
def test_product_refuses_descriptors(change, status):
    d = P.f8_matmul_desc(8, 32, 128, BF16)
    for k, v in change.items():
        setattr(d, k, v)
    refused(status, P.ifq_f8_matmul, d, X, X, X, X, X)
    assert P.ifq_f8_matmul_workspace_bytes(d) == 0


def test_product_refuses_pointers():
    d = P.f8_matmul_desc(8, 32, 128, BF16)
    good = [X, X, X, X, X]
    for i in range(5):
        refused(EINVAL, P.ifq_f8_matmul, d, *(good[:i] + [None] + good[i + 1:]))
    for i, p in ((0, X[8:]), (2, X[4:]), (1, ODD), (3, X[2:]), (4, ODD)):
        refused(EINVAL, P.ifq_f8_matmul, d, *(good[:i] + [p] + good[i + 1:]))


def kv(**change):
    d = P.kv_desc(2, 8, 4, 100, 8, 2, 128, 64, 6, 3, BF16)
    for k, v in change.items():
        setattr(d, k, v)
    return d


BAD_KV = [
    (dict(batch=-1), EINVAL), (dict(total_q=-1), EINVAL), (dict(max_q=9), EINVAL),
    (dict(max_kv=-1), EINVAL), (dict(heads=7), EINVAL), (dict(heads=0), EINVAL),
    (dict(kv_heads=0), EINVAL), (dict(type=F32), EINVAL), (dict(num_pages=0), EINVAL),
    (dict(max_pages=0), EINVAL), (dict(causal=2), EINVAL), (dict(rot_adjacent=-1), EINVAL),
    (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(window=4, causal=0), EINVAL),
    (dict(rot_dim=130), EINVAL), (dict(rot_dim=-16), EINVAL), (dict(rot_len=-1), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(page_tokens=48), EUNSUP), (dict(page_tokens=16), EUNSUP),
    (dict(page_tokens=8192), EUNSUP), (dict(head_dim=96), EUNSUP), (dict(rot_dim=8), EUNSUP),
    (dict(max_pages=2 ** 30), EUNSUP), (dict(batch=65536), EUNSUP)]


@pytest.mark.parametrize("change,status", BAD_KV)
def test_kv_refuses_descriptors(change, status):
    d = kv(**change)
    refused(status, P.ifq_kv_append, d, X, X, X, None, None, X, X, X, X, X)
    refused(status, P.ifq_kv_read, d, X, X, X, X, X, X)
    refused(status, P.ifq_kv_attention, d, X, X, X, X, X, X)
    assert P.ifq_kv_cache_bytes(d) == 0
    assert P.ifq_kv_attention_workspace_bytes(d) == 0


@pytest.mark.parametrize("name,value,status", [
    ("q_stride", 1016, EINVAL), ("k_stride", 248, EINVAL), ("v_stride", 255, EINVAL),
    ("q_stride", 1028, EUNSUP), ("k_stride", 260, EUNSUP), ("v_stride", 257, EUNSUP)])
def test_append_refuses_strides(name, value, status):
    refused(status, P.ifq_kv_append, kv(**{name: value}), X, X, X, None, None, X, X, X, X, X)


def test_attention_refuses_strides():
    for name in ("q_stride", "o_stride"):
        refused(EINVAL, P.ifq_kv_attention, kv(**{name: 1023}), X, X, X, X, X, X)
        refused(EUNSUP, P.ifq_kv_attention, kv(**{name: 1025}), X, X, X, X, X, X)


def test_kv_refuses_pointers():
    good = [X] * 10
    good[3] = good[4] = None                        # no rotation
    for i in (1, 2, 5, 6, 7, 8):
        refused(EINVAL, P.ifq_kv_append, kv(), *(good[:i] + [None] + good[i + 1:]))
    for i in (0, 9):                                # q without q_out and the other way round
        refused(EINVAL, P.ifq_kv_append, kv(), *(good[:i] + [None] + good[i + 1:]))
    for i, p in ((0, X[8:]), (1, X[8:]), (2, X[2:]), (5, ODD), (6, ODD), (7, X[2:]),
                 (8, X[8:]), (9, X[4:])):
        refused(EINVAL, P.ifq_kv_append, kv(), *(good[:i] + [p] + good[i + 1:]))
    refused(EINVAL, P.ifq_kv_append, kv(), X, X, X, X, X, *good[5:])       # rot_dim 0
    turned = kv(rot_dim=64, rot_len=100)
    refused(EINVAL, P.ifq_kv_append, turned, *good)
    refused(EINVAL, P.ifq_kv_append, turned, X, X, X, X, X[4:], *good[5:])
    six = [X] * 6
    for i in range(6):
        refused(EINVAL, P.ifq_kv_read, kv(), *(six[:i] + [None] + six[i + 1:]))
        refused(EINVAL, P.ifq_kv_attention, kv(), *(six[:i] + [None] + six[i + 1:]))
    for i, p in ((0, ODD), (1, ODD), (2, ODD), (3, X[8:]), (4, X[8:]), (5, X[8:])):
        refused(EINVAL, P.ifq_kv_read, kv(), *(six[:i] + [p] + six[i + 1:]))
    for i, p in ((0, X[8:]), (1, ODD), (2, ODD), (3, ODD), (4, X[8:]), (5, X[8:])):
        refused(EINVAL, P.ifq_kv_attention, kv(), *(six[:i] + [p] + six[i + 1:]))


def test_calls_of_the_wrong_kind():
    with pytest.raises(ctypes.ArgumentError):
        P.ifq_f8_quantize(kv(), X, X, X, stream=0)
    with pytest.raises(ctypes.ArgumentError):
        P.ifq_kv_read(P.f8_quant_desc(1, 1, BF16), X, X, X, X, X, X, stream=0)
    with pytest.raises(AttributeError):
        P.ifq_f8_matmul(P.f8_matmul_desc(1, 1, 16, BF16), 4096, X, X, X, X, stream=0)


def test_empty_calls_do_nothing():
    P.ifq_f8_quantize(P.f8_quant_desc(0, 64, BF16), None, None, None, stream=0)
    P.ifq_f8_quantize(P.f8_quant_desc(4, 0, BF16), None, None, None, stream=0)
    for m, n in ((0, 32), (8, 0)):
        d = P.f8_matmul_desc(m, n, 128, BF16)
        assert P.ifq_f8_matmul_workspace_bytes(d) == 0
        P.ifq_f8_matmul(d, None, None, None, None, None, stream=0)
    for change in (dict(batch=0), dict(total_q=0, max_q=0), dict(max_q=0)):
        d = kv(**change)
        assert P.ifq_kv_attention_workspace_bytes(d) == 0
        P.ifq_kv_append(d, *[None] * 10, stream=0)
        P.ifq_kv_read(d, *[None] * 6, stream=0)
        P.ifq_kv_attention(d, *[None] * 6, stream=0)


def test_cache_bytes():
    # codes of a key and a value, 4 bits each, and a word for either
    assert P.ifq_kv_cache_bytes(kv()) == 6 * 2 * 64 * (128 + 8)
    assert P.ifq_kv_cache_bytes(kv(num_pages=2 ** 20)) == 2 ** 20 * 2 * 64 * 136


class FakeCall:
    def __init__(self, need):
        self.need, self.seen = need, []

    def _any(self, d, *args):
        ws, nbytes, stream = args[-3:]
        self.seen.append((ws, nbytes, stream))
        return 0 if nbytes >= self.need else EBUF

    f8_matmul = kv_attention = _any


@pytest.mark.parametrize("call,desc,n", [
    ("ifq_f8_matmul", P.f8_matmul_desc(1, 32, 128, BF16), 5), ("ifq_kv_attention", kv(), 6)])
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
    fake.seen.clear()
    ws = torch.zeros(1024, dtype=torch.int32)
    getattr(P, call)(desc, *[X] * n, ws=ws, stream=7)
    assert [(a is ws, b) for a, b, _ in fake.seen] == [(True, 4096)]
