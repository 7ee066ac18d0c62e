"""What follows the attention of a decoder that serves tokens, on the library's
operators: linear layers with weights in 4-bit floats with a scale per 32, a
gated feed-forward block of them, and a classifier that answers with log
probabilities of tokens.

Nothing here waits for the GPU, so calls on fixed inputs can be captured in a
graph. Weights are laid out once; all tensors of a layer are on its weights' GPU.
"""
import collections

import torch

from . import _ffi
from . import api as P
from .attention import _TYPES, _Workspace, _check_rows, _on

_HALVES = (torch.bfloat16, torch.float16)
ACTIVATIONS = {"silu": _ffi.IFQ_ACT_SILU, "gelu": _ffi.IFQ_ACT_GELU,
               "gelu_tanh": _ffi.IFQ_ACT_GELU_TANH}

# logprob and entropy [rows] float32, top_logprobs [rows][top] float32, top_tokens int32
# likewise; None where not asked for
TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprob entropy top_logprobs top_tokens")


def _output(x, n, dtype, out):
    """x's rows of n values of dtype (None: x's), or out once it is known to be that."""
    dtype = (x.dtype if out is None else out.dtype) if dtype is None else dtype
    if dtype not in _TYPES:
        raise ValueError("an output of %s" % dtype)
    if out is None:
        return torch.empty(x.shape[0], n, dtype=dtype, device=x.device)
    _check_rows(out, n, (dtype,), x.device)
    if out.shape[0] != x.shape[0]:
        raise ValueError("an output of %d rows for %d" % (out.shape[0], x.shape[0]))
    return out


def _overlap(a, b):
    """Dense tensors that share memory."""
    return (a.data_ptr() < b.data_ptr() + b.numel() * b.element_size() and
            b.data_ptr() < a.data_ptr() + a.numel() * a.element_size())


def _check_tokens(tokens, rows, device):
    if tokens is not None and (tokens.shape != (rows,) or tokens.dtype != torch.int32 or
                               not tokens.is_contiguous() or tokens.device != device):
        raise ValueError("tokens: dense int32 of shape (%d,) on %s expected, got %s of %s on %s" % (
            rows, device, tuple(tokens.shape), tokens.dtype, tokens.device))


class F4Weight:
    """Weights [out][in] as codes and scales (ifq_f4_quantize)."""

    def __init__(self, weight):
        _check_rows(weight, weight.shape[-1:].numel(), tuple(_TYPES), weight.device)
        dev = weight.device
        if dev.type != "cuda":
            raise ValueError("weights on a GPU expected, got them on %s" % dev)
        self.n, self.k = weight.shape
        if not self.n or not self.k:
            raise ValueError("weights of shape %s" % (tuple(weight.shape),))
        self.codes = torch.empty(self.n, -(-self.k // 32) * 16, dtype=torch.uint8, device=dev)
        self.scales = torch.empty(-(-self.k // 128), self.n, 4, dtype=torch.uint8, device=dev)
        with _on(dev):
            P.ifq_f4_quantize(P.f4_weights_desc(self.n, self.k, _TYPES[weight.dtype]), weight,
                              self.codes, self.scales)

    def values(self, dtype=torch.float32):
        """What they stand for, [out][in]."""
        if dtype not in _TYPES:
            raise ValueError("values of %s" % dtype)
        out = torch.empty(self.n, self.k, dtype=dtype, device=self.codes.device)
        with _on(self.codes.device):
            P.ifq_f4_dequantize(P.f4_weights_desc(self.n, self.k, _TYPES[dtype]), self.codes,
                                self.scales, out)
        return out


class F4Linear:
    """y = x w^T with w [out][in] in 4-bit floats and x in bfloat16 or float16. Calls share
    a workspace, so they follow one another: on one stream, or ordered by events."""

    def __init__(self, weight, workspace=None):
        self.weight = F4Weight(weight)
        self.workspace = _Workspace() if workspace is None else workspace

    def __call__(self, x, out=None, dtype=None):
        """x [m][in] -> [m][out] of dtype (None: out's, or x's). out must not overlap x."""
        w = self.weight
        dev = w.codes.device
        _check_rows(x, w.k, _HALVES, dev)
        y = _output(x, w.n, dtype, out)
        if out is not None and _overlap(x, out):
            raise ValueError("an output that overlaps the input")
        return self._product(x, y)

    def _product(self, x, out):
        w = self.weight
        dev = w.codes.device
        if x.shape[0]:
            with _on(dev):
                d = P.f4_matmul_desc(x.shape[0], w.n, w.k, _TYPES[x.dtype], _TYPES[out.dtype])
                P.ifq_f4_matmul(d, x, w.codes, w.scales, out,
                                ws=self.workspace.get(P.ifq_f4_matmul_workspace_bytes(d), dev))
        return out


class FeedForward:
    """down (act(x gate^T) * (x up^T))^T with gate and up [inner][hidden] and down
    [hidden][inner] in 4-bit floats: one call for the inner values, one for the way back.
    Calls share a workspace, as F4Linear's do."""

    def __init__(self, weight_gate, weight_up, weight_down, activation="silu"):
        if (weight_gate.shape != weight_up.shape or weight_down.shape != weight_gate.shape[::-1]):
            raise ValueError("weights of shapes %s, %s and %s do not fit" % tuple(
                tuple(w.shape) for w in (weight_gate, weight_up, weight_down)))
        if len({w.device for w in (weight_gate, weight_up, weight_down)}) > 1:
            raise ValueError("weights on one GPU expected, got them on %s, %s and %s" % (
                weight_gate.device, weight_up.device, weight_down.device))
        if activation not in ACTIVATIONS:
            raise ValueError("activation %r is none of %s" % (activation, ", ".join(ACTIVATIONS)))
        self.activation = ACTIVATIONS[activation]
        self.workspace = _Workspace()
        self.gate, self.up = F4Weight(weight_gate), F4Weight(weight_up)
        self.down = F4Linear(weight_down, self.workspace)

    def __call__(self, x, out=None):
        """x [m][hidden] (bfloat16 or float16) -> [m][hidden]; out may be x."""
        gate, up = self.gate, self.up
        dev = gate.codes.device
        _check_rows(x, gate.k, _HALVES, dev)
        out = _output(x, gate.k, x.dtype, out)
        if x.shape[0]:
            with _on(dev):
                inner = torch.empty(x.shape[0], gate.n, dtype=x.dtype, device=dev)
                d = P.f4_matmul_desc(x.shape[0], gate.n, gate.k, _TYPES[x.dtype],
                                     activation=self.activation)
                P.ifq_f4_gated(d, x, gate.codes, gate.scales, up.codes, up.scales, inner,
                               ws=self.workspace.get(P.ifq_f4_gated_workspace_bytes(d), dev))
                self.down._product(inner, out)
        return out


def token_logprobs(logits, tokens=None, top=0, scale=1.0, workspace=None):
    """Log probabilities of the tokens (int32 [rows], a negative one stands for none) under
    softmax(scale * logits), the entropy, and the `top` most probable tokens, of logits
    [rows][vocabulary] in bfloat16, float16 or float32 (ifq_logprobs)."""
    dev = logits.device
    _check_rows(logits, logits.shape[-1:].numel(), tuple(_TYPES), dev)
    if dev.type != "cuda":
        raise ValueError("logits on a GPU expected, got them on %s" % dev)
    rows, n = logits.shape
    _check_tokens(tokens, rows, dev)
    d = P.logprobs_desc(rows, n, _TYPES[logits.dtype], top, scale)
    with _on(dev):
        logprob = None if tokens is None else torch.empty(rows, device=dev)
        entropy = torch.empty(rows, device=dev)
        best = torch.empty(rows, top, device=dev) if top > 0 else None
        at = torch.empty(rows, top, dtype=torch.int32, device=dev) if top > 0 else None
        need = P.ifq_logprobs_workspace_bytes(d)
        P.ifq_logprobs(d, logits, tokens, logprob, entropy, best, at,
                       ws=None if workspace is None else workspace.get(need, dev))
    return TokenLogprobs(logprob, entropy, best, at)


class Classifier:
    """Logits of a vocabulary, weights [vocabulary][hidden] in 4-bit floats, kept in float32,
    and what is asked of their distribution. Calls share a workspace, as F4Linear's do."""

    def __init__(self, weight):
        self.workspace = _Workspace()
        self.linear = F4Linear(weight, self.workspace)

    def __call__(self, x, tokens=None, top=1, scale=1.0):
        """x [m][hidden] -> TokenLogprobs of its rows (token_logprobs)."""
        weight = self.linear.weight
        _check_rows(x, weight.k, _HALVES, weight.codes.device)
        _check_tokens(tokens, x.shape[0], x.device)
        logits = self.linear(x, dtype=torch.float32)
        return token_logprobs(logits, tokens, top, scale, self.workspace)
