"""One attention layer of a decoder that serves tokens, on the library's
operators: the inputs and weights of its products in 8-bit floats, the keys and
values of past tokens in a paged cache of 4-bit codes.

A step takes the new tokens of a batch of sequences, one each (decoding) or many
(prompts; both in one step give the same, but take longer than a step each), and
makes six calls on the current stream: quantize, product to
queries, keys and values, append (with the rotation), attention, quantize,
product. Nothing in it waits for the GPU or reads the sequences' lengths on the
host, so a step on fixed inputs can be captured in a graph.
"""
import contextlib

import torch

from . import _ffi
from . import api as P

_TYPES = {torch.bfloat16: _ffi.IFQ_TYPE_BF16, torch.float16: _ffi.IFQ_TYPE_F16,
          torch.float32: _ffi.IFQ_TYPE_F32}


def rotation_tables(positions, rot_dim, base=10000.0, device="cuda"):
    """Cosines and sines [positions][rot_dim/2] of position * base^(-2i/rot_dim)."""
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().to(device), angle.sin().float().to(device)


class _Workspace:
    """One zero-filled device workspace for calls that follow one another, made
    larger when a call needs more. Smaller ones are kept, since a captured graph
    may hold them: sizes double, so together they are below the largest. A call
    under capture that needs a larger one gets one of the graph's own."""

    def __init__(self):
        self._all = []

    def get(self, nbytes, device):
        if not nbytes:
            return None
        if torch.cuda.is_current_stream_capturing():
            # filled at every replay, not now: for the graph alone
            if not self._all or self._all[-1].numel() < nbytes:
                return torch.zeros(nbytes, dtype=torch.uint8, device=device)
        if not self._all or self._all[-1].numel() < nbytes:
            most = 2 * self._all[-1].numel() if self._all else 0
            self._all.append(torch.zeros(max(nbytes, most), dtype=torch.uint8, device=device))
        return self._all[-1]


def _check_rows(x, columns, types, device):
    if x.dim() != 2 or x.shape[1] != columns or not x.is_contiguous() or x.dtype not in types:
        raise ValueError("dense rows of %d values of %s expected, got %s of %s" % (
            columns, " or ".join(str(t) for t in types), tuple(x.shape), x.dtype))
    if x.device != device:
        raise ValueError("rows on %s expected, got them on %s" % (device, x.device))


def _check_out(out, x, columns):
    _check_rows(out, columns, (x.dtype,), x.device)
    if out.shape[0] != x.shape[0]:
        raise ValueError("an output of %d rows for %d" % (out.shape[0], x.shape[0]))


def _on(device):
    """The launches and temporaries of a layer go to its own GPU's current stream,
    also where another GPU is torch's current one."""
    if device.index == torch.cuda.current_device():
        return contextlib.nullcontext()
    return torch.cuda.device(device)


class F8Linear:
    """Weights [out][in] in 8-bit floats with a scale per 128 x 128, and y = x w^T
    for x quantized with a scale per row and 128 columns. Calls share a workspace,
    so they follow one another: on one stream, or ordered by events. All tensors
    are on the weights' GPU."""

    def __init__(self, weight, workspace=None):
        _check_rows(weight, weight.shape[-1], tuple(_TYPES), weight.device)
        dev = weight.device
        if dev.type != "cuda":
            raise ValueError("weights on a GPU expected, got them on %s" % dev)
        n, k = weight.shape
        self.n, self.k, self.ld = n, k, -(-k // 16) * 16
        self.workspace = _Workspace() if workspace is None else workspace
        self.codes = torch.empty(n, self.ld, dtype=torch.uint8, device=dev)
        self.scales = torch.empty(-(-k // 128), -(-n // 128), device=dev)
        with _on(dev):
            P.ifq_f8_quantize(P.f8_quant_desc(n, k, _TYPES[weight.dtype], block_rows=128),
                              weight, self.codes, self.scales)

    def __call__(self, x, out=None):
        """x [m][k] -> [m][n] of x's type."""
        dev = self.codes.device
        _check_rows(x, self.k, tuple(_TYPES), dev)
        m = x.shape[0]
        if out is None:
            out = torch.empty(m, self.n, dtype=x.dtype, device=dev)
        else:
            _check_out(out, x, self.n)
        if m == 0:
            return out
        with _on(dev):
            codes = torch.empty(m, self.ld, dtype=torch.uint8, device=dev)
            scales = torch.empty(self.scales.shape[0], m, device=dev)
            P.ifq_f8_quantize(P.f8_quant_desc(m, self.k, _TYPES[x.dtype]), x, codes, scales)
            mm = P.f8_matmul_desc(m, self.n, self.ld, _TYPES[x.dtype])
            P.ifq_f8_matmul(mm, codes, scales, self.codes, self.scales, out,
                            ws=self.workspace.get(P.ifq_f8_matmul_workspace_bytes(mm), dev))
        return out


class AttentionLayer:
    """weight_qkv [(heads + 2 kv_heads) * head_dim][hidden] (queries, keys, values),
    weight_out [hidden][heads * head_dim]; num_pages pages of page_tokens tokens,
    of which a sequence may have max_pages. rot_dim None: the whole head. Steps
    share the cache and a workspace, so they follow one another: on one stream,
    or ordered by events. All tensors are on the weights' GPU."""

    def __init__(self, weight_qkv, weight_out, heads, kv_heads, head_dim, num_pages, max_pages,
                 page_tokens=64, rot_dim=None, rot_base=10000.0, window=0, sinks=0):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.page_tokens, self.num_pages, self.max_pages = page_tokens, num_pages, max_pages
        self.window, self.sinks = window, sinks
        self.rot_dim = head_dim if rot_dim is None else rot_dim
        if weight_qkv.shape[0] != (heads + 2 * kv_heads) * head_dim or (
                weight_out.shape != (weight_qkv.shape[1], heads * head_dim)):
            raise ValueError("weights of shapes %s and %s do not fit %d and %d heads of %d" % (
                tuple(weight_qkv.shape), tuple(weight_out.shape), heads, kv_heads, head_dim))
        dev = weight_qkv.device
        if weight_out.device != dev:
            raise ValueError("weights on one GPU expected, got them on %s and %s" % (
                dev, weight_out.device))
        self.workspace = _Workspace()
        self.qkv = F8Linear(weight_qkv, self.workspace)
        self.out = F8Linear(weight_out, self.workspace)
        self.cosines, self.sines = (
            rotation_tables(max_pages * page_tokens, self.rot_dim, rot_base, dev)
            if self.rot_dim else (None, None))
        nbytes = P.ifq_kv_cache_bytes(self._desc(0, 0, 0, 0, torch.bfloat16))
        if not nbytes:
            raise ValueError("no cache of %d pages of %d tokens for heads of %d" % (
                num_pages, page_tokens, head_dim))
        self.cache = torch.zeros(nbytes, dtype=torch.uint8, device=dev)

    def _desc(self, batch, tokens, max_q, max_kv, dtype, q_stride=None):
        row = (self.heads + 2 * self.kv_heads) * self.head_dim
        return P.kv_desc(batch, tokens, max_q, max_kv, self.heads, self.kv_heads, self.head_dim,
                         self.page_tokens, self.num_pages, self.max_pages, _TYPES[dtype],
                         scale=self.head_dim ** -0.5, window=self.window, sinks=self.sinks,
                         rot_dim=self.rot_dim, rot_len=self.max_pages * self.page_tokens,
                         q_stride=q_stride, k_stride=row, v_stride=row)

    def __call__(self, x, offsets, lengths, pages, max_q, max_kv=None, out=None):
        """x [tokens][hidden] (bfloat16 or float16), the new tokens of the batch one
        sequence after another; offsets int32 [batch + 1], lengths int32 [batch]
        (with the new tokens) and pages int32 [batch][max_pages] as for
        ifq_kv_append; max_q: the most new tokens of a sequence; max_kv: about how
        long the longest sequence is, for the split of the work (None: as long as
        the page table allows). Returns [tokens][hidden]; a row of no sequence holds
        anything."""
        dev = self.cache.device
        _check_rows(x, self.qkv.k, (torch.bfloat16, torch.float16), dev)
        tokens, batch = x.shape[0], lengths.numel()
        for name, t, shape in (("offsets", offsets, (batch + 1,)), ("lengths", lengths, (batch,)),
                               ("pages", pages, (batch, self.max_pages))):
            if t.shape != shape or t.dtype != torch.int32 or not t.is_contiguous():
                raise ValueError("%s: dense int32 of shape %s expected, got %s of %s" % (
                    name, shape, tuple(t.shape), t.dtype))
            if t.device != dev:
                raise ValueError("%s: expected on %s, got on %s" % (name, dev, t.device))
        if out is not None:
            _check_out(out, x, self.out.n)
        if max_kv is None:
            max_kv = self.max_pages * self.page_tokens
        with _on(dev):
            rows = self.qkv(x)
            q = torch.empty(tokens, self.heads * self.head_dim, dtype=x.dtype, device=dev)
            mixed = torch.empty_like(q)
            if tokens:
                k = rows[:, self.heads * self.head_dim:]
                v = rows[:, (self.heads + self.kv_heads) * self.head_dim:]
                # the queries lie in the product's rows, and dense once rotated
                P.ifq_kv_append(self._desc(batch, tokens, max_q, max_kv, x.dtype, rows.shape[1]),
                                rows, k, v, self.cosines, self.sines, offsets, lengths, pages,
                                self.cache, q)
                d = self._desc(batch, tokens, max_q, max_kv, x.dtype)
                P.ifq_kv_attention(d, q, offsets, lengths, pages, self.cache, mixed,
                                   ws=self.workspace.get(P.ifq_kv_attention_workspace_bytes(d),
                                                         dev))
            return self.out(mixed, out=out)
