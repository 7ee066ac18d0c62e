"""Python binding of the C ABI: one function per entry point, same names.

Only argument marshalling happens here (descriptors, pointers, the stream
handle; the launching calls go through the C extension _ifqcall, the others
through ctypes). Every step of the quantized substructure runs in libifq.so: host-side
packing and folding in its C++ code, everything else in its HIP kernels.
Device tensors are torch tensors; host arrays are NumPy arrays.
"""
import ctypes

import numpy as np

from . import _ffi
from ._ffi import (ConvDesc, FoldParams, JoinParams, Join, PoolDesc, Stack,
                   F8QuantDesc, F8MatmulDesc, KvDesc, F4WeightsDesc, F4MatmulDesc, LogprobsDesc,
                   IFQ_OK, IFQ_JOIN_NONE, IFQ_MAX_THRESHOLDS)


class IfqError(RuntimeError):
    def __init__(self, status, func, message):
        super().__init__("%s failed with status %d: %s" % (func, status, message))
        self.status = status


def _lib():
    return _ffi.load()


def _check(status, func):
    if status != IFQ_OK:
        msg = _lib().ifq_last_error().decode(errors="replace")
        raise IfqError(status, func, msg)


_ptr = _ffi.address


def _struct(v, cls):
    """Address of the ctypes structure v, which must be a cls."""
    if not isinstance(v, cls):
        raise ctypes.ArgumentError("expected %s, got %s" % (cls.__name__, type(v).__name__))
    return ctypes.addressof(v)


def _stream(stream):
    if stream is None:
        import torch
        dev = torch.cuda.current_device()      # initialises torch's GPU state if need be
        return _current_raw_stream(dev)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _current_raw_stream(dev):
    """torch's current stream on dev as a handle: torch's own raw query where
    it has one (no Stream object is made), resolved on first use."""
    global _current_raw_stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _current_raw_stream = raw or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _current_raw_stream(dev)


def _f64(a):
    return None if a is None else np.ascontiguousarray(a, dtype=np.float64)


def conv_desc(n, h, w, c_in, c_out, k, stride, pad, in_bits, out_bits,
              in_layout=_ffi.IFQ_LAYOUT_I8_NHWC, out_layout=None, kw=None):
    if out_layout is None:
        out_layout = (_ffi.IFQ_LAYOUT_I32_NHWC if out_bits == 0
                      else _ffi.IFQ_LAYOUT_I8_NHWC)
    return ConvDesc(n, h, w, c_in, c_out, k, k if kw is None else kw, stride,
                    pad, in_bits, out_bits, in_layout, out_layout)


def pool_desc(n, h, w, c, k, stride, mode, bits=2,
              layout=_ffi.IFQ_LAYOUT_I8_NHWC):
    return PoolDesc(n, h, w, c, k, stride, mode, bits, layout)


def ifq_version():
    return _lib().ifq_version().decode()


def ifq_last_error():
    return _lib().ifq_last_error().decode(errors="replace")


def ifq_tensor_bytes(n, h, w, c, layout):
    return int(_lib().ifq_tensor_bytes(n, h, w, c, layout))


def ifq_conv_output_dims(desc):
    ho, wo = ctypes.c_int32(), ctypes.c_int32()
    _check(_lib().ifq_conv_output_dims(ctypes.byref(desc), ctypes.byref(ho),
                                       ctypes.byref(wo)), "ifq_conv_output_dims")
    return ho.value, wo.value


def ifq_packed_weight_bytes(desc):
    return int(_lib().ifq_packed_weight_bytes(ctypes.byref(desc)))


def ifq_pack_weights(desc, w_oihw, dst=None):
    """Pack +-1 OIHW int8 weights into the device blob (host uint8 array)."""
    w = np.ascontiguousarray(w_oihw, dtype=np.int8)
    nbytes = ifq_packed_weight_bytes(desc)
    if dst is None:
        dst = np.zeros(max(nbytes, 1), dtype=np.uint8)
    _check(_lib().ifq_pack_weights(ctypes.byref(desc), _ptr(w), _ptr(dst),
                                   dst.nbytes), "ifq_pack_weights")
    return dst


def ifq_fold_thresholds(c_out, in_bits, out_bits, k, alpha, beta_in, q_thr,
                        bias=None, mean=None, var=None, gamma=None,
                        bn_beta=None, eps=0.0):
    """Integer threshold records [c_out][2^out_bits] = {s, T_1..T_{2^k-1}}."""
    arrs = [_f64(a) for a in (alpha, bias, mean, var, gamma, bn_beta, q_thr)]
    p = FoldParams(c_out, in_bits, out_bits, 0, int(k), _ptr(arrs[0]),
                   float(beta_in), _ptr(arrs[1]), _ptr(arrs[2]), _ptr(arrs[3]),
                   _ptr(arrs[4]), _ptr(arrs[5]), float(eps), _ptr(arrs[6]))
    out = np.zeros((c_out, 1 << out_bits), dtype=np.int32)
    _check(_lib().ifq_fold_thresholds(ctypes.byref(p), _ptr(out)),
           "ifq_fold_thresholds")
    return out


# One compact threshold record (ifq_thr_compact): base', offset', s, cstar.
THR_COMPACT = np.dtype([("base", "<f8"), ("offset", "<f8"), ("s", "<i4"), ("cstar", "<i4")])


def ifq_fold_thresholds_compact(c_out, in_bits, out_bits, k, alpha, beta_in, base, offset,
                                bias=None, mean=None, var=None, gamma=None,
                                bn_beta=None, eps=0.0):
    """Compact records (THR_COMPACT, c_out of them) of a uniform quantizer
    q_i = i*base + offset."""
    arrs = [_f64(a) for a in (alpha, bias, mean, var, gamma, bn_beta)]
    p = FoldParams(c_out, in_bits, out_bits, 0, int(k), _ptr(arrs[0]),
                   float(beta_in), _ptr(arrs[1]), _ptr(arrs[2]), _ptr(arrs[3]),
                   _ptr(arrs[4]), _ptr(arrs[5]), float(eps), None)
    out = np.zeros(c_out, dtype=THR_COMPACT)
    _check(_lib().ifq_fold_thresholds_compact(ctypes.byref(p), float(base), float(offset),
                                              _ptr(out)), "ifq_fold_thresholds_compact")
    return out


def ifq_expand_thresholds(recs, c_out, in_bits, k, out_bits, thr, stream=None):
    """Device: compact records -> int32 records [c_out][2^out_bits] in thr."""
    _check(_lib().ifq_expand_thresholds(_ptr(recs), int(c_out), int(in_bits), int(k),
                                        int(out_bits), _ptr(thr), _stream(stream)),
           "ifq_expand_thresholds")


def _join_params(kind, main, beta_x, down=None):
    m = {k: _f64(main.get(k)) for k in ("alpha", "bias", "mean", "var", "gamma",
                                          "bn_beta")}
    d = {k: None for k in m}
    eps_d = 0.0
    if kind == _ffi.IFQ_JOIN_CONV:
        d = {k: _f64(down.get(k)) for k in m}
        eps_d = float(down["eps"])
    c_out = m["alpha"].shape[0]
    p = JoinParams(c_out, kind, _ptr(m["alpha"]), float(main["beta_in"]),
                   _ptr(m["bias"]), _ptr(m["mean"]), _ptr(m["var"]),
                   _ptr(m["gamma"]), _ptr(m["bn_beta"]), float(main["eps"]),
                   float(beta_x), _ptr(d["alpha"]), _ptr(d["bias"]),
                   _ptr(d["mean"]), _ptr(d["var"]), _ptr(d["gamma"]),
                   _ptr(d["bn_beta"]), eps_d)
    return p, c_out, (m, d)


def ifq_fold_join(kind, main, beta_x, down=None):
    """Join coefficients [c_out][3] = {p, q, cc}.

    main / down: dicts with alpha, beta_in, bias, mean, var, gamma, bn_beta,
    eps (down is used for IFQ_JOIN_CONV only).
    """
    p, c_out, keep = _join_params(kind, main, beta_x, down)
    out = np.zeros((c_out, 3), dtype=np.float64)
    _check(_lib().ifq_fold_join(ctypes.byref(p), _ptr(out)), "ifq_fold_join")
    return out


def ifq_fold_join_table(main, beta_x, in_bits, k, out_bits, q_thr, x_bits=2):
    """Integer records of an identity join: int32 [c_out][2^x_bits][2^out_bits]
    = {s, T_1 .. T_{2^out_bits - 1}} for every shortcut code x."""
    p, c_out, keep = _join_params(_ffi.IFQ_JOIN_IDENTITY, main, beta_x)
    q = _f64(q_thr)
    out = np.zeros((c_out, 1 << x_bits, 1 << out_bits), dtype=np.int32)
    _check(_lib().ifq_fold_join_table(ctypes.byref(p), int(in_bits), int(k),
                                      int(x_bits), int(out_bits), _ptr(q),
                                      _ptr(out)), "ifq_fold_join_table")
    return out


def make_join(kind, layout, shortcut, coef, q_thr, table=None, down_w=None,
              down=None):
    """ifq_join; down_w (packed 1x1 weights) and down (its ConvDesc) are for
    IFQ_JOIN_CONV_FUSED, whose coef comes from ifq_fold_join(IFQ_JOIN_CONV)."""
    j = Join()
    j.kind = kind
    j.layout = layout
    j.shortcut = _ptr(shortcut)
    j.coef = _ptr(coef)
    j.table = _ptr(table)
    q = list(np.asarray(q_thr, dtype=np.float64))
    j.n_q = len(q)
    for i, v in enumerate(q[:IFQ_MAX_THRESHOLDS]):
        j.q_thr[i] = float(v)
    j.down_w = _ptr(down_w)
    if down is not None:
        j.down = down
    return j


def ifq_conv_kernel_name(desc, join=None):
    return _lib().ifq_conv_kernel_name(
        ctypes.byref(desc), ctypes.byref(join) if join is not None else None).decode()


def ifq_conv_workspace_bytes(desc):
    return int(_lib().ifq_conv_workspace_bytes(ctypes.byref(desc)))


def ifq_conv_forward(desc, x, w_packed, thr, y, join=None, acc_dump=None,
                     ws=None, stream=None):
    """ws None: a zero-filled device workspace of ifq_conv_workspace_bytes
    bytes is made for this call where the layer needs one (a K split)."""
    d = _struct(desc, ConvDesc)
    j = None if join is None else _struct(join, Join)
    st = _stream(stream)
    rc = _ffi.call.conv_forward(d, x, w_packed, thr, j, y, acc_dump, ws, _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        import torch
        ws = torch.zeros(ifq_conv_workspace_bytes(desc), dtype=torch.uint8, device=y.device)
        rc = _ffi.call.conv_forward(d, x, w_packed, thr, j, y, acc_dump, ws, _nbytes(ws), st)
    if rc:
        _check(rc, "ifq_conv_forward")


def _nbytes(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


def ifq_pack_weights_fp4(desc, w_oihw):
    """The fp4 weight blob (uint8) of OIHW +-1 weights."""
    w = np.ascontiguousarray(w_oihw, dtype=np.int8)
    n = int(_lib().ifq_packed_weight_bytes_fp4(ctypes.byref(desc)))
    if n == 0:
        raise IfqError(-1, "ifq_packed_weight_bytes_fp4", "no fp4 layout for this layer")
    out = np.zeros(n, dtype=np.uint8)
    _check(_lib().ifq_pack_weights_fp4(ctypes.byref(desc), _ptr(w), _ptr(out), n),
           "ifq_pack_weights_fp4")
    return out


def ifq_conv_fp4_kernel_name(desc, join=None):
    return _lib().ifq_conv_fp4_kernel_name(
        ctypes.byref(desc), ctypes.byref(join) if join is not None else None).decode()


def ifq_conv_forward_fp4(desc, x, w_fp4, thr, y, join=None, stream=None):
    _check(_ffi.call.conv_forward_fp4(
        _struct(desc, ConvDesc), x, w_fp4, thr,
        None if join is None else _struct(join, Join), y, _stream(stream)),
        "ifq_conv_forward_fp4")


def ifq_conv_pool_forward(desc, pool, x, w_packed, thr, y, stream=None):
    _check(_ffi.call.conv_pool_forward(
        _struct(desc, ConvDesc), _struct(pool, PoolDesc), x, w_packed, thr, y,
        _stream(stream)), "ifq_conv_pool_forward")


def ifq_conv_pool_forward_fp4(desc, pool, x, w_fp4, thr, y, stream=None):
    _check(_ffi.call.conv_pool_forward_fp4(
        _struct(desc, ConvDesc), _struct(pool, PoolDesc), x, w_fp4, thr, y,
        _stream(stream)), "ifq_conv_pool_forward_fp4")


def ifq_conv_pool_fp4_kernel_name(desc, pool):
    return _lib().ifq_conv_pool_fp4_kernel_name(ctypes.byref(desc), ctypes.byref(pool)).decode()


def ifq_conv_pool_kernel_name(desc, pool):
    return _lib().ifq_conv_pool_kernel_name(ctypes.byref(desc), ctypes.byref(pool)).decode()


def ifq_maxpool_codes(desc, x, y, stream=None):
    _check(_ffi.call.maxpool_codes(_struct(desc, PoolDesc), x, y, _stream(stream)),
           "ifq_maxpool_codes")


def ifq_convert_codes(n, h, w, c, src_layout, dst_layout, src, dst, stream=None):
    _check(_ffi.call.convert_codes(int(n), int(h), int(w), int(c), src_layout, dst_layout,
                                   src, dst, _stream(stream)), "ifq_convert_codes")


def ifq_stack_workspace_bytes(stack):
    return int(_lib().ifq_stack_workspace_bytes(ctypes.byref(stack)))


def ifq_stack_slot_info(stack, slot):
    off, nb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib().ifq_stack_slot_info(ctypes.byref(stack), int(slot),
                                      ctypes.byref(off), ctypes.byref(nb)),
           "ifq_stack_slot_info")
    return off.value, nb.value


def ifq_run_stack(stack, x, y, ws, stream=None):
    _check(_ffi.call.run_stack(_struct(stack, Stack), x, y, ws, _nbytes(ws),
                               _stream(stream)), "ifq_run_stack")


def ifq_run_stack_static(stack, x, y, stream=None):
    _check(_ffi.call.run_stack_static(_struct(stack, Stack), x, y, _stream(stream)),
           "ifq_run_stack_static")


def ifq_static_workspace_bytes():
    return int(_lib().ifq_static_workspace_bytes())


def ifq_conv_variant_count():
    return int(_lib().ifq_conv_variant_count())


def ifq_conv_variant_fp4(variant):
    """1: the variant runs on the fp4 scaled MFMA (takes the fp4 weight
    blob); 0: int8 MFMA; -1: no such variant."""
    return int(_lib().ifq_conv_variant_fp4(int(variant)))


def kernel_is_fp4(name):
    """Whether a kernel name (as ifq_conv_kernel_name returns it) is an fp4
    instance: the fp4 flag true (the windowed kernel's last template
    argument, conv_w2's ninth, conv_wp's fifth, conv_wv's and conv_wvh's second)."""
    if name.startswith("conv_halo<"):
        return name.endswith(", true>")
    for kern, pos in (("conv_w2<", 8), ("conv_wp<", 4), ("conv_wv<", 1), ("conv_wvh<", 1)):
        if name.startswith(kern):
            return name[len(kern):-1].split(", ")[pos] == "true"
    return False


def ifq_conv_variant_name(desc, join, variant):
    return _lib().ifq_conv_variant_name(
        ctypes.byref(desc), ctypes.byref(join) if join is not None else None,
        int(variant)).decode()


def ifq_conv_split_workspace_bytes(desc, variant, ksplit):
    return int(_lib().ifq_conv_split_workspace_bytes(ctypes.byref(desc), int(variant),
                                                     int(ksplit)))


def ifq_conv_forward_split(desc, x, w_packed, thr, y, variant, ksplit, ws, acc_dump=None,
                           stream=None):
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(_lib().ifq_conv_forward_split(
        ctypes.byref(desc), _ptr(x), _ptr(w_packed), _ptr(thr), _ptr(y), _ptr(acc_dump),
        int(variant), int(ksplit), _ptr(ws), ws_bytes, _stream(stream)),
        "ifq_conv_forward_split")


def ifq_conv_forward_variant(desc, x, w_packed, thr, y, variant, join=None, acc_dump=None,
                             stream=None):
    _check(_lib().ifq_conv_forward_variant(
        ctypes.byref(desc), _ptr(x), _ptr(w_packed), _ptr(thr),
        ctypes.byref(join) if join is not None else None, _ptr(y), _ptr(acc_dump),
        int(variant), _stream(stream)), "ifq_conv_forward_variant")


# -- operators for serving language models ---------------------------------------
def f8_quant_desc(rows, k, x_type, block_rows=1, ld_x=None, ld_codes=None):
    """ld_codes None: k up to the next multiple of 16."""
    return F8QuantDesc(rows, k, k if ld_x is None else ld_x,
                       -(-k // 16) * 16 if ld_codes is None else ld_codes, x_type, block_rows)


def f8_matmul_desc(m, n, k, y_type, ld_a=None, ld_w=None, ld_y=None):
    return F8MatmulDesc(m, n, k, k if ld_a is None else ld_a, k if ld_w is None else ld_w,
                        n if ld_y is None else ld_y, y_type, 0)


def kv_desc(batch, total_q, max_q, max_kv, heads, kv_heads, head_dim, page_tokens, num_pages,
            max_pages, type, scale=1.0, causal=True, window=0, sinks=0, rot_dim=0,
            rot_adjacent=False, rot_len=0, q_stride=None, k_stride=None, v_stride=None,
            o_stride=None):
    """Strides None: dense rows of all heads."""
    qrow, krow = heads * head_dim, kv_heads * head_dim
    return KvDesc(batch, total_q, max_q, max_kv, heads, kv_heads, head_dim, page_tokens,
                  num_pages, max_pages, type, int(causal), window, sinks, rot_dim,
                  int(rot_adjacent), rot_len, scale, qrow if q_stride is None else q_stride,
                  krow if k_stride is None else k_stride,
                  krow if v_stride is None else v_stride, qrow if o_stride is None else o_stride)


def ifq_f8_quantize(desc, x, codes, scales, stream=None):
    rc = _ffi.call.f8_quantize(_struct(desc, F8QuantDesc), x, codes, scales, _stream(stream))
    if rc:
        _check(rc, "ifq_f8_quantize")


def ifq_f8_matmul_workspace_bytes(desc):
    return int(_lib().ifq_f8_matmul_workspace_bytes(ctypes.byref(desc)))


def ifq_f8_matmul_kernel_name(desc):
    return _lib().ifq_f8_matmul_kernel_name(ctypes.byref(desc)).decode()


def ifq_f8_matmul(desc, a, a_scales, w, w_scales, y, ws=None, stream=None):
    """ws None: a zero-filled device workspace is made for this call where it
    needs one, as for ifq_conv_forward."""
    d, st = _struct(desc, F8MatmulDesc), _stream(stream)
    rc = _ffi.call.f8_matmul(d, a, a_scales, w, w_scales, y, ws, _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        ws = _workspace(ifq_f8_matmul_workspace_bytes(desc), y, st)
        rc = _ffi.call.f8_matmul(d, a, a_scales, w, w_scales, y, ws, _nbytes(ws), st)
    if rc:
        _check(rc, "ifq_f8_matmul")


def _workspace(nbytes, like, stream):
    """A zero-filled workspace on like's device for one call on that stream
    (a handle): made, filled and given back in the stream's order."""
    import torch
    with torch.cuda.device(like.device):
        if stream == _stream(None):
            return torch.zeros(nbytes, dtype=torch.uint8, device=like.device)
        on = torch.cuda.ExternalStream(stream)
        with torch.cuda.stream(on):
            return torch.zeros(nbytes, dtype=torch.uint8, device=like.device)


def ifq_kv_cache_bytes(desc):
    return int(_lib().ifq_kv_cache_bytes(ctypes.byref(desc)))


def ifq_kv_append(desc, q, k, v, cosines, sines, offsets, lengths, pages, cache, q_out,
                  stream=None):
    rc = _ffi.call.kv_append(_struct(desc, KvDesc), q, k, v, cosines, sines, offsets, lengths,
                             pages, cache, q_out, _stream(stream))
    if rc:
        _check(rc, "ifq_kv_append")


def ifq_kv_read(desc, offsets, lengths, pages, cache, k_out, v_out, stream=None):
    rc = _ffi.call.kv_read(_struct(desc, KvDesc), offsets, lengths, pages, cache, k_out, v_out,
                           _stream(stream))
    if rc:
        _check(rc, "ifq_kv_read")


def ifq_kv_attention_workspace_bytes(desc):
    return int(_lib().ifq_kv_attention_workspace_bytes(ctypes.byref(desc)))


def ifq_kv_attention_kernel_name(desc):
    return _lib().ifq_kv_attention_kernel_name(ctypes.byref(desc)).decode()


def ifq_kv_attention(desc, q, offsets, lengths, pages, cache, out, ws=None, stream=None):
    """ws None: as for ifq_f8_matmul."""
    d, st = _struct(desc, KvDesc), _stream(stream)
    rc = _ffi.call.kv_attention(d, q, offsets, lengths, pages, cache, out, ws, _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        ws = _workspace(ifq_kv_attention_workspace_bytes(desc), out, st)
        rc = _ffi.call.kv_attention(d, q, offsets, lengths, pages, cache, out, ws, _nbytes(ws),
                                    st)
    if rc:
        _check(rc, "ifq_kv_attention")


# -- weights in 4-bit floats, and log probabilities -------------------------------
def f4_weights_desc(rows, k, x_type, ld_x=None, ld_codes=None):
    """ld_codes None: 16 bytes for each group of 32 columns."""
    return F4WeightsDesc(rows, k, k if ld_x is None else ld_x,
                         -(-k // 32) * 16 if ld_codes is None else ld_codes, x_type, 0)


def f4_matmul_desc(m, n, k, x_type, y_type=None, ld_x=None, ld_w=None, ld_y=None,
                   activation=_ffi.IFQ_ACT_NONE):
    """y_type None: x's; ld_w None: 16 bytes for each group of 32 columns."""
    return F4MatmulDesc(m, n, k, k if ld_x is None else ld_x,
                        -(-k // 32) * 16 if ld_w is None else ld_w,
                        n if ld_y is None else ld_y, x_type,
                        x_type if y_type is None else y_type, activation, 0)


def logprobs_desc(rows, n, x_type, top=0, scale=1.0, ld_x=None, ld_top=None):
    return LogprobsDesc(rows, n, n if ld_x is None else ld_x, top if ld_top is None else ld_top,
                        x_type, top, scale, 0)


def ifq_f4_quantize(desc, x, codes, scales, stream=None):
    rc = _ffi.call.f4_quantize(_struct(desc, F4WeightsDesc), x, codes, scales, _stream(stream))
    if rc:
        _check(rc, "ifq_f4_quantize")


def ifq_f4_dequantize(desc, codes, scales, x, stream=None):
    rc = _ffi.call.f4_dequantize(_struct(desc, F4WeightsDesc), codes, scales, x, _stream(stream))
    if rc:
        _check(rc, "ifq_f4_dequantize")


def ifq_f4_matmul_workspace_bytes(desc):
    return int(_lib().ifq_f4_matmul_workspace_bytes(ctypes.byref(desc)))


def ifq_f4_gated_workspace_bytes(desc):
    return int(_lib().ifq_f4_gated_workspace_bytes(ctypes.byref(desc)))


def ifq_f4_matmul_kernel_name(desc):
    return _lib().ifq_f4_matmul_kernel_name(ctypes.byref(desc)).decode()


def ifq_f4_gated_kernel_name(desc):
    return _lib().ifq_f4_gated_kernel_name(ctypes.byref(desc)).decode()


def ifq_f4_matmul(desc, x, w, w_scales, y, ws=None, stream=None):
    """ws None: as for ifq_f8_matmul."""
    d, st = _struct(desc, F4MatmulDesc), _stream(stream)
    rc = _ffi.call.f4_matmul(d, x, w, w_scales, y, ws, _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        ws = _workspace(ifq_f4_matmul_workspace_bytes(desc), y, st)
        rc = _ffi.call.f4_matmul(d, x, w, w_scales, y, ws, _nbytes(ws), st)
    if rc:
        _check(rc, "ifq_f4_matmul")


def ifq_f4_gated(desc, x, w_gate, gate_scales, w_up, up_scales, y, ws=None, stream=None):
    """ws None: as for ifq_f8_matmul."""
    d, st = _struct(desc, F4MatmulDesc), _stream(stream)
    rc = _ffi.call.f4_gated(d, x, w_gate, gate_scales, w_up, up_scales, y, ws, _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        ws = _workspace(ifq_f4_gated_workspace_bytes(desc), y, st)
        rc = _ffi.call.f4_gated(d, x, w_gate, gate_scales, w_up, up_scales, y, ws, _nbytes(ws),
                                st)
    if rc:
        _check(rc, "ifq_f4_gated")


def ifq_logprobs_workspace_bytes(desc):
    return int(_lib().ifq_logprobs_workspace_bytes(ctypes.byref(desc)))


def ifq_logprobs(desc, logits, tokens, logprob, entropy, top_logprobs, top_tokens, ws=None,
                 stream=None):
    """ws None: as for ifq_f8_matmul."""
    d, st = _struct(desc, LogprobsDesc), _stream(stream)
    rc = _ffi.call.logprobs(d, logits, tokens, logprob, entropy, top_logprobs, top_tokens, ws,
                            _nbytes(ws), st)
    if rc == _ffi.IFQ_ERR_INSUFFICIENT_BUFFER and ws is None:
        ws = _workspace(ifq_logprobs_workspace_bytes(desc), logits, st)
        rc = _ffi.call.logprobs(d, logits, tokens, logprob, entropy, top_logprobs, top_tokens,
                                ws, _nbytes(ws), st)
    if rc:
        _check(rc, "ifq_logprobs")
