"""Performance cases of the operators that follow a decoder's attention: weights
in 4-bit floats with a scale per 32 (the quantizer with its read-back, and the
product of 16-bit activations with such weights), the gated feed-forward
product on the same weights, and log probabilities of given tokens with entropy
and top alternatives.

A case is one call (the quantizer: the call and the read-back of what it stored)
that a program serving a model makes per layer and step, or once per weight
matrix. Values come from the seed.

Where `own` is false, run() computes the same in elementary torch operations
in 32 bits; exact() gives the outputs in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 32                        # values under one scale
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LEAST = 2.0 ** -96                # a group's largest value counts as at least this


# -- cases ---------------------------------------------------------------------
def listed():
    return [
        # one square layer's weights are laid out when a model is loaded
        {"name": "quantize layer", "op": "quantize", "n": 4096, "k": 4096, "type": "bf16"},
        # a classifier's weights, kept in 32 bits until then
        {"name": "quantize classifier", "op": "quantize", "n": 64001, "k": 4096, "type": "f32"},
        # one token back to the hidden size: latency, reads the weights once
        {"name": "product one token", "op": "product", "m": 1, "n": 4096, "k": 14336,
         "x": "bf16", "y": "bf16"},
        # a decoding batch into queries, keys and values at once
        {"name": "product batch", "op": "product", "m": 24, "n": 6144, "k": 4096,
         "x": "f16", "y": "f16"},
        # a few sequences' last tokens through the classifier, logits kept in 32 bits
        {"name": "product classifier", "op": "product", "m": 7, "n": 128000, "k": 4096,
         "x": "bf16", "y": "f32"},
        # a prompt of ragged length back to the hidden size
        {"name": "product prompt", "op": "product", "m": 2011, "n": 4096, "k": 14336,
         "x": "bf16", "y": "bf16"},
        # one token into the inner size of the feed-forward: latency
        {"name": "gated one token", "op": "gated", "m": 1, "n": 14336, "k": 4096,
         "x": "bf16", "y": "bf16", "act": "silu"},
        # a decoding batch, sizes that fit no tile
        {"name": "gated batch", "op": "gated", "m": 41, "n": 9001, "k": 4008,
         "x": "f16", "y": "f16", "act": "gelu"},
        # a long prompt
        {"name": "gated prompt", "op": "gated", "m": 3001, "n": 14336, "k": 4096,
         "x": "bf16", "y": "bf16", "act": "silu"},
        # the alternatives of one answered token: latency
        {"name": "logprobs one token", "op": "logprobs", "rows": 1, "n": 128000, "type": "f32",
         "top": 20, "scale": 1.0, "masked": 0.0},
        # a decoding batch at a temperature, part of the vocabulary forbidden
        {"name": "logprobs batch", "op": "logprobs", "rows": 96, "n": 50001, "type": "bf16",
         "top": 5, "scale": 1.25, "masked": 0.3},
        # every token of a long prompt is scored
        {"name": "logprobs prompt", "op": "logprobs", "rows": 4000, "n": 32000, "type": "f32",
         "top": 0, "scale": 1.0, "masked": 0.0},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "gated", "gated", "logprobs", "logprobs"])
    if op == "quantize":
        n = _log(rng, 16, 64000)
        return {"op": op, "n": n, "k": _log(rng, 33, min(14336, 260000000 // n)),
                "type": rng.choice(["bf16", "f16", "f32"])}
    if op == "logprobs":
        rows = _log(rng, 1, 4096)
        n = _log(rng, 200, min(200000, 128000000 // rows))
        return {"op": op, "rows": rows, "n": n, "type": rng.choice(["bf16", "f16", "f32"]),
                "top": min(rng.choice([0, 1, 5, 20, 33]), n // 20),
                "scale": rng.choice([1.0, 1.0, 0.5, 1.25]),
                "masked": rng.choice([0.0, 0.0, 0.2, 0.8])}
    m, k = _log(rng, 1, 3000), _log(rng, 64, 14336)
    # rows whose length is a multiple of 8 as they mostly are, and some that are not
    k = k if rng.random() < 0.25 else -(-k // 8) * 8
    most = 128000 if op == "product" and m <= 16 else 14336
    n = _log(rng, 100, max(100, min(most, 500000000 // k, 170000000000 // (m * k))))
    x = rng.choice(["bf16", "f16"])
    case = {"op": op, "m": m, "n": n, "k": k, "x": x, "y": rng.choice([x, x, "f32"])}
    if op == "gated":
        case["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
    return case


def work(case):
    op = case["op"]
    if op == "quantize":
        # read and coded, and the codes read and written as values
        values = case["n"] * case["k"]
        codes = case["n"] * -(-case["k"] // GROUP) * 17
        return {"bytes": 2 * values * SIZE[case["type"]] + 2 * codes, "flops": 3 * values}
    if op == "logprobs":
        rows, values = case["rows"], case["rows"] * case["n"]
        return {"bytes": values * SIZE[case["type"]] + rows * (12 + 8 * case["top"]),
                "flops": 6 * values}
    m, n, k = case["m"], case["n"], case["k"]
    both = 2 if op == "gated" else 1
    return {"bytes": both * n * -(-k // GROUP) * 17 + m * k * 2 + m * n * SIZE[case["y"]],
            "flops": 2 * both * m * n * k}


# -- the weights' format ---------------------------------------------------------
# A code is a float of 4 bits: sign, 2 exponent bits, 1 mantissa bit (magnitudes
# 0, 0.5, 1, 1.5, 2, 3, 4, 6). A row's codes lie two in a byte, the first in the
# low half, in groups of 32. A group's scale is a byte s that stands for
# 2^(s - 127); the scales lie [128 columns][row][4].
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _encode(x):
    """Codes [n][groups][32] and the scales' exponents [n][groups] of rows x in 32 bits: the
    smallest exponent e with all of |x| <= 7 * 2^e, the nearest code, ties to the even one."""
    n, k = x.shape
    groups = -(-k // GROUP)
    x = torch.nn.functional.pad(x, (0, groups * GROUP - k)).view(n, groups, GROUP)
    part, e = torch.frexp(x.abs().amax(-1).clamp_min(LEAST))
    e = torch.where(part > 0.875, e - 2, e - 3)
    a = torch.ldexp(x.abs(), -e[..., None])
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i in range(7):
        half = (MAGNITUDES[i] + MAGNITUDES[i + 1]) / 2
        code += (a > half) if i % 2 == 0 else (a >= half)
    return code | (torch.signbit(x).to(torch.uint8) << 3), e


def _pack(code, e):
    """The layout: codes [n][groups * 16], scales [128 columns][n][4]."""
    n, groups, _ = code.shape
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -groups % 4), value=29)
    return ((code[..., 0::2] | (code[..., 1::2] << 4)).view(n, -1),
            s.view(n, -1, 4).transpose(0, 1).contiguous())


def _decode(codes, scales, k):
    """Values [n][k] in 32 bits."""
    n = codes.shape[0]
    c = torch.stack([codes & 15, codes >> 4], -1).view(n, -1, GROUP)
    s = scales.transpose(0, 1).reshape(n, -1)[:, :c.shape[1]]
    table = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=codes.device)
    v = table[c.int()] * torch.exp2(s.float() - 127.0)[..., None]
    return v.view(n, -1)[:, :k]


# -- inputs --------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _weights(g, n, k):
    codes = torch.empty(n, -(-k // GROUP) * 16, dtype=torch.uint8, device=DEV)
    scales = torch.empty(-(-k // 128), n, 4, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // k)
    for i in range(0, n, step):
        rows = min(step, n - i)
        w = _randn(g, rows, k) * torch.exp(0.3 * _randn(g, rows, 1)) * k ** -0.5
        codes[i:i + rows], scales[:, i:i + rows] = _pack(*_encode(w))
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    s = {"case": case, "op": op}
    if op == "quantize":
        n, k = case["n"], case["k"]
        w = _randn(g, n, k)
        w *= torch.exp(0.3 * _randn(g, n, 1)) * k ** -0.5
        s["x"] = w.to(TYPES[case["type"]])
        return s
    if op == "logprobs":
        rows, n = case["rows"], case["n"]
        x = 2.5 * _randn(g, rows, n)
        # what a model is sure of: a few far above the others, in most of the rows
        sure = torch.randint(0, n, (rows, 3), generator=g, device=DEV)
        x.scatter_add_(1, sure, 6.0 * _randn(g, rows, 3).abs())
        tokens = torch.where(_randn(g, rows) > 0, sure[:, 0],
                             torch.randint(0, n, (rows,), generator=g, device=DEV))
        x = x.to(TYPES[case["type"]])
        if case["masked"]:
            # half of the rows forbid with infinity, the others with the type's lowest value
            gone = torch.rand(rows, n, generator=g, device=DEV) < case["masked"]
            gone.scatter_(1, tokens[:, None], False)
            x[0::2].masked_fill_(gone[0::2], -math.inf)
            x[1::2].masked_fill_(gone[1::2], torch.finfo(x.dtype).min)
        # rows of padding have no token
        tokens[3::7] = -1
        s["x"], s["tokens"] = x, tokens.int()
        return s
    m, n, k = case["m"], case["n"], case["k"]
    # activations: channels of different spread
    x = _randn(g, m, k)
    x *= torch.exp(0.5 * _randn(g, 1, k))
    s["x"] = x.to(TYPES[case["x"]])
    if op == "gated":
        s["wg"], s["sg"] = _weights(g, n, k)
    s["w"], s["s"] = _weights(g, n, k)
    return s


# -- plain forms -----------------------------------------------------------------
def _plain_quantize(s):
    x = s["x"].float()
    return {"values": _decode(*_pack(*_encode(x)), x.shape[1]).to(s["x"].dtype)}


def _plain_product(s):
    c = s["case"]
    y = s["x"].float() @ _decode(s["w"], s["s"], c["k"]).t()
    return {"y": y.to(TYPES[c["y"]])}


def _plain_gated(s):
    c, x = s["case"], s["x"].float()
    g = x @ _decode(s["wg"], s["sg"], c["k"]).t()
    u = x @ _decode(s["w"], s["s"], c["k"]).t()
    if c["act"] == "silu":
        a = g / (1 + torch.exp(-g))
    elif c["act"] == "gelu":
        a = 0.5 * g * torch.special.erfc(g * -math.sqrt(0.5))
    else:
        a = g / (1 + torch.exp(g * (g * g * 0.044715 + 1) * (-2 * math.sqrt(2 / math.pi))))
    return {"y": (a * u).to(TYPES[c["y"]])}


def _plain_logprobs(s):
    c, logits = s["case"], s["x"]
    x = logits.float()
    z = (x - x.amax(-1, keepdim=True)) * c["scale"]
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    log = torch.log(total)
    entropy = log - torch.where(e > 0, z * e, 0.0).sum(-1, keepdim=True) / total
    t = s["tokens"].long()[:, None]
    given = torch.where(t < 0, 0.0, z.gather(1, t.clamp_min(0)) - log)
    out = {"logprob": given[:, 0], "entropy": entropy[:, 0]}
    if c["top"]:
        at = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
        out["top"], out["tokens"] = z.gather(1, at) - log, at.int()
    return out


# -- the framework's calls ---------------------------------------------------------
def _type(P, name):
    return {"bf16": P.IFQ_TYPE_BF16, "f16": P.IFQ_TYPE_F16, "f32": P.IFQ_TYPE_F32}[name]


def _plan(P, s):
    """What a program keeps between calls: the descriptor and the workspace."""
    c, op = s["case"], s["op"]
    if op == "quantize":
        return P.f4_weights_desc(c["n"], c["k"], _type(P, c["type"])), None
    if op == "logprobs":
        desc = P.logprobs_desc(c["rows"], c["n"], _type(P, c["type"]), top=c["top"],
                               scale=c["scale"])
        ws = P.ifq_logprobs_workspace_bytes(desc)
    elif op == "gated":
        act = {"silu": P.IFQ_ACT_SILU, "gelu": P.IFQ_ACT_GELU, "gelu_tanh": P.IFQ_ACT_GELU_TANH}
        desc = P.f4_matmul_desc(c["m"], c["n"], c["k"], _type(P, c["x"]), _type(P, c["y"]),
                                activation=act[c["act"]])
        ws = P.ifq_f4_gated_workspace_bytes(desc)
    else:
        desc = P.f4_matmul_desc(c["m"], c["n"], c["k"], _type(P, c["x"]), _type(P, c["y"]))
        ws = P.ifq_f4_matmul_workspace_bytes(desc)
    return desc, torch.zeros(ws, dtype=torch.uint8, device=DEV) if ws else None


def _own(s):
    import paper_1911_08076_amd as P
    if "plan" not in s:
        s["plan"] = _plan(P, s)
    desc, ws = s["plan"]
    c, op, x = s["case"], s["op"], s["x"]
    if op == "quantize":
        codes = torch.empty(c["n"], -(-c["k"] // GROUP) * 16, dtype=torch.uint8, device=DEV)
        scales = torch.empty(-(-c["k"] // 128), c["n"], 4, dtype=torch.uint8, device=DEV)
        values = torch.empty_like(x)
        P.ifq_f4_quantize(desc, x, codes, scales)
        P.ifq_f4_dequantize(desc, codes, scales, values)
        return {"values": values}
    if op == "logprobs":
        rows, top = c["rows"], c["top"]
        both = torch.empty(2, rows, device=DEV)
        if not top:
            P.ifq_logprobs(desc, x, s["tokens"], both[0], both[1], None, None, ws=ws)
            return {"logprob": both[0], "entropy": both[1]}
        best = torch.empty(rows, top, device=DEV)
        at = torch.empty(rows, top, dtype=torch.int32, device=DEV)
        P.ifq_logprobs(desc, x, s["tokens"], both[0], both[1], best, at, ws=ws)
        return {"logprob": both[0], "entropy": both[1], "top": best, "tokens": at}
    y = torch.empty(c["m"], c["n"], dtype=TYPES[c["y"]], device=DEV)
    if op == "gated":
        P.ifq_f4_gated(desc, x, s["wg"], s["sg"], s["w"], s["s"], y, ws=ws)
    else:
        P.ifq_f4_matmul(desc, x, s["w"], s["s"], y, ws=ws)
    return {"y": y}


def run(state):
    if own:
        return _own(state)
    return {"quantize": _plain_quantize, "product": _plain_product, "gated": _plain_gated,
            "logprobs": _plain_logprobs}[state["op"]](state)


# -- the operators' definitions in 64 bits -------------------------------------------
def _held(codes, scales, n, k):
    """What codes and scales stand for, [n][k], from the bits of each code."""
    w = torch.empty(n, codes.shape[1] * 2, dtype=torch.float64, device=DEV)
    for half in (0, 1):
        c = (codes >> (4 * half)) & 15
        mantissa, power = (c & 1).double() / 2, ((c >> 1) & 3).double()
        v = torch.where(power == 0, mantissa, (1 + mantissa) * torch.exp2(power - 1))
        w[:, half::2] = torch.where(c >= 8, -v, v)
    for b in range(scales.shape[0]):
        for i in range(4):
            at = slice(128 * b + 32 * i, 128 * b + 32 * (i + 1))
            w[:, at] *= torch.exp2(scales[b, :, i].double() - 127)[:, None]
    return w[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        out = torch.empty(case["n"], case["k"], dtype=torch.float64, device=DEV)
        for b in range(0, case["k"], GROUP):
            x = s["x"][:, b:b + GROUP].double()
            # 7 * 2^e holds the largest, 7 * 2^(e - 1) does not
            e = torch.ceil(torch.log2(x.abs().amax(1).clamp_min(LEAST) / 7))
            v = x / torch.exp2(e)[:, None]
            # spacing of the codes: a half up to 2, one up to 4, then two
            unit = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
            v = (torch.round(v / unit) * unit).clamp(-6, 6)
            out[:, b:b + GROUP] = v * torch.exp2(e)[:, None]
        return {"values": out}
    x = s["x"].double()
    if op == "logprobs":
        z = x * case["scale"]
        log = torch.logsumexp(z, 1, keepdim=True)
        p = torch.exp(z - log)
        entropy = torch.where(p > 0, -p * (z - log), 0.0).sum(1)
        t = s["tokens"].long()
        given = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
        some = t >= 0
        given[some] = (z - log)[some, t[some]]
        out = {"logprob": given, "entropy": entropy}
        if case["top"]:
            at = []
            number = torch.arange(case["n"], device=DEV)
            left = torch.ones_like(x, dtype=torch.bool)
            for _ in range(case["top"]):
                best = torch.where(left, x, -math.inf).amax(1, keepdim=True)
                first = torch.where(left & (x == best), number, case["n"]).amin(1)
                left.scatter_(1, first[:, None], False)
                at.append(first)
            at = torch.stack(at, 1)
            out["top"], out["tokens"] = (z - log).gather(1, at), at.int()
        return out
    n, k = case["n"], case["k"]
    u = x @ _held(s["w"], s["s"], n, k).t()
    if op == "product":
        return {"y": u}
    g = x @ _held(s["wg"], s["sg"], n, k).t()
    if case["act"] == "silu":
        g = g * torch.sigmoid(g)
    elif case["act"] == "gelu":
        g = g * torch.special.erfc(-g / math.sqrt(2)) / 2
    else:
        g = g / 2 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    return {"y": g * u}
