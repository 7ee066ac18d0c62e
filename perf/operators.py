"""Performance cases of the operators for serving language models: the quantizer
to 8-bit floating point and the block-scaled product on its codes, the append
to a paged cache of 4-bit codes with the position rotation, and attention over
that cache.

A case is one call (the append: the call and the read-back of what it stored)
that a program serving a model makes per layer and step. Lengths are spread
over a batch by a rule of the case alone, values come from the seed.

Where `own` is false, run() computes the same in elementary torch operations
in 32 bits; exact() gives the outputs in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128                       # values under one scale
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
TINY = 2.0 ** -96


# -- cases ---------------------------------------------------------------------
def listed():
    return [
        # one token's hidden state on its way into a layer: latency
        {"name": "quantize one token", "op": "quantize", "rows": 1, "k": 4096,
         "type": "bf16", "block_rows": 1},
        # the wide inner activations of a long prompt
        {"name": "quantize prompt", "op": "quantize", "rows": 8192, "k": 14336,
         "type": "bf16", "block_rows": 1},
        # one token through one square layer: reads the weights once
        {"name": "product one token", "op": "product", "m": 1, "n": 4096, "k": 4096,
         "type": "bf16"},
        # a decoding batch through a classifier of 1000 outputs, sums kept in 32 bits
        {"name": "product classifier", "op": "product", "m": 37, "n": 1000, "k": 4096,
         "type": "f32"},
        # a short prompt of ragged length into queries, keys and values at once
        {"name": "product short prompt", "op": "product", "m": 515, "n": 6144, "k": 4096,
         "type": "f16"},
        # a long prompt through the widening layer
        {"name": "product prompt", "op": "product", "m": 8192, "n": 14336, "k": 4096,
         "type": "bf16"},
        # a decoding batch stores one token for each sequence
        {"name": "append one each", "op": "append", "batch": 64, "q_min": 1, "q_max": 1,
         "len_min": 1, "len_max": 8000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "type": "bf16", "rot": 128, "adjacent": False},
        # prompts of several sequences stored together, some behind a prefix
        {"name": "append prompts", "op": "append", "batch": 7, "q_min": 129, "q_max": 3001,
         "len_min": 129, "len_max": 5000, "heads": 16, "kv_heads": 16, "dim": 64, "page": 32,
         "type": "f16", "rot": 32, "adjacent": True},
        # one sequence answers token by token: latency
        {"name": "attend one", "op": "attend", "batch": 1, "q_min": 1, "q_max": 1,
         "len_min": 1111, "len_max": 1111, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "type": "bf16", "window": 0, "sinks": 0},
        # a decoding batch of ragged lengths, one of them still empty, behind a window with sinks
        {"name": "attend batch window", "op": "attend", "batch": 96, "q_min": 1, "q_max": 1,
         "len_min": 0, "len_max": 12000, "heads": 64, "kv_heads": 8, "dim": 64, "page": 32,
         "type": "f16", "window": 4096, "sinks": 4},
        # a few sequences over long documents
        {"name": "attend long", "op": "attend", "batch": 5, "q_min": 1, "q_max": 1,
         "len_min": 20000, "len_max": 120001, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 128, "type": "bf16", "window": 0, "sinks": 0},
        # prompts in chunks behind what the cache holds already
        {"name": "attend prompt chunks", "op": "attend", "batch": 3, "q_min": 900, "q_max": 2048,
         "len_min": 2048, "len_max": 6100, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "type": "bf16", "window": 0, "sinks": 0},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["quantize", "product", "product", "append", "attend", "attend"])
    if op == "quantize":
        rows = _log(rng, 1, 8192)
        return {"op": op, "rows": rows, "k": _log(rng, 65, 14336),
                "type": rng.choice(["bf16", "f16", "f32"]), "block_rows": rng.choice([1, 1, 128])}
    if op == "product":
        return {"op": op, "m": _log(rng, 1, 8192), "n": _log(rng, 100, 14336),
                "k": 16 * _log(rng, 16, 190), "type": rng.choice(["bf16", "f16", "f32"])}
    kv = rng.choice([1, 2, 4, 8])
    case = {"op": op, "heads": kv * rng.choice([1, 4, 5, 8]), "kv_heads": kv,
            "dim": rng.choice([64, 128, 128, 256]), "page": rng.choice([32, 64, 128, 256]),
            "type": rng.choice(["bf16", "f16"])}
    if op == "append":
        most = _log(rng, 1, 3000)
        q_min = max(1, most // rng.choice([1, 2, 9]))
        case.update(batch=_log(rng, 1, 64 if most < 400 else 7), q_min=q_min, q_max=most,
                    len_min=most, len_max=most + _log(rng, 1, 4000),
                    adjacent=rng.choice([False, True]),
                    rot=rng.choice([case["dim"], case["dim"] // 2]))
        return case
    if rng.random() < 0.3:                      # prompts
        most = _log(rng, 2, min(2048, 8192000 // (case["heads"] * case["dim"])))
        case.update(batch=_log(rng, 1, 3), q_min=max(1, most // 2), q_max=most,
                    len_max=most + _log(rng, 1, 4000))
        case["len_min"] = rng.choice([most, max(1, most // 4)])
    else:
        batch = _log(rng, 1, 96)
        longest = _log(rng, 1, min(120000, 600000000 // (batch * kv * case["dim"])))
        case.update(batch=batch, q_min=1, q_max=1, len_min=longest // rng.choice([1, 3, 50]),
                    len_max=longest)
    window = rng.choice([0, 0, _log(rng, 1, 5000)])
    case.update(window=window, sinks=rng.choice([0, 4, 33]) if window else 0)
    return case


def _spread(lo, hi, n, by):
    """n whole numbers from lo to hi, both among them where n > 1, in mixed order."""
    if n == 1:
        return [hi]
    return [lo + (hi - lo) * ((i * by + n - 1) % n) // (n - 1) for i in range(n)]


def _coprime(n, near):
    while math.gcd(n, near) != 1:
        near += 1
    return near


def _lengths(case):
    """(new tokens, cached tokens with them) of each sequence. A sequence may be
    shorter than what it asks with (attention: such queries see nothing)."""
    b = case["batch"]
    lens = _spread(case["len_min"], case["len_max"], b, _coprime(b, 5))
    new = _spread(case["q_min"], case["q_max"], b, _coprime(b, 3))
    if case["op"] == "append":
        new = [min(q, n) for q, n in zip(new, lens)]
    return new, lens


def _visible(case):
    """Pairs of a query and a cached token that it sees, and cached tokens seen by any."""
    pairs = seen = 0
    w, s = case["window"], case["sinks"]
    for q, n in zip(*_lengths(case)):
        first = last = None
        for i in range(q):
            p = n - q + i
            if p < 0:
                continue
            lo = max(0, p - w + 1) if w else 0
            pairs += p - lo + 1 + min(s, lo)
            first = lo if first is None else first
            last = p
        if last is not None:
            seen += last - first + 1 + min(s, first)
    return pairs, seen


def work(case):
    if case["op"] == "quantize":
        values = case["rows"] * case["k"]
        blocks = -(-case["rows"] // case["block_rows"]) * -(-case["k"] // BLOCK)
        return {"bytes": values * (SIZE[case["type"]] + 1) + 4 * blocks, "flops": 3 * values}
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        return {"bytes": (m + n) * k + 4 * kb * (m + -(-n // BLOCK)) + m * n * SIZE[case["type"]],
                "flops": 2 * m * n * k}
    h, hk, d, e = case["heads"], case["kv_heads"], case["dim"], SIZE[case["type"]]
    new = sum(_lengths(case)[0])
    if case["op"] == "append":
        # q, k, v and the rotation read, q and the cache written, the cache read, k and v written
        return {"bytes": new * (2 * h * d * e + 2 * hk * d * e + 4 * case["rot"]
                                + 2 * hk * (d + 8) + 2 * hk * d * e),
                "flops": new * (3 * (h + hk) * case["rot"] + 8 * hk * d)}
    pairs, seen = _visible(case)
    return {"bytes": seen * hk * (d + 8) + 2 * new * h * d * e, "flops": 4 * pairs * h * d}


# -- inputs --------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case, "op": case["op"], "type": TYPES[case["type"]]}
    if case["op"] == "quantize":
        # activations: channels of different spread, a few large ones
        x = _randn(g, case["rows"], case["k"])
        x *= torch.exp(0.7 * _randn(g, 1, case["k"]))
        s["x"] = x.to(s["type"])
        return s
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        # codes fill their range up to 448 in each block of 128 as the quantizer leaves them
        s["a"] = (_randn(g, m, k) * 130).clamp_(-F8_MAX, F8_MAX).to(F8)
        s["w"] = (_randn(g, n, k) * 110).clamp_(-F8_MAX, F8_MAX).to(F8)
        s["sa"] = 0.01 * torch.exp(0.5 * _randn(g, kb, m))
        s["sw"] = 0.0002 * torch.exp(0.3 * _randn(g, kb, -(-n // BLOCK)))
        return s
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    page, batch = case["page"], case["batch"]
    new, lens = _lengths(case)
    most = max(1, -(-max(lens) // page))
    pages = batch * most + 3
    total = sum(new)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["offs"] = torch.tensor([sum(new[:i]) for i in range(batch + 1)], dtype=torch.int32,
                             device=DEV)
    s["pages"] = torch.randperm(pages, generator=g, device=DEV)[:batch * most].to(
        torch.int32).view(batch, most)
    s["total"], s["max_q"] = total, max(new)
    s["q"] = (1.5 * _randn(g, total, h, d)).to(s["type"])
    # what nobody wrote holds anything, NaN and infinity as scales among it
    cache = torch.randint(0, 256, (pages, hk, page * (d + 8)), generator=g, device=DEV,
                          dtype=torch.uint8)
    s["cache"] = cache
    if case["op"] == "append":
        # keys and values of the new tokens lie beside the queries as the layer's product leaves them
        rows = _randn(g, total, h + 2 * hk, d)
        rows[:, h:h + hk] *= torch.exp(0.6 * _randn(g, 1, hk, d))
        rows = rows.to(s["type"])
        s["q"], s["k"], s["v"] = rows[:, :h], rows[:, h:h + hk], rows[:, h + hk:]
        r = case["rot"]
        freq = 10000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
        ang = torch.arange(most * page, device=DEV, dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        return s
    std = torch.exp(0.5 * _randn(g, 1, hk, 1, d))
    mean = 0.3 * _randn(g, 1, hk, 1, d)
    live = torch.arange(most * page, device=DEV) < s["lens"][:, None]      # [batch, most*page]
    live = live.view(-1, 1, page)
    at = s["pages"].reshape(-1).long()
    for part, first in ((0, 0), (1, page * (d // 2))):
        rows = _randn(g, batch * most, hk, page, d)
        rows = rows * std if part == 0 else rows + mean
        off, step, code = _encode(rows)
        del rows
        held = _k_bytes(code) if part == 0 else _v_bytes(code)
        cache[at, :, first:first + page * (d // 2)] = held.view(batch * most, hk, -1)
        del held, code
        prm = torch.stack([off, step], -1).to(torch.bfloat16)
        first = page * d + 4 * page * part
        old = cache[at, :, first:first + 4 * page].view(torch.bfloat16).view(prm.shape)
        prm = torch.where(live[..., None], prm, old)
        cache[at, :, first:first + 4 * page] = prm.view(-1, hk, 2 * page).view(torch.uint8)
    return s


# -- the cache's format ----------------------------------------------------------
# A page holds, for each of the kv heads, the keys' codes, the values' codes, and
# a word for each key and each value: the row's offset and step in bfloat16.
#   keys    [token][dim / 2]: 8 dims in 4 bytes, dim 2p + h in nibble p + 4h
#   values  [token / 32][dim / 64][16 g + n][b]: 4 bytes of 8 tokens of one dim
#           64 .. + 16 b + n, token 16 t + 4 g + r (of 32) in nibble p + 4h with
#           4 t + r = 2p + h
def _floor_bf16(x):
    """x rounded to bfloat16 towards minus infinity."""
    bits = x.view(torch.int32)
    return torch.where(bits < 0, bits + 0xFFFF, bits).bitwise_and(-65536).view(torch.float32)


def _encode(x):
    """Offset, step and codes of the rows (last axis) of x."""
    lo, hi = x.amin(-1), x.amax(-1)
    off = _floor_bf16(lo.contiguous())
    step = torch.div(hi - off, torch.full_like(hi, 15.0))
    step = ((step.contiguous().view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)
    code = ((x - off[..., None]) / step[..., None]).round_().clamp_(0, 15)
    return off, step, code.nan_to_num_(0.0).to(torch.uint8)


def _k_bytes(code):
    c = code.view(*code.shape[:-1], -1, 4, 2)          # dims 2p + h -> nibbles p + 4h
    c = c.transpose(-1, -2).reshape(*code.shape[:-1], -1, 2)
    return c[..., 0] | (c[..., 1] << 4)


def _k_codes(held):
    c = torch.stack([held & 15, held >> 4], -1).view(*held.shape[:-1], -1, 2, 4)
    return c.transpose(-1, -2).reshape(*held.shape[:-1], -1)


def _v_bytes(code):
    *lead, page, d = code.shape
    c = code.view(*lead, page // 32, 2, 4, 2, 2, d // 64, 4, 16)   # [32][t][g][r1][h][64][b][n]
    k = len(lead)
    c = c.permute(*range(k), k, k + 5, k + 2, k + 7, k + 6, k + 4, k + 1, k + 3)
    c = c.reshape(*lead, -1, 2)                                    # [32][64][g][n][b][h][t][r1]
    return c[..., 0] | (c[..., 1] << 4)


def _v_codes(held, page, d):
    *lead, _ = held.shape
    c = torch.stack([held & 15, held >> 4], -1)
    c = c.view(*lead, page // 32, d // 64, 4, 16, 4, 2, 2, 2)      # [32][64][g][n][b][h][t][r1]
    k = len(lead)
    c = c.permute(*range(k), k, k + 6, k + 2, k + 7, k + 5, k + 1, k + 4, k + 3)
    return c.reshape(*lead, page, d)


def _plain_cached(cache, pages, page, d):
    """Keys and values of all positions in the table, [batch, kv head, position, dim] in 32 bits."""
    batch, most = pages.shape
    hk = cache.shape[1]
    got = cache[pages.reshape(-1).long()]                          # [batch*most, hk, bytes]
    out = []
    for part in (0, 1):
        held = got[:, :, part * page * (d // 2):(part + 1) * page * (d // 2)]
        code = _k_codes(held.reshape(-1, hk, page, d // 2)) if part == 0 else _v_codes(
            held, page, d)
        first = page * d + 4 * page * part
        prm = got[:, :, first:first + 4 * page].contiguous().view(torch.bfloat16)
        prm = prm.view(-1, hk, page, 2).float()
        x = prm[..., :1] + prm[..., 1:] * code.float()
        out.append(x.view(batch, most, hk, page, d).transpose(1, 2).reshape(batch, hk, -1, d))
    return out


# -- plain forms -----------------------------------------------------------------
def _plain_quantize(s):
    c, x = s["case"], s["x"].float()
    rows, k, br = c["rows"], c["k"], c["block_rows"]
    rb, kb = -(-rows // br), -(-k // BLOCK)
    x = torch.nn.functional.pad(x, (0, kb * BLOCK - k, 0, rb * br - rows))
    x = x.view(rb, br, kb, BLOCK)
    top = x.abs().amax((1, 3)).clamp_min(TINY)
    scale = torch.div(top, torch.full_like(top, F8_MAX))
    # x * 448 / top, with 448 / 512 and 512 / top so that nothing overflows
    code = torch.div(x * (F8_MAX / 512), (top / 512)[:, None, :, None])
    code = code.clamp_(-F8_MAX, F8_MAX).to(F8)
    code = code.view(torch.uint8).view(rb * br, kb * BLOCK)[:rows, :k].contiguous()
    return {"codes": code.view(F8), "scales": scale.t().contiguous()}


def _plain_product(s):
    m, k = s["a"].shape
    n = s["w"].shape[0]
    sa = s["sa"].t().repeat_interleave(BLOCK, 1)[:, :k]
    sw = s["sw"].t().repeat_interleave(BLOCK, 1)[:, :k].repeat_interleave(BLOCK, 0)[:n]
    return {"y": ((s["a"].float() * sa) @ (s["w"].float() * sw).t()).to(s["type"])}


def _rotate(x, cos, sin, adjacent):
    """x [token, head, dim], cos and sin [token, rot / 2]."""
    r = 2 * cos.shape[1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if adjacent else (x[..., :r // 2], x[..., r // 2:r])
    cos, sin = cos[:, None], sin[:, None]
    p, q = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([p, q], -1).flatten(-2) if adjacent else torch.cat([p, q], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _places(s):
    """Sequence and position of each new token."""
    t = torch.arange(s["total"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["offs"], t, right=True) - 1
    return seq, (s["lens"][seq] - s["offs"][seq + 1] + t).long()


def _plain_append(s):
    c, cache = s["case"], s["cache"]
    page, d = c["page"], c["dim"]
    hk, at = cache.shape[1], torch.arange(c["dim"], device=DEV)
    seq, pos = _places(s)
    cos, sin = s["cos"][pos], s["sin"][pos]
    q = _rotate(s["q"].float(), cos, sin, c["adjacent"]).to(s["type"])
    k = _rotate(s["k"].float(), cos, sin, c["adjacent"])
    v = s["v"].float()
    ids = s["pages"][seq, pos // page].long()
    slot = pos % page
    head = torch.arange(hk, device=DEV)
    words = cache.view(torch.int32)                                # [pages, hk, page*(d+8)/4]
    koff, kstep, kcode = _encode(k)
    voff, vstep, vcode = _encode(v)
    key = torch.arange(d // 8, device=DEV)
    words[ids[:, None, None], head[:, None], (slot * (d // 8))[:, None, None] + key] = (
        _k_bytes(kcode).view(torch.int32))
    for part, off, step in ((0, koff, kstep), (1, voff, vstep)):
        prm = torch.stack([off, step], -1).to(torch.bfloat16).view(torch.int32)[..., 0]
        words[ids[:, None], head, (page * (d // 4) + page * part + slot)[:, None]] = prm
    # a value's code is one nibble of its word: the word gets the difference to the old one
    tok = slot % 32
    e = 4 * (tok // 16) + tok % 4
    shift = (4 * (e // 2 + 4 * (e % 2)))[:, None, None].int()
    word = (page * (d // 8) + (slot // 32) * (4 * d))[:, None] + 256 * (at // 64) + (
        64 * ((tok % 16) // 4))[:, None] + 4 * (at % 16) + at % 64 // 16
    flat = (ids[:, None] * hk + head)[..., None] * words.shape[2] + word[:, None, :]
    old = (words.view(-1)[flat] >> shift) & 15
    words.view(-1).scatter_add_(0, flat.view(-1), ((vcode.int() - old) << shift).view(-1))
    # and back
    kv = []
    held = _k_codes(words[ids[:, None, None], head[:, None],
                          (slot * (d // 8))[:, None, None] + key].view(torch.uint8))
    kv.append(held)
    kv.append((words.view(-1)[flat] >> shift) & 15)
    for part in (0, 1):
        prm = words[ids[:, None], head, (page * (d // 4) + page * part + slot)[:, None]]
        prm = prm[..., None].view(torch.bfloat16).float()
        kv[part] = (prm[..., :1] + prm[..., 1:] * kv[part].float()).to(s["type"])
    return {"q": q, "k": kv[0], "v": kv[1]}


def _plain_attend(s):
    c = s["case"]
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    k, v = _plain_cached(s["cache"], s["pages"], c["page"], d)
    batch, most, i = c["batch"], s["max_q"], torch.arange(s["max_q"], device=DEV)
    j = torch.arange(k.shape[2], device=DEV)
    begin, end = s["offs"][:-1, None], s["offs"][1:, None]
    row = (begin + i).clamp(max=s["total"] - 1)                    # [batch, max_q]
    q = s["q"].float()[row].view(batch, most, hk, h // hk, d).permute(0, 2, 3, 1, 4)
    q = q.reshape(batch, hk, -1, d) * d ** -0.5
    p = (s["lens"][:, None] - (end - begin) + i)[..., None]        # [batch, max_q, 1]
    sees = j <= p
    if c["window"]:
        sees &= (j > p - c["window"]) | (j < c["sinks"])
    live = j < s["lens"][:, None]                                  # [batch, position]
    k = torch.where(live[:, None, :, None], k, 0.0)
    v = torch.where(live[:, None, :, None], v, 0.0)
    x = (q @ k.transpose(-1, -2).contiguous()).view(batch, hk, h // hk, most, -1)
    x.masked_fill_(~(sees & live[:, None])[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(torch.where(top == -math.inf, 0.0, top)))
    total = x.sum(-1, keepdim=True)
    out = x.view(batch, hk, -1, j.numel()) @ v
    out = out.view(batch, hk, h // hk, most, d) / torch.where(total == 0, 1.0, total)
    seq, _ = _places(s)
    at = torch.arange(s["total"], device=DEV) - s["offs"][seq]
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(batch, most, h, d)[seq, at].to(s["type"])}


# -- the framework's calls ---------------------------------------------------------
def _dtype(P, s):
    return {"bf16": P.IFQ_TYPE_BF16, "f16": P.IFQ_TYPE_F16, "f32": P.IFQ_TYPE_F32}[
        s["case"]["type"]]


def _plan(P, s):
    """What a program keeps between calls: the descriptor and the workspace."""
    c, op = s["case"], s["op"]
    ws = 0
    if op == "quantize":
        desc = P.f8_quant_desc(c["rows"], c["k"], _dtype(P, s), block_rows=c["block_rows"],
                               ld_codes=-(-c["k"] // 16) * 16)
    elif op == "product":
        desc = P.f8_matmul_desc(c["m"], c["n"], c["k"], _dtype(P, s))
        ws = P.ifq_f8_matmul_workspace_bytes(desc)
    else:
        more = {}
        if op == "append":
            row = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
            more = dict(q_stride=row, k_stride=row, v_stride=row, rot_dim=c["rot"],
                        rot_adjacent=c["adjacent"], rot_len=s["cos"].shape[0])
        else:
            more = dict(scale=c["dim"] ** -0.5, causal=True, window=c["window"],
                        sinks=c["sinks"])
        desc = P.kv_desc(c["batch"], s["total"], s["max_q"], c["len_max"], c["heads"],
                         c["kv_heads"], c["dim"], c["page"], s["cache"].shape[0],
                         s["pages"].shape[1], _dtype(P, s), **more)
        if op == "attend":
            ws = P.ifq_kv_attention_workspace_bytes(desc)
    return desc, torch.zeros(ws, dtype=torch.uint8, device=DEV) if ws else None


def _own(s):
    import paper_1911_08076_amd as P
    if "plan" not in s:
        s["plan"] = _plan(P, s)
    desc, ws = s["plan"]
    c, op = s["case"], s["op"]
    if op == "quantize":
        kb, rb = -(-c["k"] // BLOCK), -(-c["rows"] // c["block_rows"])
        codes = torch.empty(c["rows"], -(-c["k"] // 16) * 16, dtype=F8, device=DEV)
        scales = torch.empty(kb, rb, device=DEV)
        P.ifq_f8_quantize(desc, s["x"], codes, scales)
        return {"codes": codes[:, :c["k"]], "scales": scales}
    if op == "product":
        y = torch.empty(c["m"], c["n"], dtype=s["type"], device=DEV)
        P.ifq_f8_matmul(desc, s["a"], s["sa"], s["w"], s["sw"], y, ws=ws)
        return {"y": y}
    if op == "append":
        q = torch.empty(s["q"].shape, dtype=s["type"], device=DEV)
        k = torch.empty(s["k"].shape, dtype=s["type"], device=DEV)
        v = torch.empty_like(k)
        P.ifq_kv_append(desc, s["q"], s["k"], s["v"], s["cos"], s["sin"], s["offs"], s["lens"],
                        s["pages"], s["cache"], q)
        P.ifq_kv_read(desc, s["offs"], s["lens"], s["pages"], s["cache"], k, v)
        return {"q": q, "k": k, "v": v}
    out = torch.empty_like(s["q"])
    P.ifq_kv_attention(desc, s["q"], s["offs"], s["lens"], s["pages"], s["cache"], out, ws=ws)
    return {"out": out}


def run(state):
    if own:
        return _own(state)
    return {"quantize": _plain_quantize, "product": _plain_product, "append": _plain_append,
            "attend": _plain_attend}[state["op"]](state)


# -- the operators' definitions in 64 bits -------------------------------------------
def _e4m3(x):
    """The nearest number of 4 exponent and 3 mantissa bits, ties to even; |x| <= 448."""
    e = torch.frexp(x)[1].clamp_min(-5).double() - 4     # 2^e is the spacing at x
    unit = torch.exp2(e)
    return torch.round(x / unit) * unit


def _bf16_way(x, up):
    """x in 64 bits rounded to 8 significant bits, up or down."""
    m, e = torch.frexp(x)
    m = torch.ceil(m * 256) if up else torch.floor(m * 256)
    return m * torch.exp2(e.double() - 8)


def _stored(x):
    """What a 4-bit row of x stands for."""
    off = _bf16_way(x.min(-1, keepdim=True).values, False)
    step = _bf16_way((x.max(-1, keepdim=True).values - off) / 15, True)
    code = torch.round((x - off) / torch.where(step == 0, 1.0, step)).clamp(0, 15)
    return off + step * code


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        x = s["x"].double()
        rows, k = x.shape
        br = case["block_rows"]
        scales = torch.empty(-(-k // BLOCK), -(-rows // br), dtype=torch.float64, device=DEV)
        codes = torch.empty_like(x)
        if br == 1:
            for b in range(scales.shape[0]):
                part = x[:, b * BLOCK:(b + 1) * BLOCK]
                top = part.abs().max(1).values
                scales[b] = top / F8_MAX
                codes[:, b * BLOCK:(b + 1) * BLOCK] = _e4m3(part * F8_MAX / top[:, None])
        else:
            for b in range(scales.shape[0]):
                for r in range(scales.shape[1]):
                    part = x[r * br:(r + 1) * br, b * BLOCK:(b + 1) * BLOCK]
                    top = part.abs().max()
                    scales[b, r] = top / F8_MAX
                    codes[r * br:(r + 1) * br, b * BLOCK:(b + 1) * BLOCK] = _e4m3(
                        part * F8_MAX / top)
        return {"codes": codes, "scales": scales}
    if case["op"] == "product":
        y = torch.zeros(case["m"], case["n"], dtype=torch.float64, device=DEV)
        for b in range(s["sa"].shape[0]):
            at = slice(b * BLOCK, min(case["k"], (b + 1) * BLOCK))
            a = s["a"][:, at].double() * s["sa"][b].double()[:, None]
            w = s["w"][:, at].double()
            w *= s["sw"][b].double()[torch.arange(case["n"], device=DEV) // BLOCK][:, None]
            y += a @ w.t().contiguous()
        return {"y": y}
    offs, lens = s["offs"].tolist(), s["lens"].tolist()
    if case["op"] == "append":
        out = {"q": [], "k": [], "v": []}
        r = case["rot"]
        for b in range(case["batch"]):
            at = slice(offs[b], offs[b + 1])
            n = offs[b + 1] - offs[b]
            pos = torch.arange(lens[b] - n, lens[b], device=DEV)
            turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]
            for name in ("q", "k"):
                x = s[name][at].double().clone()
                pair = (slice(0, r, 2), slice(1, r, 2)) if case["adjacent"] else (
                    slice(0, r // 2), slice(r // 2, r))
                z = torch.complex(x[..., pair[0]].contiguous(),
                                  x[..., pair[1]].contiguous()) * turn
                x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
                out[name].append(x if name == "q" else _stored(x))
            out["v"].append(_stored(s["v"][at].double()))
        return {name: torch.cat(x) for name, x in out.items()}
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(s["total"], h, d, dtype=torch.float64, device=DEV)
    # where the code of (token of a page, dim) lies: byte, and its low or high half
    tok, dim = torch.arange(page, device=DEV)[:, None], torch.arange(d, device=DEV)
    kn = dim % 8 // 2 + 4 * (dim % 2)
    kat = tok * (d // 2) + 4 * (dim // 8) + kn // 2
    e = tok % 32 // 16 * 4 + tok % 4
    vn = e // 2 + 4 * (e % 2)
    vat = page * d // 2 + tok // 32 * (16 * d) + dim // 64 * 1024 + (
        tok % 16 // 4 * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + vn // 2
    for b in range(case["batch"]):
        n, first, last = lens[b], offs[b], offs[b + 1]
        if n == 0:
            continue
        ids = s["pages"][b, :-(-n // page)].long()
        pos = n - (last - first) + torch.arange(last - first, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)
        sees = j <= pos
        if case["window"]:
            sees &= (j > pos - case["window"]) | (j < case["sinks"])
        for g in range(hk):
            held = s["cache"][ids, g]                              # [pages, bytes]
            rows = []
            for at, half, part in ((kat, kn, 0), (vat, vn, 1)):
                code = (held[:, at.expand(page, d).reshape(-1)].view(-1, page, d)
                        >> (4 * (half % 2)).to(torch.uint8)) & 15
                prm = held[:, page * d + 4 * page * part:page * d + 4 * page * (part + 1)]
                prm = prm.contiguous().view(torch.bfloat16).view(-1, page, 2).double()
                rows.append((prm[..., :1] + prm[..., 1:] * code.double()).view(-1, d)[:n])
            for i in range(g * (h // hk), (g + 1) * (h // hk)):
                x = s["q"][first:last, i].double() @ rows[0].t().contiguous() / math.sqrt(d)
                x = x.masked_fill(~sees, -math.inf)
                x = torch.softmax(x, -1).nan_to_num(0.0)           # a row that sees nothing
                out[first:last, i] = x @ rows[1]
    return {"out": out}
