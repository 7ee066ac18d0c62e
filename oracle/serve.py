"""The operators for serving language models, plainly: 8-bit float codes with
a scale per block of 128 and their product, the paged cache of 4-bit codes, and
attention over it. NumPy on the CPU; sums and softmax in 64 bits, and fp32 step
by step where the operator's definition is in fp32.
"""
import numpy as np

F = np.float32
BLOCK = 128


# -- 8-bit floats ------------------------------------------------------------------
def _e4m3_table():
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (e == 15 and m == 7) else (
            m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v[c] = -x if c & 128 else x
    return v


E4M3 = _e4m3_table()


def e4m3_codes(x):
    """Nearest codes of |x| <= 448, ties to the even code."""
    x = np.asarray(x, np.float64)
    pos = E4M3[:127]                                  # 0 .. 448, increasing
    a = np.abs(x)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    c = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def f8_quantize(x, block_rows=1):
    """Codes [rows][k] and scales [ceil(k/128)][ceil(rows/block_rows)]."""
    x = np.asarray(x, F)
    rows, k = x.shape
    kb, rb = -(-k // BLOCK), -(-rows // block_rows)
    codes = np.zeros((rows, k), np.uint8)
    scales = np.zeros((kb, rb), F)
    for b in range(kb):
        for r in range(rb):
            at = np.s_[r * block_rows:(r + 1) * block_rows, b * BLOCK:(b + 1) * BLOCK]
            part = x[at]
            if not np.isfinite(part).all():
                scales[b, r] = np.nan
                continue
            top = max(np.abs(part).max(), F(2.0 ** -96))
            scales[b, r] = top / F(448)
            q = np.clip((part * F(0.875)) / (top * F(2.0 ** -9)), F(-448), F(448))
            codes[at] = e4m3_codes(q)
    return codes, scales


def f8_matmul(a, sa, w, sw):
    """Product, and the sum of magnitudes that rounding errors go by."""
    k, n = a.shape[1], w.shape[0]
    b = np.arange(k) // BLOCK
    fa = E4M3[a] * sa.astype(np.float64).T[:, b]
    fw = E4M3[w] * sw.astype(np.float64).T[np.arange(n) // BLOCK][:, b]
    return fa @ fw.T, np.abs(fa) @ np.abs(fw).T


# -- rows of 4-bit codes --------------------------------------------------------------
def _f32_of(word):
    return np.asarray(word, np.uint32).view(F)


def row_codes(x):
    """Word (offset, step) and codes of the rows (last axis) of x in fp32."""
    x = np.ascontiguousarray(x, F)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        # -0 is below 0, wherever in the row it is
        lo = np.where((lo == 0) & ((x == 0) & np.signbit(x)).any(-1), F(-0.0), lo)
        o = np.ascontiguousarray(lo).view(np.uint32)
        o = np.where(o >> 31, o + np.uint32(0xFFFF), o) & np.uint32(0xFFFF0000)
        off = _f32_of(o)
        t = np.ascontiguousarray((hi - off) / F(15)).view(np.uint32)
        t = (t + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)
        step = _f32_of(t)
        fine = np.isfinite(x).all(-1) & np.isfinite(off) & np.isfinite(step)
        c = np.rint((x - off[..., None]) / step[..., None])
        c = np.where((step[..., None] == 0) | ~fine[..., None], F(0), c)
    word = np.where(fine, (o >> 16) | t, np.uint32(0x7FC0)).astype(np.uint32)
    return word, np.clip(c, 0, 15).astype(np.uint8)


def row_values(word, codes):
    """What rows stand for, in fp32."""
    off, step = _f32_of(word << np.uint32(16)), _f32_of(word & np.uint32(0xFFFF0000))
    return off[..., None] + step[..., None] * codes.astype(F)


class Page:
    """Views of one head of one page (bytes of page_tokens * (dim + 8))."""

    def __init__(self, held, tokens, dim):
        self.tokens, self.dim = tokens, dim
        half = tokens * dim // 2
        self.k = held[:half].reshape(tokens, dim // 2)
        self.v = held[half:2 * half].view(np.uint32).reshape(tokens // 32, dim // 64, 4, 16, 4)
        self.kw = held[2 * half:2 * half + 4 * tokens].view(np.uint32)
        self.vw = held[2 * half + 4 * tokens:].view(np.uint32)

    @staticmethod
    def _v_place(t, d):
        e = 4 * (t % 32 // 16) + t % 4
        return (t // 32, d // 64, t % 16 // 4, d % 16, d % 64 // 16), 4 * (e // 2 + 4 * (e % 2))

    def put(self, t, kword, kcode, vword, vcode):
        self.kw[t], self.vw[t] = kword, vword
        for d in range(self.dim):
            nib = d % 8 // 2 + 4 * (d % 2)
            byte = d // 8 * 4 + nib // 2
            sh = 4 * (nib % 2)
            self.k[t, byte] = (int(self.k[t, byte]) & ~(15 << sh) & 255) | int(kcode[d]) << sh
            at, sh = self._v_place(t, d)
            self.v[at] = (int(self.v[at]) & ~(15 << sh)) & 0xFFFFFFFF | int(vcode[d]) << sh

    def codes(self):
        """Key and value codes [tokens][dim]."""
        d = np.arange(self.dim)
        nib = d % 8 // 2 + 4 * (d % 2)
        k = (self.k[:, d // 8 * 4 + nib // 2] >> (4 * (nib % 2)).astype(np.uint8)) & 15
        at, sh = self._v_place(np.arange(self.tokens)[:, None], d[None])
        return k, ((self.v[at] >> sh.astype(np.uint32)) & 15).astype(np.uint8)


def head_of(cache, page, head, tokens, dim):
    """Views of a head of a page of the byte array [pages][kv_heads][tokens*(dim+8)]."""
    return Page(cache[page, head], tokens, dim)


def rotate(x, cosines, sines, adjacent):
    """x [.., dim] in fp32, tables of its position [.., rot/2]."""
    x = np.array(x, F)
    half = cosines.shape[-1]
    a, b = (np.s_[..., 0:2 * half:2], np.s_[..., 1:2 * half:2]) if adjacent else (
        np.s_[..., :half], np.s_[..., half:2 * half])
    u, v = x[a].copy(), x[b].copy()
    x[a] = u * cosines - v * sines
    x[b] = u * sines + v * cosines
    return x


# -- attention ------------------------------------------------------------------------
def attention(q, kw, kc, vw, vc, pos, scale, window=0, sinks=0):
    """One head: q [n][dim] at positions pos [n], rows (words and codes) of its
    sequence. Returns the output, and for each element a bound on the error of a
    computation in fp32 from the rows' offsets, steps and codes with the factors
    p * step in 16 bits.

    A score's error: the products q * (16 + c) and the sum of q, each of dim
    terms with partial sums below 32 * sum|q|, are off by at most
    dim * 2^-24 * 32 * sum|q| relative to step * scale, and the combination with
    the offset by a few 2^-24 of its terms. A factor's relative error is the
    score's (times ln 2 and log2 e, which cancel) and 2^-16.
    """
    n, dim = q.shape
    q = q.astype(np.float64)
    ko, kt = _f32_of(kw << np.uint32(16)), _f32_of(kw & np.uint32(0xFFFF0000))
    vo, vt = _f32_of(vw << np.uint32(16)), _f32_of(vw & np.uint32(0xFFFF0000))
    ko, kt, vo, vt = (a.astype(np.float64) for a in (ko, kt, vo, vt))
    out, bound = np.zeros((n, dim)), np.zeros((n, dim))
    k = ko[:, None] + kt[:, None] * kc
    v = vo[:, None] + vt[:, None] * vc
    size = np.abs(vt[:, None] * (vc - 8.0)) + np.abs(vo + 8 * vt)[:, None]
    eps = 2.0 ** -24
    for i in range(n):
        j = np.arange(len(kw))
        sees = j <= pos[i]
        if window:
            sees &= (j > pos[i] - window) | (j < sinks)
        if not sees.any():
            continue
        s = scale * (k[sees] @ q[i])
        p = np.exp(s - s.max())
        p /= p.sum()
        out[i] = p @ v[sees]
        qa = np.abs(q[i]).sum()
        ds = abs(scale) * (kt[sees] * dim * 32 * qa * eps +
                           8 * eps * (np.abs(ko) + 8 * kt)[sees] * qa) + 8 * eps * np.abs(s)
        ds = ds + ds.max()                       # its own, and the normalizing sum's
        rel = np.expm1(ds) + 2.0 ** -15 + (len(p) + 8) * eps
        # the sums of factors * (16 + c) are at most 31 times that of the factors
        held = 32 * eps * (len(p) / 16 + 4) * (p @ vt[sees])
        bound[i] = (p * rel) @ size[sees] + rel.max() * np.abs(out[i]) + held
    return out, bound
