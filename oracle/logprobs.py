"""Log probabilities of given tokens, entropy and top tokens of rows of logits,
plainly. NumPy on the CPU, in 64 bits, with bounds on the error of a computation
in fp32."""
import numpy as np

EPS = 2.0 ** -24


def logprobs(x, tokens, top, scale):
    """x [rows][n] in 64 bits. Returns logprob, entropy, top logprobs, top tokens, and
    bounds on the first three.

    A term 2^t with t = c (x - M) in fp32: c is off by two roundings, the difference and
    the product by one each, so t is off by 4 EPS |t| and the term by 4 EPS |z| and an ulp
    of the exponential. Sums over runs of 32, turns of 2048 and lanes: an addition and
    two products of EPS each for every step of the longest chain.
    """
    rows, n = x.shape
    steps = 32 + 4 * (n / 2048 + 1) + 64
    lp, h = np.zeros(rows), np.zeros(rows)
    best, at = np.zeros((rows, top)), np.zeros((rows, top), np.int32)
    blp, bh, bbest = np.zeros(rows), np.zeros(rows), np.zeros((rows, top))
    for r in range(rows):
        v, t = x[r], int(tokens[r])
        if np.isnan(v).any() or (v == np.inf).any():
            lp[r], h[r], best[r], at[r] = np.nan, np.nan, np.nan, -1
            if t < 0:
                lp[r] = 0
            continue
        order = np.argsort(-v, kind="stable")[:top]
        at[r] = order
        m = v.max()
        if m == -np.inf:
            best[r], lp[r] = -np.inf, -np.inf
        else:
            z = scale * (v - m)
            p = np.exp(z)
            s = p.sum()
            log = np.log(s)
            p /= s
            seen = p > 0
            zp, pp = np.abs(z[seen]), p[seen]
            h[r] = log + (pp * zp).sum()
            ds = (pp * (4 * zp + 2)).sum() * EPS + steps * EPS
            dlog = ds + 4 * EPS * abs(log)
            bh[r] = dlog + (pp * zp * (4 * zp + 8 + steps)).sum() * EPS + (
                (pp * zp).sum() * (ds + 4 * EPS)) + 4 * EPS * h[r]
            lp[r] = z[t] - log if 0 <= t < n else 0
            best[r] = z[order] - log
            with np.errstate(invalid="ignore"):
                bound = dlog + 4 * EPS * np.abs(z) + 2 * EPS * np.abs(z - log)
            blp[r] = bound[t] if 0 <= t < n else 0
            bbest[r] = bound[order]
        if t < 0:
            lp[r] = 0
        elif t >= n:
            lp[r] = np.nan
    return (lp, h, best, at), (blp, bh, bbest)
