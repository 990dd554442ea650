"""Plain 64-bit forms of blockwise quantisation, the head's product and the
verification of drafted tokens, written from their definitions (numpy, no
library code)."""
import math

import numpy as np

TOP = 448.0
BLOCK = 128


def blocks(n, size):
    return (n + size - 1) // size


def nearest_e4m3(v):
    """The e4m3 value nearest to v: four significant bits, exponents from -6,
    ties to the even one; |v| is at most 448 (1 + 2^-23) here."""
    v = np.asarray(v, np.float64)
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    step = np.exp2(e - 3)
    return np.clip(np.round(v / step) * step, -TOP, TOP)


def quantize(x, rows, e8m0):
    """(values of q, scales) of x (float32 or wider array), float64; a block that
    is not finite is NaN."""
    x = np.asarray(x, np.float64)
    N, H = x.shape
    q = np.zeros((N, H))
    s = np.zeros((blocks(N, rows), blocks(H, BLOCK)))
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = np.s_[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            a = np.abs(x[at]).max()
            if not np.isfinite(a):
                s[i, j] = q[at] = np.nan
                continue
            if e8m0:
                m, e = math.frexp(a)  # a = m 2^e; 448 = 0.875 * 2^9
                e = max(e - 9 + (m > 0.875), -127) if a > 0 else -127
                s[i, j] = 2.0 ** e
            else:
                # (both the scale and the quotient are 32-bit numbers by definition)
                s[i, j] = max(np.float32(a / TOP), np.float32(2.0 ** -126))
            q[at] = nearest_e4m3(np.float32(x[at] / s[i, j]))
    return q, s


def head(x, sx, w, sw):
    """(logits, sum of the terms' magnitudes), from the values that x and w hold."""
    wide = np.repeat(sx, BLOCK, 1)[:, :x.shape[1]] * x
    head_ = np.repeat(np.repeat(sw, BLOCK, 1)[:, :w.shape[1]], BLOCK, 0)[:w.shape[0]] * w
    return wide @ head_.T, np.abs(wide) @ np.abs(head_).T


def log_softmax(row):
    """Log-probabilities of a row (long double), or None without a distribution."""
    z = np.asarray(row, np.longdouble)
    m = z.max()
    if not np.isfinite(m):
        return None
    with np.errstate(divide="ignore"):
        return z - (m + np.log(np.exp(z - m).sum()))


def verify(target, ids, u, draft=None, lens=None, mask=None):
    """Accepted counts, tokens, log-probs, and how near the nearest uniform came to
    a border, per sequence.  target [B, D + 1, V], draft [B, D, V]."""
    B, D = ids.shape
    V = target.shape[2]
    accepted = np.zeros(B, np.int32)
    out = np.full((B, D + 1), -1, np.int32)
    logp = np.zeros((B, D + 1))
    near = np.full(B, np.inf)
    for b in range(B):
        if mask is not None and not mask[b]:
            continue
        n = D if lens is None else int(lens[b])
        if n < 0 or n > D:
            logp[b, 0] = np.nan
            continue
        for i in range(n + 1):
            accepted[b] = i
            lp = log_softmax(target[b, i])
            bad = lp is None
            mass = None if bad else np.exp(lp)
            if not bad and i < n:
                x, ui = int(ids[b, i]), float(u[b, i])
                bad = not (0 <= x < V and 0.0 <= ui < 1.0)
                q = np.zeros(V, np.longdouble)
                if draft is not None:
                    lq = log_softmax(draft[b, i])
                    bad = bad or lq is None
                    if not bad:
                        q = np.exp(lq)
                elif not bad:
                    q[x] = 1.0
                if not bad:
                    if mass[x] > 0 or q[x] > 0:
                        near[b] = min(near[b], abs(ui * q[x] - mass[x]) / max(q[x], mass[x]))
                    if ui * q[x] < mass[x]:
                        out[b, i] = x
                        logp[b, i] = lp[x]
                        continue
                    mass = np.maximum(mass - q, 0)
            r = float(u[b, D])
            if bad or not 0.0 <= r < 1.0:
                logp[b, i] = np.nan
                break
            below = np.cumsum(mass)
            t = np.longdouble(r) * below[-1]
            j = int((below <= t).sum())
            if t > 0:
                near[b] = min(near[b], float(np.abs(below - t).min() / max(below[-1], 1e-300)))
            out[b, i] = j
            logp[b, i] = lp[j]
            break
    return accepted, out, logp, near
