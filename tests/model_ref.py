"""Plain 64-bit forms of the calls around the rows of logits (token embeddings,
low-rank adapters, beams), written from their definitions (numpy, no library
code), with bounds on what 32-bit sums may differ from them."""
import numpy as np

# half a step of a rounding, relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
# a 32-bit addition on the matrix cores is off by a unit in the last place at most, whichever
# way it rounds
ULP = 2.0 ** -23


def embed(table, ids, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for n, i in enumerate(ids):
        if i >= 0 and i < table.shape[0]:
            out[n] = scale * table[i]
        elif i != -1:
            out[n] = np.nan
    return out


def embed_grads(dy, ids, V, scale):
    """(gradient, bound of its sums): count additions, each off by half a step of
    at most the sum of magnitudes, and the multiplication."""
    d, mag, count = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1])), np.zeros((V, 1))
    for n, i in enumerate(ids):
        if 0 <= i < V:
            d[i] += dy[n]
            mag[i] += np.abs(dy[n])
            count[i] += 1
    return d * scale, (count + 2) * 2.0 ** -24 * mag * abs(scale)


def tokens_of(ids, G):
    return [np.flatnonzero(ids == g) for g in range(G)]


def _product(p, q, off_p=None):
    """p @ q of which p is off by off_p: (product, bound)."""
    mag = np.abs(p) @ np.abs(q)
    off = (p.shape[1] + 1) * ULP * mag
    return p @ q, off if off_p is None else off + off_p @ np.abs(q)


def _passed(t, off, scale, half):
    """s t as the second product takes it: a multiplication and parts of 16 bits that hold
    `half` of it."""
    return scale * t, abs(scale) * (off + np.abs(t) * (2.0 ** -24 + half))


def _half(kind, out):
    """What is lost of t and u on their way: two bf16 parts for bf16 results, three for
    fp32 ones of bf16 operands, nothing in fp32."""
    return 0.0 if kind == "f32" else 2.0 ** -17 if out == "bf16" else 2.0 ** -25


def adapters(y, x, a, b, ids, scales, kind, ykind):
    """(out, bound, low, bound)."""
    G, r = a.shape[:2]
    out, off = y.copy(), np.zeros_like(y)
    low, low_off = np.zeros((len(ids), r)), np.zeros((len(ids), r))
    for g, at in enumerate(tokens_of(ids, G)):
        if not len(at):
            continue
        t, t_off = _product(x[at], a[g].T)
        low[at], low_off[at] = t, t_off
        st, st_off = _passed(t, t_off, scales[g], _half(kind, ykind))
        d, d_off = _product(st, b[g], st_off)
        out[at] += d
        off[at] = d_off + (3 * r + 1) * ULP * (np.abs(y[at]) + np.abs(st) @ np.abs(b[g]))
    bad = (ids < -1) | (ids >= G)
    out[bad] = np.nan
    low[bad] = np.nan
    return out, off, low, low_off


def adapter_grads(dy, x, a, b, ids, scales, kind, ykind, low=None, dx_shared=None):
    """dict of (value, bound)."""
    G, r, H = a.shape
    O = b.shape[2]
    dx = np.zeros((len(ids), H)) if dx_shared is None else dx_shared.copy()
    dx_off = np.zeros_like(dx)
    da, da_off = np.zeros((G, r, H)), np.zeros((G, r, H))
    db, db_off = np.zeros((G, r, O)), np.zeros((G, r, O))
    for g, at in enumerate(tokens_of(ids, G)):
        if not len(at):
            continue
        s = scales[g]
        t, t_off = _product(x[at], a[g].T) if low is None else (low[at], np.zeros((len(at), r)))
        u, u_off = _product(dy[at], b[g].T)
        su, su_off = _passed(u, u_off, s, _half(kind, kind))
        d, d_off = _product(su, a[g], su_off)
        dx_off[at] = d_off + (3 * r + 1) * ULP * (np.abs(dx[at]) + np.abs(su) @ np.abs(a[g]))
        dx[at] += d
        su, su_off = _passed(u, u_off, s, _half(kind, "f32"))
        # (three parts of each are added apart)
        da[g], da_off[g] = su.T @ x[at], (
            su_off.T @ np.abs(x[at]) + (3 * len(at) + 65) * ULP * (np.abs(su).T @ np.abs(x[at])))
        st, st_off = _passed(t, t_off, s, _half(ykind, "f32"))
        db[g], db_off[g] = st.T @ dy[at], (
            st_off.T @ np.abs(dy[at]) + (3 * len(at) + 65) * ULP * (np.abs(st).T @ np.abs(dy[at])))
    bad = (ids < -1) | (ids >= G)
    dx[bad] = np.nan
    return {"da": (da, da_off), "db": (db, db_off), "dx": (dx, dx_off)}


def beams(z, scores, k, finished=None):
    """(scores, parents, ids, how near two neighbours of different beams come), per group;
    z [B, W, V]."""
    B, W, V = z.shape
    out = np.full((B, k), -np.inf)
    parents, ids = np.full((B, k), -1, np.int32), np.full((B, k), -1, np.int32)
    near = np.inf
    for b in range(B):
        found, bad = [], False
        for w in range(W):
            s = float(scores[b, w])
            if np.isnan(s) or s == np.inf:
                bad = True
                continue
            if s == -np.inf:
                continue
            if finished is not None and finished[b, w]:
                found.append((np.longdouble(s), w, -1))
                continue
            row = z[b, w].astype(np.longdouble)
            if np.isnan(row).any() or (row == np.inf).any():
                bad = True
                continue
            m = row.max()
            if m == -np.inf:
                continue
            logp = row - m - np.log(np.exp(row - m).sum())
            # (the k + 1 best of a row, ties to the lower token, are enough)
            order = np.lexsort((np.arange(V), -row))[:k + 1]
            found += [(s + logp[v], w, int(v)) for v in order if row[v] > -np.inf]
        if bad:
            out[b] = np.nan
            continue
        found.sort(key=lambda c: (-c[0], c[1], c[2]))
        for c, d in zip(found[:k], found[1:k + 1]):
            if c[1] != d[1]:
                near = min(near, float(c[0] - d[0]))
        for j, (s, w, v) in enumerate(found[:k]):
            out[b, j], parents[b, j], ids[b, j] = s, w, v
    return out, parents, ids, near


def reorder(states, parents, W):
    """states [B * W, ...] numpy of any type."""
    B, k = parents.shape
    out = np.zeros((B * k,) + states.shape[1:], states.dtype)
    for b in range(B):
        for j in range(k):
            if 0 <= parents[b, j] < W:
                out[b * k + j] = states[b * W + parents[b, j]]
    return out
