"""Verification where the logits' magnitude hides the logarithm of their sum: rows
that a mask of the type's lowest value covers whole, ties far from 0.

Log-probabilities are (z - m) - log sum exp(z - m) here: m + log sum itself, as
rollout_ref.log_softmax has it, is m for these rows in any floating-point type."""
import numpy as np
import pytest
import torch

from gpu_common import say
from test_gpu_verify import DT, make, run


def log_softmax(row):
    z = np.asarray(row, np.longdouble)
    d = z - z.max()
    return d - np.log(np.exp(d).sum())


def verify(target, ids, u, draft):
    """Kept counts, tokens and log-probs, and how near a uniform came to a border: a
    test's relative to p, a draw's to the rows' whole masses (1)."""
    B, D = ids.shape
    kept = np.zeros(B, np.int32)
    out = np.full((B, D + 1), -1, np.int32)
    logp = np.zeros((B, D + 1))
    near = np.full(B, np.inf)
    for b in range(B):
        for i in range(D + 1):
            lp = log_softmax(target[b, i])
            mass = p = np.exp(lp)
            if i < D:
                x, q = ids[b, i], np.zeros(len(p), np.longdouble)
                if draft is None:
                    q[x] = 1
                else:
                    q = np.exp(log_softmax(draft[b, i]))
                if u[b, i] * q[x] != p[x]:
                    near[b] = min(near[b], abs(u[b, i] * q[x] - p[x]) / max(u[b, i] * q[x], p[x]))
                if u[b, i] * q[x] < p[x]:
                    out[b, i], logp[b, i] = x, lp[x]
                    continue
                mass = np.maximum(p - q, 0)
                if mass.sum() == 0:  # (a drafted token without mass in equal rows)
                    mass = p
            kept[b] = i
            below = np.cumsum(mass)
            t = u[b, D] * below[-1]
            near[b] = min(near[b], np.abs(below - t).min())
            out[b, i] = (below <= t).sum()
            logp[b, i] = lp[out[b, i]]
            break
    return kept, out, logp, near


def check(t, name):
    out = run(t)
    torch.cuda.synchronize()
    n = {k: None if t[k] is None else t[k].numpy() if k == "ids" else t[k].double().numpy()
         for k in ("z", "y", "ids", "u")}
    kept, ids, logp, near = verify(n["z"], n["ids"], n["u"], n["y"])
    say("%s: %d sequences, %d kept, nearest border %.1e" % (name, len(kept), kept.sum(), near.min()))
    assert (near > 1e-12).all()
    assert np.array_equal(out["accepted"].cpu().numpy(), kept)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    # one rounding to fp32 of a value good to 1e-12
    off = np.abs(out["logp"].double().cpu().numpy() - logp)
    assert (off <= np.abs(logp) * 2.0 ** -24 + 1e-11).all()
    return kept


def test_ties_share_the_mass():
    for low in (np.finfo(np.float32).min, 1e17, -3e4, 0.0):
        assert np.abs(log_softmax([low] * 4) + np.log(4)).max() < 1e-15


# (the last: so many bf16 logits that their exponentials come from a table)
SIZES = [(24, 3, 4), (24, 3, 400), (6, 2, 32003), (2, 2, 151936), (40, 2, 60000)]


@pytest.mark.gpu
@pytest.mark.parametrize("B,D,V", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
def test_rows_of_the_lowest_value(B, D, V, dtype, certain):
    """All actions masked by the type's lowest value: a uniform distribution."""
    t = make(B, D, V, dtype, certain, near=0.3, seed=30)
    low = torch.finfo(DT[dtype]).min
    t["z"][:B // 2] = low
    t["z"][B // 2:, 1] = low
    t["u"][:B // 4, 0] = 0.25 / V  # (some are kept)
    if not certain:
        t["y"][::2, 0] = low
        t["y"][:, 1] = low
    kept = check(t, "lowest %d %d %d" % (B, D, V))
    if B >= 24:
        assert (kept < D).any() and (kept > 0).any()


@pytest.mark.gpu
@pytest.mark.parametrize("B,D,V", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [1e17, -1e17, 3e38, 30000.0, 700.0, -700.0])
def test_ties_far_from_zero(B, D, V, dtype, value):
    """Few or many actions of one far value; the others of no mass beside them."""
    t = make(B, D, V, dtype, near=0.3, seed=31)
    g = np.random.default_rng(32)
    for x in (t["z"], t["y"]):
        some = torch.from_numpy(g.random(tuple(x.shape)) < 0.6)
        some[..., 1] = True
        x[some] = value
        x[~some] = float("-inf") if value < 0 else -1.0
    t["ids"][:, 0] = 1
    check(t, "ties %g" % value)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_rows_beside_near_ones(dtype):
    """A target far from 0 with a drafter that is not, and the other way round."""
    t = make(30, 2, 5000, dtype, near=0.3, seed=33)
    t["z"][:10, 0] = 1e17
    t["y"][10:20, 0] = -1e17
    t["z"][20:, 1, :2500] = torch.finfo(DT[dtype]).min
    t["y"][20:, 1] = torch.finfo(DT[dtype]).min
    check(t, "far beside near")
