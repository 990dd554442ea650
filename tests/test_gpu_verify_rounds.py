"""Verification whose rows are summed in several rounds of positions, up to 2,048
sequences (whose rows each round counts) and beyond: some sequences against the
64-bit form, all against calls of few sequences."""
import numpy as np
import pytest
import torch

import paper_2606_24143_amd as opd
import rollout_ref as ref
from gpu_common import DEV, say
from test_gpu_verify import DT

pytestmark = pytest.mark.gpu


def make(B, D, V, dtype, certain, seed, near):
    """Rows on the GPU, drafts near the target, ragged, some sequences masked and
    some ended by a row without a distribution."""
    g = torch.Generator(DEV).manual_seed(seed)
    ld = (V + 7) // 8 * 8
    z = torch.full((B * (D + 1), ld), float("nan"), dtype=DT[dtype], device=DEV)
    y = torch.full((B * D, ld), float("nan"), dtype=DT[dtype], device=DEV)
    ids = torch.empty(B, D, dtype=torch.int32, device=DEV)
    for b in range(B):
        row = torch.randn(D + 1, V, device=DEV, generator=g) * 2
        z[b * (D + 1):(b + 1) * (D + 1), :V] = row
        q = row[:D] + near * torch.randn(D, V, device=DEV, generator=g)
        y[b * D:(b + 1) * D, :V] = q
        u = torch.rand(D, V, device=DEV, generator=g).clamp_(1e-30, 1 - 2.0 ** -24)
        ids[b] = torch.argmax(q - torch.log(-torch.log(u)), 1)
    if certain:  # likely drafts, so that later rounds have rows
        at = torch.arange(B * (D + 1), device=DEV).view(B, D + 1)[:, :D].reshape(-1)
        z[at, ids.view(-1).long()] = 14.0
    t = dict(z=z, y=None if certain else y, ids=ids,
             u=torch.rand(B, D + 1, device=DEV, generator=g),
             lens=torch.randint(0, D + 1, (B,), device=DEV, generator=g, dtype=torch.int32),
             mask=torch.rand(B, device=DEV, generator=g) < 0.9)
    t["lens"][::3] = D
    for b in range(5, B, 11):  # a position of each round, over the sequences
        z[b * (D + 1) + b % (D + 1), V // 2] = float("nan")
    return t


def call(t, V, D, lo, hi):
    return opd.verify_drafts(
        t["z"][lo * (D + 1):hi * (D + 1), :V], t["ids"][lo:hi], t["u"][lo:hi],
        draft_logits=None if t["y"] is None else t["y"][lo * D:hi * D, :V],
        draft_lens=t["lens"][lo:hi], mask=t["mask"][lo:hi])


def close(a, b, tol):
    """fp32 log-probs of two evaluations, each good to 1e-12 before its rounding."""
    a, b = np.float64(a), np.float64(b)
    f = np.isfinite(b)
    assert np.array_equal(a[~f], b[~f], equal_nan=True)
    assert (np.abs(a - b)[f] <= tol * np.abs(b)[f] + 1e-11).all()


def rounds(B, D, V, drafts):
    """The launches that sum rows: 2^25 elements of the first positions, then twice
    as many each."""
    many, pos, n = (1 << 25) // (drafts * B * V) + 1, 0, 0
    while pos <= D:
        pos, many, n = pos + many, 2 * many, n + 1
    return n


@pytest.mark.parametrize("B,D,V,certain,least", [
    (64, 8, 151936, False, 3),      # 2, 4 and 3 positions
    (120, 7, 151936, False, 3),     # 1, 2, 4 and 1
    (2048, 8, 4099, False, 3),      # the most that are counted
    (1500, 12, 9000, True, 3),
    (2049, 4, 20001, False, 3),     # not counted; five parts to a row
    (2500, 6, 7003, True, 3),       # not counted; certain drafts
])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounds(B, D, V, certain, least, dtype):
    assert rounds(B, D, V, 1 if certain else 2) >= least
    t = make(B, D, V, dtype, certain, B + D, 0.1)
    out = call(t, V, D, 0, B)
    step = 8 if B < 1000 else 100
    parts = [call(t, V, D, lo, min(lo + step, B)) for lo in range(0, B, step)]
    few = {k: torch.cat([p[k] for p in parts]) for k in out}
    assert torch.equal(out["accepted"], few["accepted"])
    assert torch.equal(out["ids"], few["ids"])
    close(out["logp"].cpu().numpy(), few["logp"].cpu().numpy(), 2.0 ** -23)
    kept = out["accepted"].cpu().numpy()
    say("rounds %d x %d x %d: kept per sequence %s" % (B, D, V, np.bincount(kept)))
    assert (np.bincount(kept, minlength=D + 1) > 0).all()  # sequences end everywhere
    some = np.arange(0, B, max(B // 12, 1))
    n = lambda x: x.double().cpu().numpy() if x.is_floating_point() else x.cpu().numpy()
    at = torch.as_tensor(some, device=DEV)
    a, ids, logp, near = ref.verify(
        n(t["z"].view(B, D + 1, -1)[at][..., :V]), n(t["ids"][at]), n(t["u"][at]),
        None if certain else n(t["y"].view(B, D, -1)[at][..., :V]), n(t["lens"][at]),
        n(t["mask"][at]))
    assert (near > 1e-12).all()
    assert np.array_equal(kept[some], a)
    assert np.array_equal(n(out["ids"][at]), ids)
    close(n(out["logp"][at]), logp, 2.0 ** -24)
