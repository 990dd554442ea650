"""Verification of drafted tokens on the GPU against the 64-bit form.

Counts and tokens have to be equal, unless a uniform lies within 1e-12 of a border
(no case's does); log-probs are rounded once to fp32 from double precision."""
import numpy as np
import pytest
import torch

import paper_2606_24143_amd as opd
import rollout_ref as ref
from gpu_common import DEV, say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(B, D, V, dtype, certain=False, ragged=False, near=0.5, scale=2.0, seed=0):
    g = np.random.default_rng(seed + 31 * B + 7 * D + V)
    z = g.normal(0, scale, (B, D + 1, V)).astype(np.float32)
    y = (z[:, :D] + g.normal(0, near, (B, D, V))).astype(np.float32)
    t = {"z": torch.from_numpy(z).to(DT[dtype]), "y": torch.from_numpy(y).to(DT[dtype])}
    gumbel = -np.log(-np.log(g.uniform(1e-12, 1, (B, D, V))))
    t["ids"] = torch.from_numpy(np.argmax((y if not certain else z[:, :D]) + gumbel, 2)).int()
    t["u"] = torch.from_numpy(g.random((B, D + 1), np.float32))
    t["lens"] = torch.from_numpy(g.integers(0, D + 1, B)).int() if ragged else None
    t["mask"] = None
    if certain:
        t["y"] = None
    return t


def rows(x, pad):
    """[B, D, V] as rows on the GPU, `pad` elements (multiple of 8) further apart,
    with NaN past V."""
    b, d, V = x.shape
    buf = torch.full((b * d, (V + 7) // 8 * 8 + pad), float("nan"), dtype=x.dtype, device=DEV)
    buf[:, :V] = x.reshape(b * d, V).to(DEV)
    return buf[:, :V]


def run(t, pad=(0, 8), **kw):
    on = {k: None if t[k] is None else t[k].to(DEV) for k in ("ids", "u", "lens", "mask")}
    return opd.verify_drafts(rows(t["z"], pad[0]), on["ids"], on["u"],
                             draft_logits=None if t["y"] is None else rows(t["y"], pad[1]),
                             draft_lens=on["lens"], mask=on["mask"], **kw)


def expect(t):
    n = {k: None if t[k] is None else t[k].double().numpy() if t[k].is_floating_point()
         else t[k].numpy() for k in t}
    return ref.verify(n["z"], n["ids"], n["u"], n["y"], n["lens"], n["mask"])


def check(t, name="", **kw):
    out = run(t, **kw)
    torch.cuda.synchronize()
    a, ids, logp, near = expect(t)
    sure = near > 1e-12
    say("%s: %d sequences, %d kept, %d too near a border" % (name, len(a), a.sum(), (~sure).sum()))
    assert sure.all()
    assert np.array_equal(out["accepted"].cpu().numpy(), a)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    got = out["logp"].double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(logp))
    f = np.isfinite(logp)
    # one rounding to fp32 of a value good to 1e-12
    assert (np.abs(got - logp)[f] <= np.abs(logp)[f] * 2.0 ** -24 + 1e-11).all()
    assert np.array_equal(got[~f], logp[~f], equal_nan=True)
    return out


@pytest.mark.parametrize("B,D,V", [(1, 1, 2), (3, 1, 3), (2, 2, 5), (5, 3, 64), (4, 7, 127),
                                   (1, 4, 511), (33, 2, 513), (7, 3, 2049), (2, 66, 700),
                                   (1, 256, 40), (300, 4, 1000), (6, 4, 32003)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
def test_verify(B, D, V, dtype, certain, ragged):
    check(make(B, D, V, dtype, certain, ragged, near=0.3), "verify %d %d %d" % (B, D, V))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("B,D", [(1, 2), (40, 3)])
def test_full_vocabulary(B, D, dtype, certain):
    check(make(B, D, 151936, dtype, certain, True, near=0.2), "full vocabulary")


@pytest.mark.parametrize("near", [0.0, 0.05, 3.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_good_and_bad_drafters(near, dtype):
    """Drafters equal to the target (all kept), near it, and far from it."""
    t = make(50, 5, 700, dtype, near=near, seed=4)
    out = check(t, "near %g" % near)
    if near == 0.0:
        assert (out["accepted"] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [0.0, 1e-7, 300.0, 700.0, -700.0, -30000.0])
def test_unusual_logits(dtype, value):
    """Rows shifted far from 0, and single logits far from the others."""
    t = make(20, 3, 900, dtype, near=0.3, seed=5)
    t["z"][:, 0] += value
    t["z"][:10, 1, 5] = value
    t["y"][:, 1] -= value
    t["y"][5:15, 2, 890] = value
    check(t, "value %g" % value)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
def test_masked_actions(dtype, certain):
    """-inf logits, and the types' lowest values, have no mass: a drafted one is
    refused, none is drawn, and a draft row may have them where the target has not."""
    t = make(40, 4, 600, dtype, certain, near=0.4, seed=6)
    g = np.random.default_rng(7)
    low = torch.finfo(DT[dtype]).min
    dead = torch.from_numpy(g.random((40, 5, 600)) < 0.9)
    dead[:, :, 17] = False
    z = t["z"].masked_fill(dead, float("-inf"))
    z[20:] = torch.where(dead[20:], torch.tensor(low, dtype=z.dtype), t["z"][20:])
    t["z"] = z
    if not certain:
        deady = torch.from_numpy(g.random((40, 4, 600)) < 0.5)
        deady[:, :, 17] = False
        t["y"] = t["y"].masked_fill(deady, float("-inf"))
    out = check(t, "masked actions")
    ids = out["ids"].cpu().long()
    used = ids >= 0
    drawn = torch.gather(t["z"].float(), 2, ids.clamp(min=0)[..., None])[..., 0]
    assert (drawn[used] > low).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), "none"])
@pytest.mark.parametrize("where", ["target", "draft"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_distribution(bad, where, dtype):
    """They end their own sequence, if it gets to them, and touch no other."""
    t = make(12, 3, 400, dtype, near=0.0, seed=8)
    x = t["z"] if where == "target" else t["y"]
    if bad == "none":
        x[:6, 1] = float("-inf")
    else:
        x[:6, 1, 399] = bad
    x[11, 2, 0] = float("nan")
    t["u"][11, 0] = 0.999999
    t["y"][11, 0, int(t["ids"][11, 0])] += 3  # refused at 0: row 2 is not reached
    out = check(t, "undefined %s" % where)
    assert (out["accepted"][:6] == 1).all() and (out["ids"][:6, 1] == -1).all()
    assert int(out["accepted"][11]) == 0 and int(out["ids"][11, 0]) >= 0


def test_bad_arguments_in_the_data_end_their_sequence():
    t = make(12, 3, 400, "bf16", near=0.0, ragged=True, seed=9)
    t["lens"][:] = 3
    t["ids"][0, 1] = 400
    t["ids"][1, 0] = -1
    t["ids"][2, 2] = 2 ** 31 - 1
    t["u"][3, 1] = 1.0
    t["u"][4, 0] = float("nan")
    t["u"][5, 3] = -0.5
    t["u"][6, 3] = float("inf")
    t["lens"][7], t["lens"][8], t["lens"][9] = -1, 4, -2 ** 31
    t["ids"][10, 2], t["lens"][10] = -5, 2  # past its drafts: not looked at
    out = check(t, "bad data")
    assert out["accepted"].cpu().tolist()[:10] == [1, 0, 2, 1, 0, 3, 3, 0, 0, 0]


def large(certain=False, near=0.2, seed=0):
    """So many bf16 logits that their exponentials come from a table."""
    return make(40, 2, 110000, "bf16", certain, near=near, seed=seed)


@pytest.mark.parametrize("value", [0.0, 1e-7, 88.0, 300.0, 700.0, -700.0, -30000.0])
def test_unusual_logits_of_large_batches(value):
    t = large(seed=16)
    t["z"][:, 0] += value
    t["z"][:10, 1, 5] = value
    t["y"][:, 1] -= value
    t["y"][5:15, 1, 109990] = value
    t["z"][20:30, 2, ::2] = value
    check(t, "large, value %g" % value)


@pytest.mark.parametrize("certain", [False, True])
def test_masked_actions_of_large_batches(certain):
    t = large(certain, seed=17)
    g = np.random.default_rng(18)
    low = torch.finfo(torch.bfloat16).min
    dead = torch.from_numpy(g.random((40, 3, 110000)) < 0.99)
    dead[:, :, 17] = False
    z = t["z"].masked_fill(dead, float("-inf"))
    z[20:] = torch.where(dead[20:], torch.tensor(low, dtype=z.dtype), t["z"][20:])
    z[7, 0, :] = float("-inf")
    z[7, 0, 100001] = 3.0  # one action
    t["z"] = z
    if not certain:
        t["y"][:, :, 50000:] = float("-inf")
        t["ids"].clamp_(max=49999)
    check(t, "large, masked actions")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), "none"])
@pytest.mark.parametrize("where", ["target", "draft"])
def test_rows_without_a_distribution_in_large_batches(bad, where):
    t = large(near=0.0, seed=19)
    x = t["z"] if where == "target" else t["y"]
    if bad == "none":
        x[:6, 1] = float("-inf")
    else:
        x[:6, 1, 109999] = bad
    out = check(t, "large, undefined %s" % where)
    assert (out["accepted"][:6] == 1).all() and (out["ids"][:6, 1] == -1).all()


@pytest.mark.parametrize("B,D,V", [(2049, 2, 77), (2500, 3, 300), (9000, 2, 520)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
def test_many_sequences(B, D, V, dtype, certain):
    t = make(B, D, V, dtype, certain, True, near=0.3, seed=20)
    t["mask"] = torch.from_numpy((np.random.default_rng(21).random(B) < 0.8).astype(np.uint8))
    check(t, "many sequences %d %d %d" % (B, D, V))


@pytest.mark.parametrize("B", [1, 5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("certain", [False, True])
def test_rows_of_over_a_million(B, dtype, certain):
    check(make(B, 1, 1100003, dtype, certain, near=0.1, seed=22), "long rows")


def test_masked_sequences_are_left_alone():
    t = make(9, 3, 500, "f32", near=0.3, seed=10)
    t["mask"] = torch.tensor([1, 0, 1, 1, 0, 0, 1, 1, 0], dtype=torch.uint8)
    t["z"][1] = float("nan")
    t["ids"][4] = -9
    out = check(t, "masked")
    assert (out["ids"][1] == -1).all() and (out["logp"][4] == 0).all()
    t["mask"] = t["mask"].bool()
    check(t, "bool mask")


def test_uniforms_at_their_ends():
    """u = 0 keeps any token of mass and draws the first index of mass; the largest
    u below 1 draws the last."""
    t = make(8, 2, 300, "f32", near=1.0, seed=11)
    t["u"][:4] = 0.0
    t["u"][4:] = 1.0 - 2.0 ** -24
    t["z"][:, :, :3] = float("-inf")
    t["z"][:, :, 290:] = float("-inf")
    t["ids"] = t["ids"].clamp(3, 289)
    out = run(t)
    a, ids, _, _ = expect(t)
    assert np.array_equal(out["accepted"].cpu().numpy(), a)
    assert np.array_equal(out["ids"].cpu().numpy(), ids)
    assert (out["accepted"][:4] == 2).all() and (out["ids"][:4, 2] == 3).all()


def test_equal_rows_leave_no_residual_to_draw_from():
    """Where the target's row is the drafter's, no token is refused."""
    t = make(6, 4, 256, "bf16", near=0.0, seed=12)
    t["u"][:] = 1.0 - 2.0 ** -24
    out = run(t)
    assert (out["accepted"] == 4).all()


def test_draws_at_length_zero_are_sample_actions():
    t = make(30, 2, 5000, "bf16", seed=13)
    t["lens"] = torch.zeros(30, dtype=torch.int32)
    out = run(t)
    plain = opd.sample_actions(rows(t["z"][:, :1], 0), t["u"][:, 2:].to(DEV).contiguous())
    assert torch.equal(out["ids"][:, :1], plain["ids"])
    assert torch.equal(out["logp"][:, :1], plain["logp"])


def test_no_sequences_and_no_logp():
    z = torch.empty(0, 64, device=DEV)
    out = opd.verify_drafts(z, torch.empty(0, 3, dtype=torch.int32, device=DEV),
                            torch.empty(0, 4, device=DEV))
    assert out["accepted"].shape == (0,) and out["ids"].shape == (0, 4)
    t = make(5, 2, 100, "f32", seed=14)
    assert "logp" not in run(t, want_logp=False)
    assert torch.equal(run(t, want_logp=False)["ids"], run(t)["ids"])


def test_rows_past_4_gib():
    """Offsets that pass 32 bits: rows of a batch of over 4 GiB."""
    B, D, V = 3600, 3, 151936
    t = make(4, D, V, "bf16", near=0.1, seed=15)
    z = torch.zeros(B * (D + 1), V, dtype=torch.bfloat16, device=DEV)
    z[-4 * (D + 1):] = t["z"].reshape(-1, V).to(DEV)
    mask = torch.zeros(B, dtype=torch.uint8, device=DEV)
    mask[-4:] = 1
    ids = torch.zeros(B, D, dtype=torch.int32, device=DEV)
    ids[-4:] = t["ids"].to(DEV)
    u = torch.zeros(B, D + 1, device=DEV)
    u[-4:] = t["u"].to(DEV)
    t["y"] = None
    out = opd.verify_drafts(z, ids, u, mask=mask)
    a, want, _, near = expect(t)
    assert (near > 1e-12).all()
    assert np.array_equal(out["ids"][-4:].cpu().numpy(), want)
