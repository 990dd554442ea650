"""Selection of beams against a plain 64-bit form, and the reordering of states bit for
bit."""
import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2606_24143_amd as opd
from gpu_common import DEV

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


def logits(g, B, W, V, kind, size=2.0):
    """Rows that end in NaN."""
    ld = (V + 7) // 8 * 8 + 8
    z = torch.full((B * W, ld), float("nan"), dtype=DT[kind], device=DEV)
    z[:, :V] = (torch.randn(B * W, V, device=DEV, generator=g) * size).to(DT[kind])
    return z[:, :V]


def check(z, scores, k, finished=None, ties=False, **kw):
    """Parents and tokens equal the reference's; no two beams' candidates there are nearer
    than 1e-6 (a hundred times what the kernels' sums are off)."""
    B, W = scores.shape
    got = opd.beam_select(z, scores, k=k, finished=finished, **kw)
    want, parents, ids, near = ref.beams(z.double().cpu().numpy().reshape(B, W, -1),
                                         scores.double().cpu().numpy(), k,
                                         None if finished is None else finished.cpu().numpy())
    assert ties or near > 1e-6
    assert np.array_equal(got["parents"].cpu().numpy(), parents)
    assert np.array_equal(got["ids"].cpu().numpy(), ids)
    s = got["scores"].double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(s[~fine], want[~fine], equal_nan=True)
    # the rounding to fp32, and the sums
    assert (np.abs(s[fine] - want[fine]) <= 2.0 ** -24 * np.abs(want[fine]) + 1e-7).all()
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,W,V,k", [
    (1, 1, 2, 1), (1, 1, 2, 4), (1, 2, 3, 5), (2, 3, 7, 3), (3, 4, 255, 8), (1, 4, 2049, 4),
    (5, 5, 4000, 10), (2, 8, 16385, 8), (1, 16, 33001, 32), (70, 2, 5000, 2), (3, 64, 300, 64),
    (150, 8, 2100, 8), (1, 1, 300_000, 64), (40, 4, 50_257, 4)])
def test_sizes(kind, B, W, V, k):
    g = torch.Generator(DEV).manual_seed(V + B)
    z = logits(g, B, W, V, kind)
    scores = -3.0 * torch.rand(B, W, device=DEV, generator=g)
    check(z, scores, k)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(20_000, 8), (20_000, 16), (20_000, 17), (20_000, 64),
                                 (100_000, 1), (100_000, 16), (100_000, 33)])
def test_more_candidates_than_are_kept_at_once(kind, V, k):
    """64 beams of many parts; one beam far ahead, and all of them near each other."""
    g = torch.Generator(DEV).manual_seed(k)
    B, W = 2, 64
    z = logits(g, B, W, V, kind)
    scores = -torch.rand(B, W, device=DEV, generator=g)
    scores[0, 50] = 60.0
    check(z, scores, k)
    # rows alike: equal candidates of all beams
    z[W:] = z[W]
    scores[1] = -0.25
    check(z, scores, k, ties=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_finished_and_missing_beams(kind):
    g = torch.Generator(DEV).manual_seed(1)
    B, W, V = 12, 4, 1000
    z = logits(g, B, W, V, kind)
    scores = -8.0 * torch.rand(B, W, device=DEV, generator=g)
    done = torch.rand(B, W, device=DEV, generator=g) < 0.4
    done[3] = True        # nothing but what has ended: fewer than k
    done[4] = False
    scores[5, 1:] = -INF  # a first step: one beam
    done[5] = False
    scores[6] = -INF      # no beam at all
    z[7 * W:8 * W, 5:] = -INF  # few tokens allowed
    done[7] = False
    z[8 * W + 2] = -INF   # a row without any
    got = check(z, scores, 30, done)
    assert (got["parents"][6] == -1).all() and (got["scores"][6] == -INF).all()
    assert (got["ids"][3] == -1).all() and int((got["parents"][3] >= 0).sum()) == W
    assert int((got["parents"][7] >= 0).sum()) == 5 * W
    # rows of finished and missing beams are not read
    z.view(B, W, V)[done] = float("nan")
    z[5 * W + 1:6 * W] = INF
    z[6 * W:7 * W] = float("nan")
    again = opd.beam_select(z, scores, k=30, finished=done.to(torch.uint8))
    for key in got:
        assert torch.equal(again[key], got[key])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_what_is_no_distribution_stays_in_its_group(kind):
    g = torch.Generator(DEV).manual_seed(2)
    B, W, V = 6, 3, 4100
    z = logits(g, B, W, V, kind)
    scores = -torch.rand(B, W, device=DEV, generator=g)
    z[0 * W + 1, 4099] = float("nan")
    z[1 * W, 0] = INF
    scores[2, 2] = float("nan")
    scores[3, 0] = INF
    got = check(z, scores, 4)
    assert got["scores"][:4].isnan().all() and got["scores"][4:].isfinite().all()
    assert (got["parents"][:4] == -1).all() and (got["ids"][:4] == -1).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(50, 7), (5000, 9), (40_000, 64)])
def test_ties_go_to_the_lower_beam_then_the_lower_token(kind, V, k):
    B, W = 2, 3
    z = torch.zeros(B * W, (V + 7) // 8 * 8, dtype=DT[kind], device=DEV)[:, :V]
    scores = torch.zeros(B, W, device=DEV)
    got = check(z, scores, k, ties=True)
    assert (got["parents"] == 0).all()
    assert torch.equal(got["ids"], torch.arange(k, device=DEV, dtype=torch.int32).expand(B, k))
    # some above, many equal below them, in the other rows too
    z[:, V - 1] = 1.0
    z[2::3, V // 2] = 1.0
    z[:, 1] = -INF
    check(z, scores, k, ties=True)
    # rows of few distinct values
    g = torch.Generator(DEV).manual_seed(V)
    z.copy_(torch.randint(0, 3, z.shape, device=DEV, generator=g))
    z[3:] = z[:3]
    scores[:, 1] = -0.75
    check(z, scores, k, ties=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 8, 64])
def test_sorted_rows(kind, k):
    """All that is large lies in few lanes, or rises along a part."""
    B, W, V = 2, 2, 20_000
    up = torch.arange(V, device=DEV, dtype=torch.float32) / V * 30
    if kind == "bf16":  # distinct values are few: large ones in runs
        up = (up * 8).floor() / 8
    z = torch.zeros(B * W, V, dtype=DT[kind], device=DEV)
    z[0], z[1], z[2] = up, up.flip(0), -up
    z[3] = torch.where(torch.arange(V, device=DEV) // 64 == 77, 20.0, 0.0)
    scores = torch.tensor([[0.0, -0.37], [0.0, -1.7]], device=DEV)
    check(z, scores, k, ties=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_far_logits(kind):
    """Logits far from 0, masked ones of the type's lowest value, and rows of nothing
    else."""
    B, W, V = 4, 2, 3000
    g = torch.Generator(DEV).manual_seed(3)
    z = logits(g, B, W, V, kind)
    low = torch.finfo(DT[kind]).min
    z[0:2] += 1000.0
    z[2:4] -= 3000.0
    z[4:6, 10:] = low
    z[6:8] = low
    scores = torch.tensor([[0.0, -0.3]] * 4, device=DEV)
    got = check(z, scores, 8, ties=True)
    assert np.isclose(float(got["scores"][3, 0]), -np.log(V))


def test_a_long_vocabulary_and_many_rows():
    """More parts to a row than lanes of a wavefront."""
    g = torch.Generator(DEV).manual_seed(4)
    z = logits(g, 1, 3, 1_100_000, "bf16")
    check(z, torch.zeros(1, 3, device=DEV), 16, ties=True)


def test_scores_are_log_probabilities():
    g = torch.Generator(DEV).manual_seed(5)
    z = logits(g, 3, 1, 9000, "f32")
    got = opd.beam_select(z, torch.zeros(3, 1, device=DEV), k=20)
    top = opd.topk_support(z, 20)
    assert torch.equal(got["ids"], top["idx"])
    assert torch.allclose(got["scores"], top["logp"], atol=2e-6)


# ---------------------------------------------------------------- reordering

@pytest.mark.parametrize("place", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.int64, torch.uint8,
                                   torch.float8_e4m3fn, torch.bool])
@pytest.mark.parametrize("B,W,shape", [
    (1, 1, (1,)), (1, 4, (7,)), (3, 2, (1023,)), (2, 5, (3, 129)), (1, 16, (64, 33)),
    (2, 17, (40,)), (1, 64, (5, 7, 11)), (2, 8, (4, 1024)), (5, 3, ())])
def test_reorder(place, dtype, B, W, shape):
    rng = np.random.default_rng(B + W)
    raw = torch.from_numpy(rng.integers(0, 2 if dtype == torch.bool else 100,
                                        (B * W,) + shape)).to(DEV)
    states = raw.to(torch.uint8).view(dtype) if dtype == torch.float8_e4m3fn else raw.to(dtype)
    parents = rng.integers(0, W, (B, W)).astype(np.int32)
    want = ref.reorder(raw.cpu().numpy(), parents, W)
    p = torch.from_numpy(parents).to(DEV)
    got = opd.reorder_beams(states, p, out=states if place else None)["states"]
    assert got.shape == states.shape and got.dtype == dtype
    assert not place or got is states
    back = got.contiguous().view(torch.uint8) if dtype == torch.float8_e4m3fn else got
    assert np.array_equal(back.long().cpu().numpy(), want)


def test_reorder_keeps_every_bit():
    x = torch.randint(-2 ** 31, 2 ** 31 - 1, (8, 999), device=DEV, dtype=torch.int32)
    x = torch.nn.functional.pad(x, (0, 1)).view(torch.float32)[:, :999]  # NaN payloads among them
    p = torch.tensor([[3, 3, 0, 1], [0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    got = opd.reorder_beams(x, p)["states"]
    want = x[torch.tensor([3, 3, 0, 1, 4, 5, 6, 7], device=DEV)]
    assert torch.equal(got.contiguous().view(torch.int32), want.contiguous().view(torch.int32))


@pytest.mark.parametrize("place", [True, False])
def test_parents_that_are_none(place):
    states = torch.ones(6, 50, device=DEV)
    p = torch.tensor([[0, -1, 3], [2, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device=DEV)
    got = opd.reorder_beams(states, p, out=states if place else None)["states"]
    assert got.sum(1).tolist() == [50, 0, 0, 50, 0, 0]


@pytest.mark.parametrize("k", [1, 3, 9])
def test_more_or_fewer_beams_than_there_were(k):
    rng = np.random.default_rng(k)
    states = torch.arange(4 * 5 * 6, device=DEV).view(20, 6).to(torch.int16)
    parents = rng.integers(0, 5, (4, k)).astype(np.int32)
    got = opd.reorder_beams(states, torch.from_numpy(parents).to(DEV))["states"]
    assert np.array_equal(got.cpu().numpy(), ref.reorder(states.cpu().numpy(), parents, 5))


@pytest.mark.parametrize("length", [1, 5, 32])
def test_a_cache_cut_at_its_length(length):
    """[beams, heads, longest, width]: what lies past the length stays as it is."""
    g = torch.Generator(DEV).manual_seed(6)
    cache = torch.randn(6, 3, 32, 20, device=DEV, generator=g).bfloat16()
    p = torch.tensor([[2, 0, 1], [1, 1, 1]], dtype=torch.int32, device=DEV)
    at = torch.tensor([2, 0, 1, 4, 4, 4], device=DEV)
    want = cache.clone()
    want[:, :, :length] = cache[at][:, :, :length]
    fresh = opd.reorder_beams(cache[:, :, :length], p)["states"]
    assert torch.equal(fresh, want[:, :, :length])
    to = torch.zeros_like(cache)
    opd.reorder_beams(cache[:, :, :length], p, out=to[:, :, :length])
    assert torch.equal(to[:, :, :length], want[:, :, :length]) and (to[:, :, length:] == 0).all()
    cut = cache[:, :, :length]
    opd.reorder_beams(cut, p, out=cut)
    assert torch.equal(cache, want)


@pytest.mark.parametrize("place", [False, True])
def test_caches_of_all_layers(place):
    L, B, W = 3, 2, 4
    g = torch.Generator(DEV).manual_seed(8)
    cache = torch.randn(L, B * W, 5, 24, device=DEV, generator=g)
    parents = torch.randint(0, W, (B, W), device=DEV, generator=g, dtype=torch.int32)
    at = (parents.long() + torch.arange(B, device=DEV)[:, None] * W).view(-1)
    want = cache[:, at]
    states = cache.transpose(0, 1)
    got = opd.reorder_beams(states, parents, out=states if place else None)["states"]
    assert torch.equal(got, want.transpose(0, 1))
    if place:
        assert torch.equal(cache, want)
    # into another such buffer
    if not place:
        other = torch.zeros_like(cache)
        opd.reorder_beams(states, parents, out=other.transpose(0, 1))
        assert torch.equal(other, want)


def test_states_at_odd_addresses():
    buf = torch.arange(4000, device=DEV, dtype=torch.int32).to(torch.uint8)
    states = buf[3:3 + 8 * 101].view(8, 101)
    p = torch.tensor([[1, 0, 3, 2], [3, 3, 0, 2]], dtype=torch.int32, device=DEV)
    want = ref.reorder(states.cpu().numpy(), p.cpu().numpy(), 4)
    before, after = buf[:3].clone(), buf[3 + 808:].clone()
    assert np.array_equal(opd.reorder_beams(states, p)["states"].cpu().numpy(), want)
    opd.reorder_beams(states, p, out=states)
    assert np.array_equal(states.cpu().numpy(), want)
    assert torch.equal(buf[:3], before) and torch.equal(buf[811:], after)


@pytest.mark.parametrize("k", [3, 20])
@pytest.mark.parametrize("inner", list(range(1, 36)) + [255, 4095, 4097, 4111])
def test_states_of_any_length(inner, k):
    """Bytes of a state that are no multiple of what a lane moves, to another buffer and in
    place, with guards around each."""
    rng = np.random.default_rng(inner)
    raw = torch.from_numpy(rng.integers(0, 256, (2 * k, inner + 5))).to(torch.uint8).to(DEV)
    parents = torch.from_numpy(rng.integers(-1, k, (2, k)).astype(np.int32)).to(DEV)
    want = ref.reorder(raw[:, 2:2 + inner].cpu().numpy(), parents.cpu().numpy(), k)
    to = torch.full_like(raw, 9)
    opd.reorder_beams(raw[:, 2:2 + inner], parents, out=to[:, 2:2 + inner])
    assert np.array_equal(to[:, 2:2 + inner].cpu().numpy(), want)
    assert (to[:, :2] == 9).all() and (to[:, 2 + inner:] == 9).all()
    before = raw.clone()
    states = raw[:, 2:2 + inner]
    opd.reorder_beams(states, parents, out=states)
    assert np.array_equal(states.cpu().numpy(), want)
    assert torch.equal(raw[:, :2], before[:, :2]) and torch.equal(raw[:, 2 + inner:],
                                                                  before[:, 2 + inner:])


def test_states_past_four_gib():
    W, n = 4, 1_300_000_000
    states = torch.zeros(W, n, dtype=torch.uint8, device=DEV)
    for w in range(W):
        states[w, -5:] = w + 1
        states[w, 0] = 10 + w
    p = torch.tensor([[3, 2, 2, 0]], dtype=torch.int32, device=DEV)
    opd.reorder_beams(states, p, out=states)
    assert states[:, -1].tolist() == [4, 3, 3, 1] and states[:, 0].tolist() == [13, 12, 12, 10]
