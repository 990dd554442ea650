"""Token embeddings and their gradient against a plain 64-bit form, at the sizes, ids and
strides where they can go wrong."""
import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2606_24143_amd as opd
from gpu_common import DEV, say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows(g, n, m, kind, pad=0, size=1.0):
    """[n, m] normal values in rows that end in NaN."""
    each = 4 if kind == "f32" else 8
    ld = (m + each - 1) // each * each + pad * each
    buf = torch.full((n, ld), float("nan"), dtype=DT[kind], device=DEV)
    buf[:, :m] = (torch.randn(n, m, device=DEV, generator=g) * size).to(DT[kind])
    return buf[:, :m]


def np64(t):
    return t.double().cpu().numpy()


def ids_of(rng, n, V, skew=False, bad=False):
    ids = rng.integers(0, V, n)
    if skew:  # most tokens are one of three entries
        ids = np.where(rng.random(n) < 0.8, rng.integers(0, min(3, V), n) * (V // 3), ids)
    if bad:
        ids[rng.random(n) < 0.2] = -1
    return ids.astype(np.int32)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,H", [(1, 1, 1), (1, 7, 8), (5, 100, 63), (17, 33, 64), (64, 1000, 257),
                                   (130, 50, 512), (33, 211, 1025), (9, 40, 2049), (3, 5, 4104)])
def test_lookup(kind, out, N, V, H):
    g = torch.Generator(DEV).manual_seed(N + H)
    table = rows(g, V, H, kind, pad=1)
    ids = ids_of(np.random.default_rng(H), N, V, bad=True)
    each = 4 if out == "f32" else 8
    ld = (H + each - 1) // each * each + each
    buf = torch.full((N, ld), 7.0, dtype=DT[out], device=DEV)
    got = opd.embed_tokens(table, torch.from_numpy(ids).to(DEV), scale=1.7, dtype=DT[out],
                           out=buf[:, :H])["hidden"]
    want = ref.embed(np64(table), ids, float(np.float32(1.7)))
    off = np.abs(np64(got) - want)
    # the product's rounding, and the result's
    assert (off <= (2.0 ** -24 + ref.HALF[out] * (1 + 2.0 ** -24)) * np.abs(want)).all()
    assert (got[torch.from_numpy(ids).to(DEV) == -1] == 0).all()
    assert (buf[:, H:] == 7.0).all()
    fresh = opd.embed_tokens(table, torch.from_numpy(ids).to(DEV), scale=1.7, dtype=DT[out])
    assert torch.equal(fresh["hidden"], got)


def test_lookup_of_ids_outside_the_table():
    table = torch.ones(10, 40, device=DEV)
    ids = torch.tensor([0, 9, 10, -1, -2, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    got = opd.embed_tokens(table, ids)["hidden"]
    assert (got[:2] == 1).all() and (got[3] == 0).all()
    assert got[[2, 4, 5, 6]].isnan().all()
    dy = torch.ones(7, 40, device=DEV)
    d = opd.embed_grads(dy, ids, 10)["dtable"]
    want = torch.zeros(10, 40, device=DEV)
    want[0] = want[9] = 1
    assert torch.equal(d, want)
    # (the same where tokens are sorted)
    d = opd.embed_grads(dy.repeat(100, 1), ids.repeat(100), 10)["dtable"]
    assert torch.equal(d, 100 * want)


def test_lookup_far_into_a_table():
    """Rows past 4 GiB."""
    V, H = 600_000, 4096
    table = torch.zeros(V, H, dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([V - 1, 524_287, 524_288, 524_289], dtype=torch.int32, device=DEV)
    for i in ids.tolist():
        table[i] = i % 251
    got = opd.embed_tokens(table, ids)["hidden"]
    assert torch.equal(got, table[ids.long()])
    out = torch.full((V, H), 3.0, dtype=torch.bfloat16, device=DEV)
    opd.embed_grads(got, ids, V, dtype=torch.bfloat16, out=out)
    assert torch.equal(out, table)


def check_grads(dy, ids, V, scale, out, **kw):
    got = opd.embed_grads(dy, torch.from_numpy(ids).to(DEV), V, scale=scale, dtype=DT[out],
                          **kw)["dtable"]
    want, off = ref.embed_grads(np64(dy), ids, V, float(np.float32(scale)))
    off = off + ref.HALF[out] * (np.abs(want) + off)
    err = np.abs(np64(got) - want)
    assert (err <= off).all(), "off by %g where %g may be" % (err.max(), off.ravel()[err.argmax()])
    return got


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"),
                                      ("f32", "bf16")])
@pytest.mark.parametrize("N,V,H,skew", [
    (0, 5, 8, False), (1, 1, 1, False), (3, 40, 65, False), (256, 20, 128, False),
    (257, 20, 128, False), (300, 2000, 260, True), (1000, 64, 515, True), (700, 65, 1030, True),
    (4097, 1500, 96, True), (2500, 3, 33, False), (1025, 70_001, 12, True)])
def test_gradient(kind, out, N, V, H, skew):
    g = torch.Generator(DEV).manual_seed(N + V)
    dy = rows(g, N, H, kind, pad=1)
    ids = ids_of(np.random.default_rng(N + H), N, V, skew, bad=True)
    got = check_grads(dy, ids, V, 0.7, out)
    say("%s -> %s %s: %d rows with tokens" % (kind, out, (N, V, H),
                                              int((got != 0).any(1).sum())))
    again = opd.embed_grads(dy, torch.from_numpy(ids).to(DEV), V, scale=0.7, dtype=DT[out])
    assert torch.equal(again["dtable"], got)


@pytest.mark.parametrize("N", [64, 65, 200, 256])
def test_few_tokens_of_a_large_table(N):
    V = 300_000
    g = torch.Generator(DEV).manual_seed(N)
    ids = ids_of(np.random.default_rng(N), N, V, True, bad=True)
    check_grads(rows(g, N, 12, "f32"), ids, V, 1.0, "bf16")


@pytest.mark.parametrize("N,V", [(8192, 100), (8193, 2), (30_011, 1500)])
def test_many_tokens(N, V):
    """More than a wavefront of the sort holds at once, and as many."""
    g = torch.Generator(DEV).manual_seed(N)
    ids = ids_of(np.random.default_rng(N), N, V, True, bad=True)
    check_grads(rows(g, N, 40, "bf16"), ids, V, 1.0, "f32")


@pytest.mark.parametrize("N", [100, 3000])
@pytest.mark.parametrize("first", [0, 1, 63, 64, 65])
def test_entries_whose_tokens_end_at_any_place_of_a_tile(N, first):
    """Runs of sorted tokens of 63 to 129, which begin and end at, before and past the
    borders of the tiles that long ones are summed by."""
    lengths = [first, 64, 65, 1, 128, 129, 63, 66, 2, 200]
    ids = np.repeat(np.arange(len(lengths)), lengths)
    ids = np.concatenate([ids, np.full(max(0, N - len(ids)), 12)])[:N].astype(np.int32)
    np.random.default_rng(1).shuffle(ids)
    g = torch.Generator(DEV).manual_seed(first)
    check_grads(rows(g, N, 100, "f32"), ids, 14, 1.0, "f32")


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N", [40, 900])
def test_gradient_added_to_another(out, N):
    V, H = 500, 70
    g = torch.Generator(DEV).manual_seed(N)
    dy = rows(g, N, H, "bf16")
    ids = ids_of(np.random.default_rng(N), N, V // 2, True)
    have = rows(g, V, H, out, pad=1)
    have[V // 2 + 3] = float("nan")  # (no token: neither read nor written)
    before = have.clone()
    want, off = ref.embed_grads(np64(dy), ids, V, 2.0)
    total = want + np64(before)
    got = opd.embed_grads(dy, torch.from_numpy(ids).to(DEV), V, scale=2.0, dtype=DT[out], out=have,
                          accumulate=True)["dtable"]
    assert got.data_ptr() == have.data_ptr()
    some = np.zeros(V, bool)
    some[ids] = True
    off = off + 2.0 ** -24 * (np.abs(total) + off) + ref.HALF[out] * (np.abs(total) + off)
    assert (np.abs(np64(got) - total) <= off)[some].all()
    assert np.array_equal(np64(got)[~some], np64(before)[~some], equal_nan=True)


def test_gradient_leaves_what_lies_past_its_rows():
    ids = torch.tensor([1, 1, 0], dtype=torch.int32, device=DEV)
    buf = torch.full((4, 24), 5.0, device=DEV)
    opd.embed_grads(torch.ones(3, 20, device=DEV)[:, :17], ids, 3,
                    out=buf[:3, :17])
    assert (buf[:, 17:] == 5).all() and (buf[3] == 5).all()
    assert (buf[0, :17] == 1).all() and (buf[1, :17] == 2).all() and (buf[2, :17] == 0).all()


@pytest.mark.parametrize("N", [30, 700])
def test_gradient_is_that_of_the_lookup(N):
    """<lookup(table), dy> is linear in the table: it is <table, gradient>, and so are its
    differences."""
    V, H = 90, 72
    g = torch.Generator(DEV).manual_seed(N)
    table, dy = rows(g, V, H, "f32"), rows(g, N, H, "f32")
    ids = torch.from_numpy(ids_of(np.random.default_rng(N), N, V, True, True)).to(DEV)
    d = opd.embed_grads(dy, ids, V, scale=0.5)["dtable"].double()
    loss = lambda t: (opd.embed_tokens(t, ids, scale=0.5)["hidden"].double() * dy.double()).sum()
    for v, c in ((0, 0), (V // 3, 5), (V - 1, H - 1)):
        up, down = table.clone(), table.clone()
        up[v, c] += 1.0
        down[v, c] -= 1.0
        step = float(up[v, c].double() - down[v, c].double())
        # the products are exact (a scale of 1 / 2): the gradient's sums, N additions at most
        bound = (N + 2) * 2.0 ** -24 * float(dy.abs().double().sum(0)[c])
        assert abs(float(loss(up) - loss(down)) / step - float(d[v, c])) <= bound


def test_infinities_and_nan_stay_in_their_entries():
    dy = torch.ones(400, 16, device=DEV)
    ids = torch.arange(400, dtype=torch.int32, device=DEV) % 40
    dy[7, 3] = float("nan")
    dy[13, 5] = float("inf")
    d = opd.embed_grads(dy, ids, 50)["dtable"]
    assert d[7, 3].isnan() and d[13, 5] == float("inf")
    d[7, 3] = d[13, 5] = 10.0
    assert (d[:40] == 10).all() and (d[40:] == 0).all()


@pytest.mark.parametrize("N", [5, 400])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -2.0])
def test_entries_without_a_token_are_zeros_whatever_the_scale(N, scale):
    ids = torch.arange(N, dtype=torch.int32, device=DEV) % 5
    d = opd.embed_grads(torch.ones(N, 24, device=DEV), ids, 20, scale=scale)["dtable"]
    assert (d[5:] == 0).all() and not d[5:].signbit().any()
    want = torch.full_like(d[:5], scale * (N // 5))
    assert torch.equal(d[:5].nan_to_num(9.0), want.nan_to_num(9.0))


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("first", [0, 1, 15, 16, 17])
def test_runs_of_tokens_around_a_tile_of_16(kind, out, first):
    """Entries of up to 16 tokens are summed by themselves, longer ones tile by tile: runs on
    both sides of that, which begin and end at, before and past the tiles' borders."""
    lengths = [first, 15, 16, 17, 31, 32, 33, 1, 2, 48, 16, 16, 17, 14, 18, 30]
    ids = np.repeat(np.arange(len(lengths)), lengths).astype(np.int32)
    assert len(ids) > 256  # (sorted)
    np.random.default_rng(first).shuffle(ids)
    g = torch.Generator(DEV).manual_seed(first)
    for H in (100, 300):  # one vector to a lane, and two
        check_grads(rows(g, len(ids), H, kind), ids, len(lengths) + 3, 1.0, out)
