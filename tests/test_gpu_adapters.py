"""Low-rank adapters beside a shared projection and their gradients, against a plain
64-bit form with bounds derived from the sums' lengths (model_ref)."""
import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2606_24143_amd as opd
from gpu_common import DEV

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN = float("nan")


def rows(g, *shape, kind, pad=0, size=1.0):
    """Normal values in rows that end in NaN."""
    each = 4 if kind == "f32" else 8
    m = shape[-1]
    ld = (m + each - 1) // each * each + pad * each
    buf = torch.full(shape[:-1] + (ld,), NAN, dtype=DT[kind], device=DEV)
    buf[..., :m] = (torch.randn(*shape, device=DEV, generator=g) * size).to(DT[kind])
    return buf[..., :m]


def aligned(t):
    """A copy in rows a multiple of 16 bytes apart."""
    each = 16 // t.element_size()
    buf = t.new_zeros(t.shape[:-1] + ((t.shape[-1] + each - 1) // each * each,))
    buf[..., :t.shape[-1]] = t
    return buf[..., :t.shape[-1]]


def np64(t):
    return t.double().cpu().numpy()


def batch(seed, N, H, O, G, r, kind, ykind, bad=True, packed=False):
    g = torch.Generator(DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, G, N)
    if packed:
        ids = np.sort(ids)
    if bad:
        ids[rng.random(N) < 0.15] = -1
    return dict(x=rows(g, N, H, kind=kind, pad=1), a=rows(g, G, r, H, kind=kind, pad=1, size=H ** -0.5),
                b=rows(g, G, r, O, kind=kind, size=0.5), y=rows(g, N, O, kind=ykind, pad=2),
                scales=torch.rand(G, device=DEV, generator=g) + 0.5,
                ids=torch.from_numpy(ids.astype(np.int32)).to(DEV))


def near(name, got, want, off, half):
    off = off + half * (np.abs(want) + off)
    got = np64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), name
    err = np.where(np.isnan(want), 0.0, np.abs(got - want))
    worst = np.max(err - np.nan_to_num(off)) if err.size else -1.0
    assert worst <= 0.0, "%s: off by %g more than it may be (of %g)" % (name, worst, err.max())


def check(s, kind, ykind):
    """Forward and backward of one batch, with all that is optional and without."""
    call = dict(x=s["x"], a=s["a"], b=s["b"], adapter_ids=s["ids"], scales=s["scales"])
    ids, scales = s["ids"].cpu().numpy(), np64(s["scales"])
    x, a, b, y = (np64(s[k]) for k in ("x", "a", "b", "y"))
    out = opd.add_adapters(s["y"], want_low=True, **call)
    want, off, low, low_off = ref.adapters(y, x, a, b, ids, scales, kind, ykind)
    near("out", out["out"], want, off, ref.HALF[ykind])
    near("low", out["low"], low, low_off, 0.0)
    plain = opd.add_adapters(s["y"], **call)
    assert torch.equal(plain["out"].nan_to_num(), out["out"].nan_to_num()) and set(plain) == {"out"}
    # the gradients (y stands for dy)
    d = opd.adapter_grads(s["y"], **call)
    want = ref.adapter_grads(y, x, a, b, ids, scales, kind, ykind)
    for k in ("da", "db", "dx"):
        near(k, d[k], *want[k], ref.HALF[kind if k == "dx" else "f32"])
    e = opd.adapter_grads(s["y"], low=out["low"], dx=s["x"], **call)
    want = ref.adapter_grads(y, x, a, b, ids, scales, kind, ykind, low=np64(out["low"]), dx_shared=x)
    for k in ("da", "db", "dx"):
        near(k + " with low", e[k], *want[k], ref.HALF[kind if k == "dx" else "f32"])
    f = opd.adapter_grads(s["y"], want_dx=False, **call)
    assert set(f) == {"da", "db"}
    for k in f:
        assert torch.equal(f[k], d[k])  # (and every call repeats itself bit for bit)
    return out, d


KINDS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("N,H,O,G,r", [
    (1, 1, 1, 1, 1), (1, 64, 130, 1, 16), (2, 33, 7, 5, 3), (15, 65, 129, 2, 8), (16, 128, 512, 1, 17),
    (17, 200, 513, 4, 16), (64, 520, 600, 64, 16), (65, 96, 640, 3, 32), (130, 70, 260, 2, 33),
    (200, 1031, 300, 7, 64), (90, 256, 1025, 2, 65), (70, 136, 200, 3, 128), (700, 300, 250, 2, 5)])
def test_sizes(kind, ykind, N, H, O, G, r):
    check(batch(N + O, N, H, O, G, r, kind, ykind), kind, ykind)


@pytest.mark.parametrize("kind,ykind", KINDS)
def test_long_axes(kind, ykind):
    """Axes that are cut into parts, of unequal lengths, and tokens that are."""
    check(batch(1, 40, 5003, 2600, 3, 8, kind, ykind), kind, ykind)
    check(batch(2, 1500, 72, 100, 1, 16, kind, ykind, packed=True), kind, ykind)
    check(batch(3, 1300, 100, 72, 1000, 4, kind, ykind), kind, ykind)


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("N,G", [(8192, 3), (8193, 70), (20_001, 1000)])
def test_many_tokens(kind, ykind, N, G):
    """More than a wavefront of the sort holds at once, and as many."""
    check(batch(8, N, 24, 40, G, 5, kind, ykind), kind, ykind)


@pytest.mark.parametrize("kind,ykind", KINDS)
def test_one_adapter_has_nearly_all_tokens(kind, ykind):
    s = batch(4, 520, 80, 140, 6, 12, kind, ykind)
    s["ids"].fill_(4)
    s["ids"][[0, 63, 64, 519]] = torch.tensor([1, -1, 0, 1], dtype=torch.int32, device=DEV)
    _, d = check(s, kind, ykind)
    assert (d["da"][[2, 3, 5]] == 0).all() and (d["db"][[2, 3, 5]] == 0).all()


@pytest.mark.parametrize("kind,ykind", KINDS)
def test_tokens_without_an_adapter_and_bad_ids(kind, ykind):
    s = batch(5, 150, 40, 90, 3, 6, kind, ykind, bad=False)
    s["ids"][::3] = -1
    s["ids"][1::7] = torch.tensor([3, -2, 2 ** 31 - 1, -2 ** 31] * 6, dtype=torch.int32,
                                  device=DEV)[:len(s["ids"][1::7])]
    out, d = check(s, kind, ykind)
    none = s["ids"] == -1
    assert torch.equal(out["out"][none], s["y"][none])
    assert (d["dx"][none] == 0).all()
    # none has any
    s["ids"].fill_(-1)
    out, d = check(s, kind, ykind)
    assert torch.equal(out["out"], s["y"])
    assert all((d[k] == 0).all() for k in d)


@pytest.mark.parametrize("kind,ykind", KINDS)
def test_in_place(kind, ykind):
    s = batch(6, 100, 64, 300, 4, 16, kind, ykind)
    call = dict(x=s["x"], a=s["a"], b=s["b"], adapter_ids=s["ids"])
    want = opd.add_adapters(s["y"], **call)["out"]
    y = torch.full((100, 304), 9.0, dtype=DT[ykind], device=DEV)
    y[:, :300] = s["y"]
    got = opd.add_adapters(y[:, :300], out=y[:, :300], **call)["out"]
    assert got.data_ptr() == y.data_ptr() and torch.equal(got, want)
    assert (y[:, 300:] == 9).all()
    to = torch.full((100, 312), 9.0, dtype=DT[ykind], device=DEV)
    opd.add_adapters(s["y"], out=to[:, :300], **call)
    assert torch.equal(to[:, :300], want) and (to[:, 300:] == 9).all()


def test_no_tokens():
    s = batch(7, 0, 64, 100, 3, 4, "bf16", "f32")
    call = dict(x=s["x"], a=s["a"], b=s["b"], adapter_ids=s["ids"])
    assert opd.add_adapters(s["y"], **call)["out"].shape == (0, 100)
    d = opd.adapter_grads(s["y"], **call)
    assert (d["da"] == 0).all() and (d["db"] == 0).all() and d["dx"].shape == (0, 64)


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_rows(kind, ykind, value):
    s = batch(8, 90, 70, 140, 3, 16, kind, ykind, bad=False)
    call = dict(x=s["x"], a=s["a"], b=s["b"], adapter_ids=s["ids"], scales=s["scales"])
    want, dwant = opd.add_adapters(s["y"], **call)["out"], opd.adapter_grads(s["y"], **call)
    n = 37
    g = int(s["ids"][n])
    s["x"][n, 11] = value
    got = opd.add_adapters(s["y"], **call)["out"]
    others = torch.arange(90, device=DEV) != n
    assert torch.equal(got[others], want[others]) and not got[n].isfinite().any()
    d = opd.adapter_grads(s["y"], **call)
    mine = torch.arange(3, device=DEV) == g
    for k in ("da", "db"):
        assert torch.equal(d[k][~mine], dwant[k][~mine])
    assert torch.equal(d["dx"], dwant["dx"])
    # in dy: its own row of dx, its adapter's gradients
    s["x"][n, 11] = 1.0
    dwant = opd.adapter_grads(s["y"], **call)
    s["y"][n, 77] = value
    d = opd.adapter_grads(s["y"], **call)
    assert torch.equal(d["dx"][others], dwant["dx"][others]) and not d["dx"][n].isfinite().any()
    for k in ("da", "db"):
        assert torch.equal(d[k][~mine], dwant[k][~mine])
    keep = torch.arange(140, device=DEV) != 77
    assert torch.equal(d["db"][g][:, keep], dwant["db"][g][:, keep])


@pytest.mark.parametrize("which", ["x", "a", "b"])
def test_gradients_are_differences_of_the_forward(which):
    """out is linear in each of x, a and b: differences over any step, in fp32."""
    s = batch(9, 60, 40, 50, 3, 6, "f32", "f32")
    call = dict(adapter_ids=s["ids"], scales=s["scales"])
    args = {k: s[k] for k in ("x", "a", "b")}
    dy = torch.randn(60, 50, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    dy = aligned(dy)
    d = opd.adapter_grads(dy, **args, **call)["d" + which].double()
    zero = aligned(torch.zeros(60, 50, device=DEV))
    loss = lambda p: float((opd.add_adapters(zero, **{**args, which: p}, **call)["out"].double() *
                            dy.double()).sum())
    # the sum of magnitudes that roundings are relative to
    size = float((opd.add_adapters(zero, **{k: aligned(s[k].abs() + 1) for k in ("x", "a", "b")},
                                   **call)["out"].double() * dy.abs().double()).sum())
    rng = np.random.default_rng(2)
    for _ in range(6):
        at = tuple(int(rng.integers(0, n)) for n in args[which].shape)
        up, down = aligned(args[which]), aligned(args[which])
        up[at] += 1.0
        down[at] -= 1.0
        step = float(up[at].double() - down[at].double())
        # (sums of 40, then of 6: each addition off by a unit)
        assert abs((loss(up) - loss(down)) / step - float(d[at])) <= 64 * ref.ULP * size / abs(step)


@pytest.mark.parametrize("kind,ykind", KINDS)
@pytest.mark.parametrize("N", [1, 70])
def test_results_that_cancel_keep_their_bits(kind, ykind, N):
    """t (and u) = (1 + 2^-12 + 2^-20, -2^-12), which meet a -1: 2^-20 is left.  Exact, since
    every partial sum in any order is a multiple of 2^-20 below 2: 21 bits of the 24 of fp32."""
    put = lambda t, rows: aligned(torch.tensor(rows, dtype=DT[t], device=DEV))
    long = [1.0, 2.0 ** -12, 2.0 ** -20] + [0.0] * 13
    pick = [[[1.0] * 3 + [0.0] * 13, [0.0, -1.0] + [0.0] * 14]]
    ones = [[[1.0] * 40] * 2]
    ids = torch.zeros(N, dtype=torch.int32, device=DEV)
    y = put(ykind, [[-1.0] * 40] * N)
    out = opd.add_adapters(y, put(kind, [long] * N), put(kind, pick), put(kind, ones), ids)["out"]
    assert (out.double() == 2.0 ** -20).all()
    # the gradient of x, where the shared projection's is -1
    dx = opd.adapter_grads(put(ykind, [long] * N), put(kind, [[0.0] * 40] * N), put(kind, ones),
                           put(kind, pick), ids, dx=put(kind, [[-1.0] * 40] * N))["dx"]
    assert (dx.double() == 2.0 ** -20).all()


@pytest.mark.parametrize("N,r", [(40, 16), (130, 5)])
def test_adapters_of_a_head(N, r):
    """bf16 states and adapters, fp32 rows of a whole vocabulary: forward, and the gradients
    from the loss's dlogits."""
    check(batch(N, N, 136, 151_936, 3, r, "bf16", "f32"), "bf16", "f32")
