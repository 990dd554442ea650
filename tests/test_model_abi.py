"""Refusals of the calls on token embeddings, adapters and beams, without a GPU: the C
ABI's error codes (each case has one invalid argument and never reaches a launch) and the
binding's checks before it passes a pointer on; workspace sizes; and the reference forms
that the GPU tests go by, against other ways to the same numbers."""
import numpy as np
import pytest
import torch

import model_ref as ref
import paper_2606_24143_amd as opd

OK, NULL, SHAPE, SUPPORT, DTYPE, ALIGN, WORKSPACE, PARAM = 0, -1, -2, -3, -4, -5, -6, -10
FAKE = 0x10000  # 16-byte aligned placeholder address, never dereferenced
OTHER = 0x20000


def embed(table=FAKE, dtype=1, V=1000, H=256, ld=None, ids=FAKE, N=4, out=FAKE, odt=1, ldo=None):
    return opd.lib().opd_embed_tokens(table, dtype, V, H, H if ld is None else ld, ids, N, 1.0, out,
                                      odt, H if ldo is None else ldo, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE),
    (dict(odt=-1), DTYPE),
    (dict(N=-1), SHAPE),
    (dict(N=2 ** 31), SHAPE),
    (dict(V=0), SHAPE),
    (dict(V=2 ** 31), SHAPE),
    (dict(H=0), SHAPE),
    (dict(H=2 ** 22 + 8), SHAPE),
    (dict(ld=248), SHAPE),
    (dict(ldo=248), SHAPE),
    (dict(table=None), NULL),
    (dict(ids=None), NULL),
    (dict(out=None), NULL),
    (dict(table=FAKE + 8), ALIGN),
    (dict(out=FAKE + 2), ALIGN),
    (dict(ld=260), ALIGN),             # bf16 rows of 520 bytes
    (dict(ldo=258, odt=0), ALIGN),     # fp32 rows of 1,032 bytes
])
def test_embed_errors(kw, code):
    assert embed(**kw) == code


def embed_grad(dy=FAKE, dtype=1, N=1000, H=256, ldy=None, ids=FAKE, V=500, out=FAKE, odt=0,
               ldo=None, acc=0, ws=FAKE, ws_bytes=1 << 30):
    return opd.lib().opd_embed_grads(dy, dtype, N, H, H if ldy is None else ldy, ids, V, 1.0, out,
                                     odt, H if ldo is None else ldo, acc, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), DTYPE),
    (dict(odt=2), DTYPE),
    (dict(N=-1), SHAPE),
    (dict(V=0), SHAPE),
    (dict(H=0), SHAPE),
    (dict(ldy=128), SHAPE),
    (dict(ldo=128), SHAPE),
    (dict(acc=2), PARAM),
    (dict(dy=None), NULL),
    (dict(ids=None), NULL),
    (dict(out=None), NULL),
    (dict(dy=FAKE + 4), ALIGN),
    (dict(out=FAKE + 4), ALIGN),
    (dict(ldy=257), ALIGN),
    (dict(ldo=257), ALIGN),
    (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 8), WORKSPACE),
    (dict(ws_bytes=1000), WORKSPACE),
    (dict(V=2 ** 31 - 1), SHAPE),              # more workgroups than a launch has
    (dict(V=2 ** 31 - 512), WORKSPACE),
])
def test_embed_grad_errors(kw, code):
    assert embed_grad(**kw) == code


def adapt(y=FAKE, ydt=1, ldy=None, x=FAKE, dtype=1, ldx=None, a=FAKE, lda=None, b=FAKE, ldb=None,
          ids=FAKE, N=100, H=256, O=512, G=4, r=8, out=OTHER, ldo=None, ws=FAKE, ws_bytes=1 << 30):
    return opd.lib().opd_add_adapters(
        y, ydt, O if ldy is None else ldy, x, dtype, H if ldx is None else ldx, a,
        H if lda is None else lda, b, O if ldb is None else ldb, None, ids, N, H, O, G, r, out,
        O if ldo is None else ldo, None, ws, ws_bytes, None)


def adapt_grad(dy=FAKE, ydt=1, ldy=None, x=FAKE, dtype=1, ldx=None, a=FAKE, lda=None, b=FAKE,
               ldb=None, ids=FAKE, N=100, H=256, O=512, G=4, r=8, dxs=None, ldds=0, dx=FAKE,
               lddx=None, da=FAKE, ldda=None, db=FAKE, lddb=None, ws=FAKE, ws_bytes=1 << 30):
    return opd.lib().opd_adapter_grads(
        dy, ydt, O if ldy is None else ldy, x, dtype, H if ldx is None else ldx, a,
        H if lda is None else lda, b, O if ldb is None else ldb, None, ids, N, H, O, G, r, None,
        dxs, ldds, dx, H if lddx is None else lddx, da, H if ldda is None else ldda, db,
        O if lddb is None else lddb, ws, ws_bytes, None)


ADAPTER_ERRORS = [
    (dict(dtype=2), DTYPE),
    (dict(ydt=2), DTYPE),
    (dict(dtype=0, ydt=1), DTYPE),     # fp32 adapters beside bf16 rows
    (dict(N=-1), SHAPE),
    (dict(N=2 ** 24 + 1), SHAPE),
    (dict(H=0), SHAPE),
    (dict(O=2 ** 22 + 8), SHAPE),
    (dict(ldx=128), SHAPE),
    (dict(ldy=256), SHAPE),
    (dict(lda=128), SHAPE),
    (dict(ldb=256), SHAPE),
    (dict(G=0), SUPPORT),
    (dict(G=1001), SUPPORT),
    (dict(r=0), SUPPORT),
    (dict(r=129), SUPPORT),
    (dict(x=None), NULL),
    (dict(a=None), NULL),
    (dict(b=None), NULL),
    (dict(ids=None), NULL),
    (dict(x=FAKE + 8), ALIGN),
    (dict(a=FAKE + 8), ALIGN),
    (dict(b=FAKE + 8), ALIGN),
    (dict(ldx=260), ALIGN),
    (dict(lda=260), ALIGN),
    (dict(ldb=516), ALIGN),
    (dict(ldy=516), ALIGN),
    (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 8), WORKSPACE),
    (dict(ws_bytes=100), WORKSPACE),
]


@pytest.mark.parametrize("call", [adapt, adapt_grad])
@pytest.mark.parametrize("kw,code", ADAPTER_ERRORS)
def test_adapter_errors(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("call,kw,code", [
    (adapt, dict(y=None), NULL),
    (adapt, dict(out=None), NULL),
    (adapt, dict(y=FAKE + 8), ALIGN),
    (adapt, dict(out=FAKE + 8), ALIGN),
    (adapt, dict(ldo=256), SHAPE),
    (adapt, dict(ldo=516), ALIGN),
    (adapt, dict(out=FAKE, ldo=520), SHAPE),   # in place, another stride
    # (too many to launch at once: 1,000 adapters' sums of 2^22 columns)
    (adapt_grad, dict(G=1000, O=2 ** 22), SHAPE),
    (adapt_grad, dict(dy=None), NULL),
    (adapt_grad, dict(da=None), NULL),
    (adapt_grad, dict(db=None), NULL),
    (adapt_grad, dict(dxs=FAKE, ldds=256, dx=None), NULL),
    (adapt_grad, dict(dxs=FAKE, ldds=128), SHAPE),
    (adapt_grad, dict(dxs=FAKE, ldds=264), SHAPE),  # in place, another stride
    (adapt_grad, dict(lddx=128), SHAPE),
    (adapt_grad, dict(ldda=128), SHAPE),
    (adapt_grad, dict(lddb=256), SHAPE),
    (adapt_grad, dict(dx=FAKE + 8), ALIGN),
    (adapt_grad, dict(da=FAKE + 8), ALIGN),
    (adapt_grad, dict(ldda=258), ALIGN),
    (adapt_grad, dict(lddb=514), ALIGN),
])
def test_more_adapter_errors(call, kw, code):
    assert call(**kw) == code


def beam(z=FAKE, dtype=1, B=4, W=4, V=1024, ld=None, scores=FAKE, k=4, out=FAKE, parents=FAKE,
         ids=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return opd.lib().opd_beam_select(z, dtype, B, W, V, V if ld is None else ld, scores, None, k,
                                     out, parents, ids, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE),
    (dict(B=-1), SHAPE),
    (dict(B=2 ** 31), SHAPE),
    (dict(B=2 ** 30), SHAPE),
    (dict(V=1), SHAPE),
    (dict(ld=1000), SHAPE),
    (dict(W=0), SUPPORT),
    (dict(W=65), SUPPORT),
    (dict(k=0), SUPPORT),
    (dict(k=65), SUPPORT),
    (dict(z=None), NULL),
    (dict(scores=None), NULL),
    (dict(out=None), NULL),
    (dict(parents=None), NULL),
    (dict(ids=None), NULL),
    (dict(z=FAKE + 8), ALIGN),
    (dict(V=1020), ALIGN),
    (dict(V=1022, dtype=0), ALIGN),
    (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 8), WORKSPACE),
    (dict(ws_bytes=64), WORKSPACE),
])
def test_beam_errors(kw, code):
    assert beam(**kw) == code


def move(states=FAKE, B=2, W=4, outer=3, inner=64, stride=256, apart=64, parents=FAKE, k=4,
         out=OTHER, to_stride=256, to_apart=64):
    return opd.lib().opd_reorder_beams(states, B, W, outer, inner, stride, apart, parents, k, out,
                                       to_stride, to_apart, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), SHAPE),
    (dict(outer=-1), SHAPE),
    (dict(inner=-1), SHAPE),
    (dict(inner=2 ** 41, apart=2 ** 42, to_apart=2 ** 42), SHAPE),
    (dict(stride=-256), SHAPE),
    (dict(apart=32), SHAPE),
    (dict(to_apart=32), SHAPE),
    (dict(W=0), SUPPORT),
    (dict(W=65), SUPPORT),
    (dict(k=0), SUPPORT),
    (dict(k=65), SUPPORT),
    (dict(states=None), NULL),
    (dict(parents=None), NULL),
    (dict(out=None), NULL),
    (dict(out=FAKE, k=3), SHAPE),             # in place, fewer states
    (dict(out=FAKE, to_stride=512), SHAPE),   # in place, another stride
    (dict(out=FAKE, to_apart=80), SHAPE),
    (dict(to_stride=0), SHAPE),               # states of out on top of each other
    (dict(outer=1, to_stride=48), SHAPE),
    (dict(outer=2, to_stride=64, to_apart=64), SHAPE),
    (dict(outer=2, to_stride=48, to_apart=1 << 20), SHAPE),
    (dict(outer=2, to_stride=64, to_apart=1 << 20, parents=None), NULL),  # slices apart: sound
])
def test_reorder_errors(kw, code):
    assert move(**kw) == code


def test_nothing_to_do():
    assert embed(N=0, table=None, ids=None, out=None) == OK
    assert embed_grad(N=0, dy=None, ids=None, acc=1, ws=None, ws_bytes=0) == OK
    assert adapt(N=0, y=None, x=None, ids=None, out=None, ws=None, ws_bytes=0) == OK
    assert beam(B=0, z=None, scores=None, out=None, parents=None, ids=None, ws=None) == OK
    assert move(B=0, states=None, parents=None, out=None) == OK
    assert move(outer=0, states=None, parents=None, out=None) == OK
    assert move(inner=0, states=None, parents=None, out=None) == OK


def test_workspaces():
    L = opd.lib()
    e = L.opd_embed_workspace_bytes
    assert e(7, 32000, 1000) == 0                       # few tokens are not sorted
    assert e(8192, 32000, 1000) >= 4 * (32001 + 8192) + 128 * 2 * 1000 * 4
    assert e(8192, 0, 1000) == 0 and e(-1, 10, 10) == 0
    a = L.opd_adapter_workspace_bytes
    assert 0 < a(64, 4096, 32000, 32, 16, 1, 1, 0) < a(64, 4096, 32000, 32, 16, 1, 1, 1)
    assert a(64, 4096, 32000, 0, 16, 1, 1, 0) == 0
    assert a(64, 4096, 32000, 4, 129, 1, 1, 0) == 0
    assert a(64, 4096, 32000, 4, 16, 0, 1, 0) == 0
    b = L.opd_beam_workspace_bytes
    assert b(4, 8, 32000, 1) >= 4 * 8 * 64 * 8
    assert b(0, 8, 32000, 1) == 0 and b(4, 65, 32000, 1) == 0 and b(4, 8, 1, 1) == 0


# ---------------------------------------------------------------- the binding

I32 = torch.int32


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(table=torch.zeros(256)), "2-D"),
    (dict(table=torch.zeros(256, 10).t()), "unit column stride"),
    (dict(table=torch.zeros(10, 257)[:, :256]), "16-byte"),
    (dict(ids=torch.zeros(4, dtype=torch.int64)), "int32"),
    (dict(ids=torch.zeros(2, 2, dtype=I32)), "int32"),
    (dict(ids=torch.zeros(8, dtype=I32)[::2]), "contiguous"),
    (dict(dtype=torch.float16), "dtype must be"),
    (dict(out=torch.zeros(3, 256)), "out must be"),
    (dict(out=torch.zeros(4, 256, dtype=torch.bfloat16)), "out must be"),
    (dict(out=torch.zeros(4, 257)[:, 1:]), "16-byte"),
])
def test_binding_refuses_embed(over, match):
    args = dict(table=torch.zeros(10, 256), ids=torch.zeros(4, dtype=I32))
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.embed_tokens(args.pop("table"), args.pop("ids"), **args)


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(grad=torch.zeros(4, 257)[:, :256]), "16-byte"),
    (dict(ids=torch.zeros(5, dtype=I32)), "shape"),
    (dict(ids=torch.zeros(4)), "int32"),
    (dict(V=0), "V must be"),
    (dict(V=2 ** 31), "V must be"),
    (dict(dtype=torch.float64), "dtype must be"),
    (dict(accumulate=True), "accumulate"),
    (dict(out=torch.zeros(9, 256)), "out must be"),
    (dict(workspace=torch.zeros(4)), "dtype"),
])
def test_binding_refuses_embed_grads(over, match):
    args = dict(grad=torch.zeros(4, 256), ids=torch.zeros(4, dtype=I32), V=10)
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.embed_grads(args.pop("grad"), args.pop("ids"), args.pop("V"), **args)


def adapters():
    return dict(x=torch.zeros(6, 64), a=torch.zeros(3, 5, 64), b=torch.zeros(3, 5, 32),
                adapter_ids=torch.zeros(6, dtype=I32))


SHARED = [
    ({}, "GPU tensor"),
    (dict(x=torch.zeros(6, 65)[:, :64]), "16-byte"),
    (dict(x=torch.zeros(64, 6).t()), "unit column stride"),
    (dict(a=torch.zeros(3, 4, 64)), "a must have shape"),
    (dict(a=torch.zeros(3, 5, 60)), "a must have shape"),
    (dict(a=torch.zeros(3, 5, 64, dtype=torch.bfloat16)), "a must be"),
    (dict(a=torch.zeros(3, 64, 5).transpose(1, 2)), "row stride"),
    (dict(a=torch.zeros(3, 6, 64)[:, :5]), "row stride"),   # adapters more than r rows apart
    (dict(b=torch.zeros(3, 5)), "b must be a"),
    (dict(b=torch.zeros(3, 5, 33)[:, :, :32]), "row stride"),
    (dict(adapter_ids=torch.zeros(5, dtype=I32)), "shape"),
    (dict(adapter_ids=torch.zeros(6, dtype=torch.int64)), "int32"),
    (dict(scales=torch.zeros(2)), "shape"),
    (dict(scales=torch.zeros(3, dtype=torch.float64)), "float32"),
    (dict(workspace=torch.zeros(4)), "dtype"),
]


@pytest.mark.parametrize("over,match", SHARED + [
    (dict(y=torch.zeros(6, 31)), "y must have"),
    (dict(y=torch.zeros(6, 33)[:, :32]), "16-byte"),
    (dict(y=torch.zeros(6, 32, dtype=torch.bfloat16)), "y must be"),
    (dict(out=torch.zeros(6, 36)), "out must be"),
])
def test_binding_refuses_add_adapters(over, match):
    args = dict(adapters(), y=torch.zeros(6, 32))
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.add_adapters(**args)


@pytest.mark.parametrize("over,match", SHARED + [
    (dict(dy=torch.zeros(5, 32)), "dy must have"),
    (dict(low=torch.zeros(6, 4)), "shape"),
    (dict(low=torch.zeros(6, 5, dtype=torch.bfloat16)), "float32"),
    (dict(dx=torch.zeros(6, 32)), "dx must be"),
    (dict(dx=torch.zeros(6, 64), want_dx=False), "not wanted"),
])
def test_binding_refuses_adapter_grads(over, match):
    args = dict(adapters(), dy=torch.zeros(6, 32))
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.adapter_grads(**args)


def test_binding_refuses_a_result_on_its_inputs():
    table, ids = torch.zeros(6, 16), torch.zeros(4, dtype=I32)
    with pytest.raises(ValueError, match="overlap"):
        opd.embed_tokens(table, ids, out=table[2:])
    with pytest.raises(ValueError, match="overlap"):
        opd.embed_grads(table[:4], ids, 4, out=table[1:5])
    s = adapters()
    buf = torch.zeros(3 * 2 * 32)
    b = buf.view(3, 2, 32)
    with pytest.raises(ValueError, match="overlap"):
        opd.add_adapters(torch.zeros(6, 32), s["x"], torch.zeros(3, 2, 64), b, s["adapter_ids"],
                         out=buf.view(6, 32))


def test_binding_refuses_an_overlap():
    buf = torch.zeros(7, 32)
    with pytest.raises(ValueError, match="overlap"):
        opd.add_adapters(buf[:6], adapters()["x"], adapters()["a"], adapters()["b"],
                         adapters()["adapter_ids"], out=buf[1:])


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(logits=torch.zeros(7, 64)), "rows"),
    (dict(scores=torch.zeros(8)), "scores must be"),
    (dict(scores=torch.zeros(2, 4, dtype=torch.float64)), "float32"),
    (dict(logits=torch.zeros(130, 64), scores=torch.zeros(2, 65)), "W up to"),
    (dict(k=0), "k must be"),
    (dict(k=65), "k must be"),
    (dict(finished=torch.zeros(2, 4)), "dtype"),
    (dict(finished=torch.zeros(4, 2, dtype=torch.bool)), "shape"),
    (dict(workspace=torch.zeros(4)), "dtype"),
])
def test_binding_refuses_beam_select(over, match):
    args = dict(logits=torch.zeros(8, 64), scores=torch.zeros(2, 4))
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.beam_select(args.pop("logits"), args.pop("scores"), **args)


BUFFER = torch.zeros(12, 16)


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(parents=torch.zeros(2, 4)), "int32"),
    (dict(parents=torch.zeros(8, dtype=I32)), "parents must be"),
    (dict(parents=torch.zeros(2, 65, dtype=I32)), "k must be"),
    (dict(states=torch.zeros(7, 16)), "B \\* W"),
    (dict(states=torch.zeros(2 * 65, 16)), "W up to"),
    (dict(states=torch.zeros(1, 16).expand(8, 16)), "overlap"),
    (dict(states=torch.zeros(8, 5, 4, 6)[:, :4, :3, :5]), "evenly"),
    (dict(out=torch.zeros(8, 15)), "out must be"),
    (dict(out=torch.zeros(8, 16, dtype=torch.int32)), "out must be"),
    (dict(states=BUFFER[:8], out=BUFFER[4:]), "overlap"),
    (dict(states=BUFFER[:8], out=BUFFER[:8].view(8, 16).flip(0).flip(0)[:6]), "out must be"),
])
def test_binding_refuses_reorder(over, match):
    args = dict(states=torch.zeros(8, 16), parents=torch.zeros(2, 4, dtype=I32))
    args.update(over)
    with pytest.raises(ValueError, match=match):
        opd.reorder_beams(args.pop("states"), args.pop("parents"), **args)


def test_binding_refuses_dtypes():
    for call in (lambda t: opd.embed_tokens(t, torch.zeros(1, dtype=I32)),
                 lambda t: opd.embed_grads(t, torch.zeros(4, dtype=I32), 5),
                 lambda t: opd.beam_select(t, torch.zeros(1, 4))):
        with pytest.raises(TypeError):
            call(torch.zeros(4, 64, dtype=torch.float16))


# ---------------------------------------------------------------- the reference forms

def test_reference_gradients_are_differences_of_the_reference():
    """The adapters' map is linear in each of x, a and b alone, the embedding's in its
    table: central differences are exact but for 64-bit rounding."""
    rng = np.random.default_rng(3)
    N, H, O, G, r = 7, 5, 6, 3, 2
    x, y, dy = rng.normal(size=(N, H)), rng.normal(size=(N, O)), rng.normal(size=(N, O))
    a, b, s = rng.normal(size=(G, r, H)), rng.normal(size=(G, r, O)), rng.uniform(0.5, 2, G)
    ids = np.array([0, 2, -1, 0, 2, 2, -1])
    d = ref.adapter_grads(dy, x, a, b, ids, s, "f32", "f32")
    loss = lambda: float((ref.adapters(y, x, a, b, ids, s, "f32", "f32")[0] * dy).sum())
    for name, p in (("dx", x), ("da", a), ("db", b)):
        for at in np.ndindex(p.shape):
            keep = p[at]
            p[at] = keep + 1.0
            up = loss()
            p[at] = keep - 1.0
            assert abs((up - loss()) / 2 - d[name][0][at]) < 1e-11
            p[at] = keep
    table, tok, g = rng.normal(size=(4, H)), np.array([1, 3, -1, 1]), rng.normal(size=(4, H))
    want, _ = ref.embed_grads(g, tok, 4, 1.5)
    for at in np.ndindex(table.shape):
        up, down = table.copy(), table.copy()
        up[at] += 1.0
        down[at] -= 1.0
        diff = ((ref.embed(up, tok, 1.5) - ref.embed(down, tok, 1.5)) * g).sum() / 2
        assert abs(diff - want[at]) < 1e-12


def test_reference_beams_are_the_best_of_all_candidates():
    rng = np.random.default_rng(4)
    z, s = rng.normal(size=(3, 4, 11)), rng.normal(size=(3, 4))
    out, parents, ids, _ = ref.beams(z, s, 6)
    for b in range(3):
        p = np.log(np.exp(z[b]) / np.exp(z[b]).sum(1, keepdims=True)) + s[b][:, None]
        best = np.argsort(-p.ravel())[:6]
        assert np.array_equal(parents[b], best // 11) and np.array_equal(ids[b], best % 11)
        assert np.allclose(out[b], p.ravel()[best], atol=1e-12)
