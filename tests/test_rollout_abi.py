"""Refusals of the blockwise calls and of the verification of drafts, without a
GPU: the C ABI's error codes (each case has one invalid argument and never
reaches a launch) and the binding's checks before it passes a pointer on."""
import pytest
import torch

import paper_2606_24143_amd as opd

OK, NULL, SHAPE, SUPPORT, DTYPE, ALIGN, WORKSPACE, PARAM = 0, -1, -2, -3, -4, -5, -6, -10
FAKE = 0x10000  # 16-byte aligned placeholder address, never dereferenced


def quantize(x=FAKE, dtype=1, N=4, H=256, ldx=None, rows=1, scale=0, q=FAKE, ldq=None,
             scales=FAKE):
    return opd.lib().opd_quantize_blocks(x, dtype, N, H, H if ldx is None else ldx, rows, scale, q,
                                         H if ldq is None else ldq, scales, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE),
    (dict(scale=2), DTYPE),
    (dict(scale=-1), DTYPE),
    (dict(N=-1), SHAPE),
    (dict(N=2 ** 31), SHAPE),
    (dict(H=0), SHAPE),
    (dict(H=2 ** 24 + 16), SHAPE),
    (dict(ldx=240), SHAPE),
    (dict(ldq=240), SHAPE),
    (dict(rows=0), PARAM),
    (dict(rows=64), PARAM),
    (dict(x=None), NULL),
    (dict(q=None), NULL),
    (dict(scales=None), NULL),
    (dict(x=FAKE + 8), ALIGN),
    (dict(q=FAKE + 4), ALIGN),
    (dict(scales=FAKE + 2), ALIGN),
    (dict(ldx=260), ALIGN),          # bf16 rows of 520 bytes
    (dict(dtype=0, ldx=258), ALIGN),  # fp32 rows of 1,032 bytes
    (dict(ldq=264), ALIGN),
])
def test_quantize_errors(kw, code):
    assert quantize(**kw) == code


def head(x=FAKE, ldx=None, sx=FAKE, w=FAKE, ldw=None, sw=FAKE, scale=0, N=4, V=1024, H=256,
         dtype=1, out=FAKE, ld=None):
    return opd.lib().opd_head_logits(x, H if ldx is None else ldx, sx, w, H if ldw is None else ldw,
                                     sw, scale, N, V, H, dtype, out, V if ld is None else ld, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE),
    (dict(scale=7), DTYPE),
    (dict(N=-1), SHAPE),
    (dict(N=2 ** 31), SHAPE),
    (dict(V=1), SHAPE),
    (dict(V=2 ** 31), SHAPE),
    (dict(V=2 ** 29 + 8, ld=2 ** 29 + 8), SHAPE),
    (dict(V=2 ** 30 + 8), SHAPE),
    (dict(H=0), SHAPE),
    (dict(ld=1000), SHAPE),
    (dict(H=2 ** 22 + 16), SHAPE),
    (dict(ldx=128), SHAPE),
    (dict(ldw=128), SHAPE),
    (dict(ldx=2 ** 22 + 16), SHAPE),
    (dict(ldw=2 ** 22 + 16), SHAPE),
    (dict(N=2 ** 30, V=2 ** 17, ld=2 ** 17), SHAPE),
    (dict(x=None), NULL),
    (dict(sx=None), NULL),
    (dict(w=None), NULL),
    (dict(sw=None), NULL),
    (dict(out=None), NULL),
    (dict(x=FAKE + 8), ALIGN),
    (dict(w=FAKE + 8), ALIGN),
    (dict(out=FAKE + 8), ALIGN),
    (dict(sx=FAKE + 1), ALIGN),
    (dict(sw=FAKE + 2), ALIGN),
    (dict(ldx=264), ALIGN),
    (dict(ldw=264), ALIGN),
    (dict(V=1020), ALIGN),
    (dict(V=1022, dtype=0), ALIGN),
])
def test_head_errors(kw, code):
    assert head(**kw) == code


def verify(z=FAKE, y=FAKE, dtype=1, B=4, D=3, V=1024, ld=None, ldd=None, ids=FAKE, lens=None,
           u=FAKE, mask=None, acc=FAKE, out=FAKE, logp=None, ws=FAKE, ws_bytes=1 << 20):
    return opd.lib().opd_verify_drafts(z, y, dtype, B, D, V, V if ld is None else ld,
                                       V if ldd is None else ldd, ids, lens, u, mask, acc, out,
                                       logp, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), DTYPE),
    (dict(D=0), SUPPORT),
    (dict(D=257), SUPPORT),
    (dict(B=-1), SHAPE),
    (dict(B=2 ** 31), SHAPE),
    (dict(B=2 ** 30, D=1), SHAPE),
    (dict(V=1), SHAPE),
    (dict(V=2 ** 31), SHAPE),
    (dict(ld=1016), SHAPE),
    (dict(ldd=1016), SHAPE),
    (dict(z=None), NULL),
    (dict(ids=None), NULL),
    (dict(u=None), NULL),
    (dict(acc=None), NULL),
    (dict(out=None), NULL),
    (dict(z=FAKE + 4), ALIGN),
    (dict(y=FAKE + 4), ALIGN),
    (dict(V=1020), ALIGN),
    (dict(ldd=1028), ALIGN),
    (dict(dtype=0, ldd=1026), ALIGN),
    (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 8), WORKSPACE),
    (dict(ws_bytes=64), WORKSPACE),
])
def test_verify_errors(kw, code):
    assert verify(**kw) == code


def test_nothing_to_do():
    assert quantize(N=0, x=None, q=None, scales=None) == OK
    assert head(N=0, x=None, sx=None, w=None, sw=None, out=None) == OK
    assert verify(B=0, z=None, ids=None, u=None, acc=None, out=None, ws=None, ws_bytes=0) == OK


def test_verify_workspace():
    ws = opd.lib().opd_verify_workspace_bytes
    assert ws(64, 5, 151936, 1) >= 64 * 11 * 8
    assert ws(64, 5, 151936, 1) % 8 == 0
    assert ws(128, 5, 151936, 1) > ws(64, 5, 151936, 1)
    for bad in ((0, 5, 100, 1), (4, 0, 100, 1), (4, 257, 100, 1), (4, 5, 1, 1), (4, 5, 100, 2)):
        assert ws(*bad) == 0


# ---------------------------------------------------------------- the binding

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def f8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8).view(E4M3)


@pytest.mark.parametrize("x,kw,match", [
    (torch.zeros(4, 256), {}, "GPU tensor"),
    (torch.zeros(4, 256), dict(block_rows=2), "block_rows"),
    (torch.zeros(4, 256), dict(scale_dtype=torch.bfloat16), "scale_dtype"),
    (torch.zeros(256), {}, "2-D"),
    (torch.zeros(256, 4).t(), {}, "unit column stride"),
    (torch.zeros(4, 257)[:, :256], {}, "16-byte"),
    (torch.zeros(4, 260)[:, 1:257], {}, "16-byte"),
])
def test_binding_refuses_quantize(x, kw, match):
    with pytest.raises(ValueError, match=match):
        opd.quantize_blocks(x, **kw)


def test_binding_refuses_dtypes():
    with pytest.raises(TypeError):
        opd.quantize_blocks(torch.zeros(4, 256, dtype=torch.float16))
    with pytest.raises(TypeError):
        opd.head_logits(torch.zeros(4, 256), torch.zeros(4, 2), f8(64, 256), torch.zeros(1, 2))
    with pytest.raises(TypeError):
        opd.verify_drafts(torch.zeros(8, 64, dtype=torch.float16),
                          torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 2))


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(hidden_scales=torch.zeros(4, 1)), "shape"),
    (dict(weight_scales=torch.zeros(2, 2)), "shape"),
    (dict(weight_scales=torch.zeros(1, 2, dtype=torch.uint8).view(E8M0)), "one dtype"),
    (dict(hidden_scales=torch.zeros(2, 4).t()), "contiguous"),
    (dict(hidden_scales=torch.zeros(4, 2, dtype=torch.bfloat16)), "dtype"),
    (dict(weight=f8(64, 128)), "weight must be"),
    (dict(hidden=f8(4, 264)[:, :256]), "16-byte"),
    (dict(dtype=torch.float16), "dtype must be"),
    (dict(out=torch.zeros(4, 64)), "out must have dtype"),
    (dict(out=torch.zeros(4, 32, dtype=torch.bfloat16)), "out must have shape"),
])
def test_binding_refuses_head(over, match):
    a = dict(hidden=f8(4, 256), hidden_scales=torch.zeros(4, 2), weight=f8(64, 256),
             weight_scales=torch.zeros(1, 2))
    a.update(over)
    with pytest.raises(ValueError, match=match):
        opd.head_logits(**a)


@pytest.mark.parametrize("over,match", [
    ({}, "GPU tensor"),
    (dict(target_logits=torch.zeros(11, 64)), "rows"),
    (dict(draft_ids=torch.zeros(4, 2, dtype=torch.int64)), "int32"),
    (dict(draft_ids=torch.zeros(4, 0, dtype=torch.int32)), "rows"),
    (dict(draft_ids=torch.zeros(2, 4, dtype=torch.int32).t()), "contiguous"),
    (dict(uniforms=torch.zeros(4, 2)), "shape"),
    (dict(uniforms=torch.zeros(4, 3, dtype=torch.float64)), "float32"),
    (dict(draft_logits=torch.zeros(8, 64, dtype=torch.bfloat16)), "draft_logits"),
    (dict(draft_logits=torch.zeros(12, 64)), "draft_logits"),
    (dict(draft_logits=torch.zeros(64, 8).t()), "unit column stride"),
    (dict(draft_lens=torch.zeros(4, dtype=torch.int64)), "int32"),
    (dict(mask=torch.zeros(4, dtype=torch.int32)), "dtype"),
    (dict(workspace=torch.zeros(64)), "dtype"),
])
def test_binding_refuses_verify(over, match):
    a = dict(target_logits=torch.zeros(12, 64), draft_ids=torch.zeros(4, 2, dtype=torch.int32),
             uniforms=torch.zeros(4, 3), draft_logits=torch.zeros(8, 64))
    a.update(over)
    with pytest.raises(ValueError, match=match):
        opd.verify_drafts(**a)
