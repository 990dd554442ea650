"""Blockwise quantisation and the head's product on the GPU against 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2606_24143_amd as opd
import rollout_ref as ref
from gpu_common import DEV, say

pytestmark = pytest.mark.gpu

SCALES = {"f32": torch.float32, "e8m0": torch.float8_e8m0fnu}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24  # half a step of fp32


def strided(x, dtype, to=8, fill=float("nan")):
    """x on the GPU as a view of wider rows that hold `fill` past it."""
    n, h = x.shape
    buf = torch.full((n, (h + to - 1) // to * to + to), fill, dtype=torch.float32, device=DEV)
    buf[:, :h] = torch.as_tensor(x, device=DEV)
    return buf.to(dtype)[:, :h]


def rows_for(kind, N, H, seed):
    g = np.random.default_rng(seed)
    x = g.normal(0, 1, (N, H)).astype(np.float32)
    if kind == "ties":  # small integers over a power of two: many quotients are ties
        x = g.integers(-255, 256, (N, H)).astype(np.float32) * np.float32(2.0 ** -5)
    elif kind == "wide":
        x *= np.exp2(g.integers(-120, 100, (N, 1))).astype(np.float32)
    elif kind == "tiny":
        x *= np.float32(2.0 ** -130)
    elif kind == "zeros":
        x[g.random((N, H)) < 0.5] = 0
        x[:, :min(H, 128)] = 0
    elif kind == "bad":
        x[0, H // 2] = np.nan
        x[N - 1, 0] = -np.inf
        x[N // 2, H - 1] = np.inf
    return torch.from_numpy(x)


@pytest.mark.parametrize("kind", ["plain", "ties", "wide", "tiny", "zeros", "bad"])
@pytest.mark.parametrize("N,H", [(1, 1), (3, 127), (5, 128), (2, 129), (130, 200), (128, 384),
                                 (257, 1000)])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_is_exact(kind, N, H, rows, scale, dtype):
    x = rows_for(kind, N, H, N * 1000 + H).to(DT[dtype])
    want_q, want_s = ref.quantize(x.double().numpy(), rows, scale == "e8m0")
    out = opd.quantize_blocks(strided(x.float().numpy(), DT[dtype]), block_rows=rows,
                              scale_dtype=SCALES[scale])
    torch.cuda.synchronize()
    s = out["scales"]
    if scale == "e8m0":
        e = s.view(torch.uint8).cpu().numpy().astype(np.float64)
        got_s = np.where(e == 255, np.nan, np.exp2(e - 127))
    else:
        got_s = s.double().cpu().numpy()
    got_q = out["q"].double().cpu().numpy()
    assert np.array_equal(got_s, want_s, equal_nan=True)
    assert np.array_equal(got_q, want_q, equal_nan=True)
    assert out["q"].shape == (N, H) and out["q"].stride(0) % 16 == 0


def quantized(x, rows, scale):
    """(q, scales on the GPU; their values in float64)."""
    vq, vs = ref.quantize(x, rows, scale == "e8m0")
    q = strided(vq.astype(np.float32), torch.float8_e4m3fn, 16)
    if scale == "f32":
        s = torch.from_numpy(vs.astype(np.float32)).to(DEV)
    else:
        s = torch.from_numpy((np.log2(vs) + 127).astype(np.uint8)).to(DEV).view(
            torch.float8_e8m0fnu)
    return q, s, vq, vs


def head_tolerance(mags, z, H, out, x, sx, w, sw):
    """fp32 sums: every term passes at most 128 additions inside its block (a step
    each, should the matrix core truncate) and one rounding of the scales'
    product, one of the scaled sum and one addition per block outside, each half a
    step of at most the sum of the terms' magnitudes.

    bf16 logits: the 8-bit instructions cut each product at 2^-13 of the largest
    they sum it with, which is at most a block's largest x times its largest w:
    128 products a block, so 2^-6 of that in all; then the output's rounding."""
    t = (2 * 128 + 3 + ref.blocks(H, ref.BLOCK)) * U32 * mags
    if out == "bf16":
        for b in range(sx.shape[1]):
            cols = np.s_[:, b * 128:(b + 1) * 128]
            largest = np.abs(w[cols]).max(1) * np.repeat(sw[:, b], 128)[:w.shape[0]]
            t = t + 2.0 ** -6 * np.outer(np.abs(x[cols]).max(1) * sx[:, b], largest)
        t = t + (np.abs(z) + t) * 2.0 ** -8
    return t + 1e-30


@pytest.mark.parametrize("N,V,H", [
    (1, 2, 1), (1, 130, 128), (2, 257, 129), (5, 1000, 640), (15, 333, 1000), (16, 2048, 256),
    (17, 129, 384), (33, 515, 2000), (63, 700, 384), (64, 1030, 512), (65, 256, 257),
    (100, 1537, 768), (128, 384, 128), (129, 260, 1024), (200, 3001, 896), (256, 512, 2048),
    (257, 1025, 272), (300, 2050, 1152), (520, 777, 640),
    (600, 30011, 272), (300, 515, 7), (260, 300, 135), (150, 777, 1001), (31, 4100, 333),
    (100, 640, 2047), (16, 13001, 384), (40, 25003, 256), (90, 30000, 640),
    (129, 108701, 130), (257, 54501, 200), (1000, 14100, 7), (14001, 1000, 384), (4100, 3500, 2047),
    (700, 20100, 16), (300, 50001, 1008)])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_head_logits(N, V, H, scale, out):
    g = np.random.default_rng(N + V + H)
    # (rows of unequal size, and blocks of unequal scale)
    x = g.normal(0, 1, (N, H)) * np.exp(g.normal(0, 1, (N, 1)))
    x[:, :H // 3] *= 30
    w = g.normal(0, 0.02, (V, H)) * np.exp(g.normal(0, 0.5, (V, 1)))
    x, sx, vx, vsx = quantized(x.astype(np.float32), 1, scale)
    w, sw, vw, vsw = quantized(w.astype(np.float32), 128, scale)
    z, mags = ref.head(vx, vsx, vw, vsw)
    buf = torch.full((N, (V + 7) // 8 * 8 + 8), 777.0, dtype=DT[out], device=DEV)
    got = opd.head_logits(x, sx, w, sw, dtype=DT[out], out=buf)["logits"]
    again = opd.head_logits(x, sx, w, sw, dtype=DT[out])["logits"]
    torch.cuda.synchronize()
    err = np.abs(got.double().cpu().numpy() - z)
    tol = head_tolerance(mags, z, H, out, vx, vsx, vw, vsw)
    # (and of the whole: half a step of bf16, or a hundredth of the worst fp32 sum)
    off = np.linalg.norm(err) / np.linalg.norm(z)
    assert off <= (2.0 ** -8 if out == "bf16" else 2.6 * U32 * np.linalg.norm(mags) /
                   np.linalg.norm(z)), off
    say("head %d x %d x %d %s %s: worst err / tolerance %.3g" % (N, V, H, scale, out,
                                                              (err / tol).max()))
    assert (err <= tol).all()
    assert torch.equal(got, again)
    assert (buf[:, V:] == 777.0).all(), "columns past V are not written"


@pytest.mark.parametrize("N,V,H", [(1, 100, 9), (20, 300, 130), (128, 700, 255), (260, 300, 135),
                                   (300, 1000, 2047), (130, 515, 15), (300, 50001, 135),
                                   (14100, 1000, 255), (1000, 14100, 2047)])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_what_lies_past_a_row_is_not_used(N, V, H, scale, out):
    g = np.random.default_rng(6)
    x, sx, _, _ = quantized(g.normal(0, 1, (N, H)).astype(np.float32), 1, scale)
    w, sw, _, _ = quantized(g.normal(0, 1, (V, H)).astype(np.float32), 128, scale)

    def padded(q, fill, extra):
        buf = torch.full((q.shape[0], (H + 15) // 16 * 16 + extra), fill, dtype=torch.uint8,
                         device=DEV)
        buf[:, :H] = q.contiguous().view(torch.uint8)
        return buf.view(torch.float8_e4m3fn)[:, :H]

    z = [opd.head_logits(padded(x, f, e), sx, padded(w, f, e), sw, dtype=DT[out])["logits"]
         for f, e in ((0, 0), (0x7F, 0), (0xFF, 32), (0x38, 16))]
    torch.cuda.synchronize()
    assert torch.isfinite(z[0]).all()
    for other in z[1:]:
        assert torch.equal(other, z[0])


@pytest.mark.parametrize("N", [1, 40, 300, 50000])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_head_keeps_nan_to_its_rows(N, scale, out):
    V, H = 300, 400
    g = np.random.default_rng(5)
    x, sx, vx, vsx = quantized(g.normal(0, 1, (N, H)).astype(np.float32), 1, scale)
    w, sw, vw, vsw = quantized(g.normal(0, 1, (V, H)).astype(np.float32), 128, scale)
    want = opd.head_logits(x, sx, w, sw, dtype=DT[out])["logits"].clone()
    assert torch.isfinite(want).all()
    n, v, block = N // 2, 77, 2  # a value of one token, one of a head row, a scale of 128 rows
    x = x.clone()
    w = torch.as_strided(w.clone(), (V, H), (400, 1)) if w.stride(0) == 400 else w
    xb, wb = x.contiguous().view(torch.uint8).clone(), w.contiguous().view(torch.uint8).clone()
    xb[n, 399] = 0x7F
    wb[v, 0] = 0xFF
    sw2 = sw.clone()
    if scale == "f32":
        sw2[block, 1] = float("nan")
    else:
        sw2.view(torch.uint8)[block, 1] = 255
    got = opd.head_logits(xb.view(torch.float8_e4m3fn), sx, wb.view(torch.float8_e4m3fn), sw2,
                          dtype=DT[out])["logits"]
    torch.cuda.synchronize()
    bad = torch.zeros(N, V, dtype=torch.bool, device=DEV)
    bad[n] = True
    bad[:, v] = True
    bad[:, block * 128:] = True
    assert torch.isnan(got[bad]).all()
    assert torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("H", [100, 135, 272, 400])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_edges_of_tiles(H, scale, out):
    """A token's logits are the same in a tile that it shares with any number of
    others, and an entry's in one that the vocabulary ends in anywhere."""
    N, V = 512, 54784  # (tiles of 256 by 256 from 257 tokens and 54,500 entries on)
    g = np.random.default_rng(9)
    x, sx, _, _ = quantized(g.normal(0, 1, (N, H)).astype(np.float32), 1, scale)
    w, sw, _, _ = quantized(g.normal(0, 1, (V, H)).astype(np.float32), 128, scale)
    want = opd.head_logits(x, sx, w, sw, dtype=DT[out])["logits"]
    buf = torch.empty(N, V, dtype=DT[out], device=DEV)
    for n in range(257, 513):
        buf.fill_(777.0)
        got = opd.head_logits(x[:n], sx[:n], w, sw, dtype=DT[out], out=buf[:n])["logits"]
        assert torch.equal(got, want[:n]) and (buf[n:] == 777.0).all(), n
    for v in range(V - 256, V):
        buf.fill_(777.0)
        opd.head_logits(x[:257], sx[:257], w[:v], sw[:(v + 127) // 128], dtype=DT[out],
                        out=buf[:257])
        assert torch.equal(buf[:257, :v], want[:257, :v]) and (buf[:257, v:] == 777.0).all(), v
    assert torch.isfinite(want).all()


def test_no_rows():
    w, sw, _, _ = quantized(np.ones((64, 128), np.float32), 128, "f32")
    x = torch.empty(0, 128, dtype=torch.float8_e4m3fn, device=DEV)
    out = opd.head_logits(x, torch.empty(0, 1, device=DEV), w, sw)["logits"]
    assert out.shape == (0, 64)
    q = opd.quantize_blocks(torch.empty(0, 128, device=DEV))
    assert q["q"].shape == (0, 128) and q["scales"].shape == (0, 1)


@pytest.mark.parametrize("rows", [1, 128])
def test_rows_past_4_gib(rows):
    """Offsets that pass 32 bits in the rows and in the values."""
    N, H = (1 << 22) + 128 + 5, 1024
    x = torch.zeros(N, H, dtype=torch.bfloat16, device=DEV)
    x[-133:] = torch.randn(133, H, device=DEV, generator=torch.Generator(DEV).manual_seed(4))
    out = opd.quantize_blocks(x, block_rows=rows)
    alone = opd.quantize_blocks(x[-133:], block_rows=rows)
    assert torch.equal(out["q"][-133:].view(torch.uint8), alone["q"].view(torch.uint8))
    assert torch.equal(out["scales"][-alone["scales"].shape[0]:], alone["scales"])
    assert (out["q"][:-133].view(torch.uint8) == 0).all()


def test_logits_past_4_gib():
    """Rows whose offsets pass 32 bits, in the weights' rows and in the logits."""
    N, V, H = 1100, 1 << 21, 128
    g = torch.Generator(DEV).manual_seed(3)
    w = torch.randint(0, 0x70, (V, H), dtype=torch.uint8, device=DEV, generator=g)
    buf = torch.zeros(V, 2176, dtype=torch.uint8, device=DEV)  # 4.25 GiB of rows
    buf[:, :H] = w
    w8 = buf.view(torch.float8_e4m3fn)[:, :H]
    x = torch.randint(0, 0x70, (N, H), dtype=torch.uint8, device=DEV, generator=g)
    x8 = x.view(torch.float8_e4m3fn)
    sw = torch.ones(V // 128, 1, device=DEV)
    z = opd.head_logits(x8, torch.ones(N, 1, device=DEV), w8, sw)["logits"]
    for n, v in ((0, 0), (N - 1, V - 1), (N - 1, 0), (N // 2, V // 2 + 5)):
        want = (x8[n].double() * w8[v].double()).sum()
        assert abs(float(z[n, v]) - float(want)) <= float(want) * (2.0 ** -8 + 300 * U32)
