"""The bytes of blockwise quantisation: a zero keeps its sign, whatever lies beside
it, and every value that rounds to zero has its own."""
import numpy as np
import pytest
import torch

import paper_2606_24143_amd as opd
import rollout_ref as ref
from test_gpu_head import DT, SCALES, strided


def bytes_of(q, x):
    """The e4m3 bytes of values q with the signs of x."""
    q = np.copysign(np.abs(q), x).astype(np.float32)
    return torch.from_numpy(q).to(torch.float8_e4m3fn).view(torch.uint8)


def test_signs_of_zeros_have_bytes_of_their_own():
    assert bytes_of(np.zeros(2), np.float32([0.0, -0.0])).tolist() == [0x00, 0x80]
    assert bytes_of(np.float64([448.0, 2.0 ** -9]), np.float32([-1, -1])).tolist() == [0xFE, 0x81]


def signed(N, H, beside, seed):
    """Values with zeros of both signs and values that round to zero, in blocks
    of ordinary scale; `beside` them blocks of other kinds."""
    g = np.random.default_rng(seed)
    x = g.normal(0, 1, (N, H)).astype(np.float32)
    x[g.random((N, H)) < 0.3] *= 0.0  # (both signs)
    small = g.random((N, H)) < 0.2
    x[small] *= np.float32(2.0 ** -14)
    x[g.random((N, H)) < 0.05] = np.float32(-1e-42)
    if beside != "ordinary":
        for at in range(0, H, 256):  # every other block
            block = x[:, at:at + 128]
            block *= 0.0 if beside == "zeros" else np.float32(2.0 ** -70)
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("beside", ["ordinary", "zeros", "tiny"])
@pytest.mark.parametrize("N,H", [(1, 128), (3, 700), (130, 512), (256, 1001)])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantized_bytes(beside, N, H, rows, scale, dtype):
    x = torch.from_numpy(signed(N, H, beside, N + H)).to(DT[dtype]).double().numpy()
    q, _ = ref.quantize(x, rows, scale == "e8m0")
    want = bytes_of(q, x)
    assert (want == 0x80).any() and (want == 0x00).any()
    got = opd.quantize_blocks(strided(x.astype(np.float32), DT[dtype]), block_rows=rows,
                              scale_dtype=SCALES[scale])["q"]
    assert torch.equal(got.contiguous().view(torch.uint8).cpu(), want)
