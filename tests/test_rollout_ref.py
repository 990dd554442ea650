"""Pins of the 64-bit forms the rollout operators are tested against (CPU)."""
import numpy as np
import pytest
import torch

import rollout_ref as ref


def test_nearest_e4m3_is_the_8_bit_types_own_rounding():
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.02, 4000),
                        np.arange(-16, 17) * 2.0 ** -10, [0.0, 448.0, -448.0, 2.0 ** -6]])
    v = v.astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.nearest_e4m3(v), want)
    # ties go to the even neighbour, between normal values and below them
    assert ref.nearest_e4m3([1.0625, 1.1875, 3 * 2.0 ** -10, 5 * 2.0 ** -10]).tolist() == \
        [1.0, 1.25, 2.0 ** -8, 2.0 ** -8]


def test_power_of_two_scales_are_the_least_that_reach():
    a = np.float32([[448.0] * 128, [448.1] * 128, [1.0] * 128, [0.0] * 128, [1e-38] * 128])
    _, s = ref.quantize(a, 1, True)
    assert s[:, 0].tolist()[:4] == [1.0, 2.0, 2.0 ** -8, 2.0 ** -127]
    assert s[4, 0] * 448 >= 1e-38 > s[4, 0] * 224 or s[4, 0] == 2.0 ** -127


@pytest.mark.parametrize("certain", [False, True])
def test_verified_tokens_follow_the_target(certain):
    """Summed over the drafter's draws and a fine grid of uniforms, the first
    token's distribution is the target's, for any drafter."""
    rng = np.random.default_rng(2)
    V, G = 4, 60
    target, draft = rng.normal(0, 1, (1, 2, V)), rng.normal(0, 1, (1, 1, V))
    p = np.exp(ref.log_softmax(target[0, 0]).astype(float))
    q = np.exp(ref.log_softmax(draft[0, 0]).astype(float))
    grid = (np.arange(G) + 0.5) / G
    got = np.zeros(V)
    for x in range(V):
        weight = (1.0 / V if certain else q[x]) / G ** 2
        for a in grid:
            for r in grid:
                _, out, _, _ = ref.verify(target, np.array([[x]]), np.array([[a, r]]),
                                          None if certain else draft)
                got[out[0, 0]] += weight
    # each of the V tests and draws is off by at most a grid step
    assert np.abs(got - p).max() < 2.0 * V / G / 4


def test_borders_of_the_reference():
    z = np.log(np.array([[[0.5, 0.25, 0.25], [0.2, 0.3, 0.5]]]))
    # kept while u < p: then the next row's draw, in index order
    assert ref.verify(z, np.array([[0]]), np.array([[0.4, 0.21]]))[1].tolist() == [[0, 1]]
    # refused: the draw is from p without the token
    assert ref.verify(z, np.array([[0]]), np.array([[0.6, 0.49]]))[1].tolist() == [[1, -1]]
    assert ref.verify(z, np.array([[0]]), np.array([[0.6, 0.51]]))[1].tolist() == [[2, -1]]
    a, out, lp, _ = ref.verify(z, np.array([[7]]), np.array([[0.6, 0.51]]))
    assert a[0] == 0 and out.tolist() == [[-1, -1]] and np.isnan(lp[0, 0])
