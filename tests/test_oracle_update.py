"""The fp64 oracles of token log-probabilities, pair losses and the optimiser's step, against differences and closed forms."""
import math

import numpy as np
import pytest

from oracle import adamw, preference


@pytest.mark.parametrize("temperature", [0.5, 1.0, 1.7])
@pytest.mark.parametrize("a,b", [(1.0, 0.0), (-0.7, 0.4), (0.0, -1.0)])
def test_gradient_of_logp_and_entropy_is_that_of_differences(temperature, a, b):
    rng = np.random.default_rng(1)
    z = rng.normal(size=9) * 2
    g = preference.logp_grad_row(z, 4, temperature, a, b)
    def f(x):
        logp, _, H = preference.logp_row(x, 4, temperature)
        return a * logp + b * H
    for i in range(9):
        d = np.zeros(9)
        d[i] = 1e-5
        assert abs((f(z + d) - f(z - d)) / 2e-5 - g[i]) < 1e-8
    assert abs(g.sum()) < 1e-12


def test_uniform_and_empty_rows():
    logp, lse, H = preference.logp_row(np.full(8, 3.0), 0, 2.0)
    assert math.isclose(logp, -math.log(8)) and math.isclose(lse, 1.5 + math.log(8)) and math.isclose(H, math.log(8))
    assert preference.logp_row(np.full(4, -np.inf), 0, 1.0)[1] == -math.inf
    assert math.isnan(preference.logp_row(np.array([0.0, np.inf]), 0, 1.0)[0])


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.2), ("hinge", 0.0), ("squared", 0.0)])
@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("nll", [0.0, 0.3])
def test_pair_gradient_is_that_of_differences(kind, smoothing, average, nll):
    rng = np.random.default_rng(2)
    cu = [0, 4, 4, 9, 15]
    logp, ref = -rng.random(15) * 3, -rng.random(15) * 3
    mask = rng.random(15) < 0.8
    pairs = [(0, 2), (0, 3), (3, 2), (-1, 2), (1, 0)]
    kw = dict(kind=kind, smoothing=smoothing, margin=0.1, average=average, nll=nll)
    def f(x):
        return preference.preference(x, ref, mask, cu, pairs, 0.4, **kw)[0]
    loss, g, reward, losses = preference.preference(logp, ref, mask, cu, pairs, 0.4, **kw)
    assert math.isclose(loss, losses[[0, 1, 2, 4]].mean()) and losses[3] == 0 and reward[1] == 0
    for t in range(15):
        d = np.zeros(15)
        d[t] = 1e-6
        assert abs((f(logp + d) - f(logp - d)) / 2e-6 - g[t]) < 1e-7, t
        if not mask[t]:
            assert g[t] == 0


def test_equal_scores_lose_log_2_with_half_a_slope():
    loss, g, _, _ = preference.preference(np.zeros(2), None, None, [0, 1, 2], [(0, 1)], 0.5)
    assert math.isclose(loss, math.log(2)) and np.allclose(g, [-0.25, 0.25])


def test_the_grid_is_e4m3():
    import torch
    codes = torch.arange(256, dtype=torch.uint8)
    got = codes.view(torch.float8_e4m3fn).double().numpy()
    want = adamw.decode(codes.numpy(), np.full(8, 127))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)]) and np.array_equal(np.isnan(got), np.isnan(want))
    v = adamw.e4m3_values()
    assert np.allclose(adamw.place_on_grid(v, np.full(4, 127)), np.arange(127))


def test_random_bits_look_random():
    """Means and correlations of 2^16 words within six standard deviations of those of independent uniform numbers."""
    n = 1 << 16
    words = [w.astype(np.float64) / 65536 - 0.5 for w in adamw.random_bits(7, 3, 1 << 20, n)]
    words += [w.astype(np.float64) / 65536 - 0.5 for w in adamw.random_bits(7, 4, 1 << 20, n)]
    words += [words[0][1:].tolist() + [0.0]]
    bound = 6 / math.sqrt(n)
    for i, a in enumerate(words):
        assert abs(np.mean(a)) < bound * math.sqrt(1 / 12)
        for b in words[:i]:
            assert abs(np.mean(np.asarray(a) * b)) < bound / 12


def test_first_step_moves_by_the_learning_rate():
    g = np.array([3.0, -0.01, 0.0])
    p, m, v = adamw.step(np.ones(3), g, np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.99, 1e-12, decay=0.5)
    assert np.allclose(p, 0.95 - 0.1 * np.sign(g)) and np.allclose(m, 0.1 * g) and np.allclose(v, 0.01 * g * g)
