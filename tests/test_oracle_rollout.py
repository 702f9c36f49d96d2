"""Pins of the sampling, list and distillation oracle: hand-worked rows, closed forms, brute force over kept sets, frequency
of draws over an even grid of random numbers, and finite differences."""
import numpy as np
import pytest

from oracle import rollout


def test_a_hand_worked_row():
    row = np.log(np.array([1.0, 4.0, 2.0, 1.0]))           # probabilities 1/8, 1/2, 1/4, 1/8
    draw = lambda u, **kw: rollout.sample_row(row, u, **kw)  # noqa: E731
    assert [draw(u)["token"] for u in (0.0, 0.12, 0.13, 0.62, 0.63, 0.87, 0.88, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert draw(0.7, top_k=2)["kept"].tolist() == [1, 2] and draw(0.7, top_k=2)["token"] == 2
    assert draw(0.0, top_k=3)["kept"].tolist() == [1, 2, 0]  # the tie goes to the lower id
    assert draw(0.0, top_p=0.5)["kept"].tolist() == [1]
    assert draw(0.0, top_p=0.51)["kept"].tolist() == [1, 2]
    assert draw(0.0, top_p=0.0)["kept"].tolist() == [1]
    assert draw(0.0, min_p=0.5)["kept"].tolist() == [1, 2]
    assert draw(0.0, min_p=1.0)["kept"].tolist() == [1]
    got = draw(0.7, top_k=2)
    assert got["logp"] == pytest.approx(np.log(0.25)) and got["logq"] == pytest.approx(np.log(1 / 3))
    # top_p is taken of the top-k sum: 4 of 6 is 0.667
    assert draw(0.0, top_k=2, top_p=0.66)["kept"].tolist() == [1]
    assert draw(0.0, top_k=2, top_p=0.67)["kept"].tolist() == [1, 2]
    assert draw(0.9, tau=0.0)["token"] == 1 and draw(0.9, tau=0.0)["logq"] == 0.0
    assert draw(0.5, tau=0.5)["logp"] == pytest.approx(np.log(16 / 22))


def test_an_even_grid_of_random_numbers_gives_the_distribution():
    rng = np.random.default_rng(0)
    row = rng.normal(0, 1.5, 12)
    n = 20000
    tokens = np.array([rollout.sample_row(row, (i + 0.5) / n, tau=0.8, top_k=7)["token"] for i in range(n)])
    kept = np.sort(np.argsort(-row)[:7])
    want = np.exp(row[kept] / 0.8) / np.exp(row[kept] / 0.8).sum()
    assert set(tokens) <= set(kept.tolist())
    assert np.abs(np.bincount(tokens, minlength=12)[kept] / n - want).max() <= 1.0 / n   # a grid misses by one point at most


def test_rows_without_a_distribution():
    assert rollout.sample_row(np.full(4, -np.inf), 0.3)["token"] == -1
    assert np.isnan(rollout.sample_row(np.array([0.0, np.nan]), 0.3)["logp"])
    row = np.array([-np.inf, 1.0, -np.inf])
    assert all(rollout.sample_row(row, u)["token"] == 1 for u in (0.0, 0.5, 0.99999))


def test_topk_order_and_normaliser():
    row = np.array([2.0, 3.0, -0.0, 3.0, 0.0])
    got = rollout.topk_row(row, 5, tau=2.0)
    assert got["ids"].tolist() == [1, 3, 0, 2, 4]
    assert got["lse"] == pytest.approx(np.log(np.exp(row / 2).sum()))


@pytest.mark.parametrize("rest,lse", [(False, False), (False, True), (True, True)])
def test_distillation_gradient_by_differences(rest, lse):
    rng = np.random.default_rng(3)
    V, K, tau = 11, 4, 1.7
    z, y = rng.normal(0, 1.5, V), rng.normal(0, 1.5, V)
    ids = rng.permutation(V)[:K]
    L = np.log(np.exp(y / tau).sum()) if lse else None
    f = lambda x: rollout.distill_row(x, ids, y[ids], L, tau, rest)  # noqa: E731
    got = f(z)
    assert got["kl"] > 0 or not rest
    h = 1e-5
    for v in range(V):
        up, dn = z.copy(), z.copy()
        up[v] += h
        dn[v] -= h
        # the oracle's gradient is with respect to z / tau; the difference's error is h^2 times a third derivative below 10
        assert abs((f(up)["kl"] - f(dn)["kl"]) / (2 * h) - got["grad"][v] / tau) <= 1e-8


def test_distillation_closed_forms():
    rng = np.random.default_rng(4)
    z = rng.normal(0, 2, 9)
    full = np.arange(9)
    lse = np.log(np.exp(z).sum())
    same = rollout.distill_row(z, full, z, lse)
    assert abs(same["kl"]) < 1e-12 and np.abs(same["grad"]).max() < 1e-12
    part = rollout.distill_row(z, full[:3], z[:3], lse, rest=True)       # the same policy seen through three ids and the rest
    assert abs(part["kl"]) < 1e-12 and np.abs(part["grad"]).max() < 1e-12
    # the gradient's sum is zero: a shift of the row changes nothing
    y = rng.normal(0, 2, 9)
    got = rollout.distill_row(z, full[:4], y[:4], np.log(np.exp(y).sum()), tau=0.6, rest=True)
    assert abs(got["grad"].sum()) < 1e-12
    # an id in two entries counts with the sum of their masses
    twice = rollout.distill_row(z, [2, 5, 2], [0.1, 0.2, 0.3])
    q = np.exp([0.1, 0.2, 0.3]) / np.exp([0.1, 0.2, 0.3]).sum()
    p = np.exp(z - lse)
    assert twice["grad"][2] == pytest.approx(p[2] - q[0] - q[2]) and twice["grad"][0] == pytest.approx(p[0])
    # nothing outside the list: the rest's term is left out
    none = rollout.distill_row(np.array([0.0, 1.0, -np.inf]), [0, 1], [0.0, 0.0], np.log(3.0), rest=True)
    assert none["r"] == 0.0 and np.isfinite(none["kl"])
