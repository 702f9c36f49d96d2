"""pods_adamw and pods_grad_norm on sets of tensors that fill the tables of their launches exactly, by one more, and several times over: 24
entries of the small table, 352 of 8-bit states, 432 of 32-bit states, 1248 gradients.  No tensor is empty unless said, so that the
counts are those of the entries."""
import math

import numpy as np
import pytest
import torch

from test_gpu_adamw import SET, U, check_step, make, snapshot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def norm_of(before):
    return math.sqrt(sum((g * g).sum() for _, g, _ in before))


@pytest.mark.parametrize("bits,count", [(8, 24), (8, 25), (8, 352), (8, 353), (8, 705), (32, 24), (32, 25), (32, 432), (32, 433), (32, 900)])
def test_sets_at_the_tables_ends(binding, bits, count):
    rng = np.random.default_rng(count)
    table = make(binding, rng.integers(1, 300, count).tolist(), "bf16", "fp32", bits, copy="fp16", seed=count)
    before = snapshot(table)
    norm = binding.pods_grad_norm(table)
    assert abs(norm.item() - norm_of(before)) <= 4 * U * norm_of(before)
    binding.pods_adamw(table, 2, 1e-2, stochastic=True, seed=5, norm=norm, max_norm=0.5, **SET)
    check_step(table, before, 2, 1e-2, seed=5, stochastic=True, norm=norm.item(), max_norm=0.5)


@pytest.mark.parametrize("count", [24, 25, 1248, 1249, 2497])
def test_norms_at_the_tables_ends(binding, count):
    g = torch.Generator(device="cuda").manual_seed(count)
    sizes = np.random.default_rng(count).integers(1, 200, count).tolist()
    flat = torch.randn(sum(sizes), generator=g, device="cuda")
    flat[-sizes[-1]:] *= 100.0                         # the last one counts
    want = flat.double().norm().item()
    assert abs(binding.pods_grad_norm(list(flat.split(sizes))).item() - want) <= 4 * U * want


def test_states_of_both_kinds_by_turns_beyond_both_tables(binding):
    """Random bits go by an element's place among all tensors, so each launch has to count the ones of the other kind that it skips."""
    rng = np.random.default_rng(1)
    sizes = rng.integers(0, 400, (2, 460)).tolist()
    a, b = make(binding, sizes[0], "bf16", "fp32", 8, seed=1), make(binding, sizes[1], "bf16", "fp32", 32, seed=2)
    order = rng.permutation(920)
    mixed = [[(x + y)[i] for i in order] for x, y in zip((a.params, a.grads, a.states), (b.params, b.grads, b.states))]
    table = binding.pods_adamw_table(*mixed, weight_decay=0.1)
    before = snapshot(table)
    norm = binding.pods_grad_norm(table)
    assert abs(norm.item() - norm_of(before)) <= 4 * U * norm_of(before)
    binding.pods_adamw(table, 4, 1e-3, stochastic=True, seed=9, **SET)
    check_step(table, before, 4, 1e-3, seed=9, stochastic=True)
