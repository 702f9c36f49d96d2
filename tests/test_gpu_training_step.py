"""Selection, pair losses, gradients and the weights' step together, as a training program uses them."""
import numpy as np
import pytest
import torch

from oracle import adamw, preference
from paper_2504_13818_b200 import accumulation as ga, binding, workloads as wl

pytestmark = pytest.mark.gpu


def f32(x):
    return float(np.float32(x))


def pairs_of(rewards, idx):
    """Of every group's kept rollouts the best against the worst, the second best against the second worst, ... where rewards differ."""
    G, m = idx.shape
    kept = rewards.gather(1, idx.long())
    order = kept.argsort(dim=1, descending=True, stable=True)
    best, worst = order[:, :m // 2], order.flip(1)[:, :m // 2]
    base = torch.arange(G, device=idx.device)[:, None] * m
    pairs = torch.stack((base + best, base + worst), 2).to(torch.int32)
    pairs[kept.gather(1, best) == kept.gather(1, worst)] = -1
    return pairs.reshape(-1, 2).contiguous()


@pytest.mark.parametrize("V", [520, 16384])
def test_from_rewards_to_a_gradient_and_in_accumulation_steps(V):
    w = wl.Workload("pairs", G=3, n=32, m=8, rewards="bernoulli_uniform", seed=5, V=V, len_kind="uniform", len_lo=4, len_hi=12, logit_sigma=2.0)
    plan = ga.make_plan(w.G, w.n, w.m, steps=4)
    lengths, src = wl.make_rollouts(w)
    L = src.shape[1]
    dev = torch.device("cuda:0")
    status = binding.new_status(dev)
    rewards = torch.from_numpy(ga.step_major(wl.make_rewards(w), plan)).to(dev)
    idx, _, _ = binding.pods_select(rewards, plan.m_step, status=status)
    len_sm = torch.from_numpy(ga.step_major(lengths.reshape(w.G, w.n), plan).reshape(-1)).to(dev)
    tok_sm = torch.from_numpy(ga.step_major(src.reshape(w.G, w.n, L), plan).reshape(-1, L)).to(dev)
    cu, toks, _ = binding.pods_compact(idx, plan.n_step, len_sm, tok_sm, status=status)
    T = int(cu[-1])
    tokens = toks[:T].contiguous()
    logits = torch.from_numpy(wl.make_logits_host(w, tokens.cpu().numpy())).view(torch.bfloat16).to(dev)
    pairs = pairs_of(rewards, idx)
    zn, tn, cun = logits.double().cpu().numpy(), tokens.cpu().numpy(), cu.cpu().numpy()
    exact = np.array([preference.logp_row(zn[t], tn[t], 1.0)[0] for t in range(T)])
    ref = (exact + 0.05 * np.random.default_rng(0).normal(size=T)).astype(np.float32)
    refd = torch.from_numpy(ref).to(dev)
    loss, logp, dlogits, reward, losses = binding.pods_preference_fwd_bwd(logits, tokens, refd, None, cu, pairs, 0.1, status=status)
    want = preference.preference(exact, ref, None, cun, pairs.tolist(), f32(0.1))
    assert np.abs(logp.cpu().numpy() - exact).max() <= 2.0 ** -18 + 2.0 ** -23 * np.abs(exact).max()
    assert abs(loss.item() - want[0]) <= 2.0 ** -18 * 12 + 2.0 ** -23 * abs(want[0])
    for t in range(T):
        g = preference.logp_grad_row(zn[t], tn[t], 1.0, want[1][t])
        # slopes move by a quarter of beta^2 times the scores' error, 2^-18 a token
        assert np.all(np.abs(dlogits[t].double().cpu().numpy() - g) <= (2.0 ** -8 + 2.0 ** -12) * np.abs(g) + 12 * 2.0 ** -18 * 0.01), t

    ranges = ga.step_ranges(cu.cpu(), plan)
    logp2, lse = torch.zeros(T, device=dev), torch.zeros(T, dtype=torch.float64, device=dev)
    for a, (_, _, lo, hi) in enumerate(ranges):
        ga.logp_step(a, ranges, logits[lo:hi], tokens, None, logp2, lse, status=status)
    acc = torch.zeros(1, dtype=torch.float64, device=dev)
    dlogp, reward2, losses2 = binding.pods_preference(logp2, refd, None, cu, pairs, 0.1, acc, status=status)
    out = torch.empty_like(logits)
    for a, (_, _, lo, hi) in enumerate(ranges):
        ga.logp_grad_step(a, ranges, logits[lo:hi], tokens, lse, dlogp, out[lo:hi], status=status)
    assert torch.allclose(logp2, logp, rtol=2.0 ** -22, atol=2.0 ** -18) and abs(acc.item() - loss.item()) <= 12 * 2.0 ** -18
    assert torch.allclose(out.float(), dlogits.float(), rtol=2.0 ** -7, atol=12 * 2.0 ** -18 * 0.01)
    assert binding.read_status(status) == 0
    with pytest.raises(ValueError, match="rows"):
        ga.logp_step(0, ranges, logits[:1], tokens, None, logp2, lse)
    with pytest.raises(ValueError, match="rows"):
        ga.logp_grad_step(0, ranges, logits[:1], tokens, lse, dlogp, out[:1])


@pytest.mark.parametrize("bits", [8, 32])
def test_the_objective_from_hidden_states_and_the_projections_step(bits):
    """Two accumulation steps add to dW, then the projection's weights move; a second round starts from them."""
    g = torch.Generator(device="cuda").manual_seed(3)
    T, V, d = 180, 1000, 96
    W = (torch.randn((V, d), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    W[13] = 0
    cu = torch.tensor([0, 70, 100, T], device="cuda")
    adv = torch.tensor([1.0, -0.5, 0.25], device="cuda")
    sw = binding.grpo_seq_weights(None, cu)
    dW = torch.zeros((V, d), device="cuda")
    states = binding.new_adamw_state(W, bits)
    table = binding.pods_adamw_table([W], [dW], [states], weight_decay=0.01)
    status, first = binding.new_status(), W.clone()
    m = v = np.zeros(V * d)
    for step in (1, 2):
        dW.zero_()
        acc = torch.zeros(1, dtype=torch.float64, device="cuda")
        hidden = (torch.randn((T, d), generator=g, device="cuda")).to(torch.bfloat16)
        tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        old, _ = binding.grpo_logp_from_hidden(hidden, W, tokens, status=status)
        for lo, hi in ((0, 100), (100, T)):
            binding.grpo_loss_from_hidden(hidden[lo:hi], W, tokens[lo:hi], old[lo:hi], None, adv, sw, cu, lo, None, 0.2, 0.0, acc, dW, status=status)
        p0, g0 = W.double().cpu().numpy().reshape(-1), dW.double().cpu().numpy().reshape(-1)
        norm = ga.update(table, step, 2e-3, max_norm=0.05, stochastic=True, seed=step, beta2=0.95, status=status)
        assert abs(norm.item() - np.linalg.norm(g0)) <= 2.0 ** -22 * np.linalg.norm(g0) and norm.item() > 0.05
        want, m1, v1 = adamw.step(p0, g0, m, v, step, f32(2e-3), f32(0.9), f32(0.95), f32(1e-8), decay=f32(0.01), norm=norm.item(), max_norm=f32(0.05))
        got = W.double().cpu().numpy().reshape(-1)
        # rounded with random bits: off by less than one step of bf16 (2^-7), and by what a step of few fp32 roundings is off
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -20 * 2e-3 * 10)
        if bits == 32:
            # two products, a sum and the scaled gradient: 4 * 2^-24 of the terms added, which may cancel
            terms = 0.9 * np.abs(m) + 0.1 * np.abs(g0) * (0.05 / norm.item())
            m, v = (s.double().cpu().numpy() for s in states)
            assert np.all(np.abs(m - m1) <= 4.1 * 2.0 ** -24 * terms + 1e-44) and np.all(np.abs(v - v1) <= 6 * 2.0 ** -24 * v1 + 1e-44)
        else:
            k = [s.cpu().numpy() for s in states]
            m, v = adamw.decode(k[0], k[1]), adamw.decode(k[2], k[3]) ** 2
    assert binding.read_status(status) == 0 and not torch.equal(first, W)
