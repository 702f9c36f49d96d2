"""An entropy bonus in accumulation steps: the rows of each step with their entropies and the gradient of both terms, as over the whole
batch at once."""
import numpy as np
import pytest
import torch

from oracle import preference
from paper_2504_13818_b200 import accumulation as ga, binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("masked", [False, True])
def test_log_probabilities_entropies_and_their_gradient_step_by_step(masked):
    g = torch.Generator(device="cuda").manual_seed(2)
    T, V, tau = 90, 1200, 0.75
    z = (torch.randn((T, V), generator=g, device="cuda") * 2.0).to(torch.bfloat16)
    tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dlogp, dent = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda") * 0.1
    mask = (torch.arange(T, device="cuda") % 4 != 1).to(torch.uint8) if masked else None
    if masked:
        dlogp, dent = dlogp * mask, dent * mask
        z[mask == 0] = torch.nan
    plan = ga.make_plan(G=1, n=6, m=6, steps=3)
    ranges = ga.step_ranges(torch.tensor([0, 10, 31, 31, 50, 52, T]), plan)
    logp, entropy = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    lse, out = torch.zeros(T, dtype=torch.float64, device="cuda"), torch.empty_like(z)
    status = binding.new_status()
    for a, (_, _, lo, hi) in enumerate(ranges):
        ga.logp_step(a, ranges, z[lo:hi], tokens, mask, logp, lse, temperature=tau, entropy=entropy, status=status)
    for a, (_, _, lo, hi) in enumerate(ranges):
        ga.logp_grad_step(a, ranges, z[lo:hi], tokens, lse, dlogp, out[lo:hi], temperature=tau, entropy=entropy, dentropy=dent, status=status)
    assert binding.read_status(status) == 0
    want = binding.pods_logp_chunk(z, tokens, temperature=tau, mask=mask, want_lse=True, want_entropy=True)
    assert torch.equal(logp, want[0]) and torch.equal(lse, want[1]) and torch.equal(entropy, want[2])
    assert torch.equal(out, binding.pods_logp_grad_chunk(z, tokens, lse, dlogp, entropy=entropy, dentropy=dent, temperature=tau))
    # a few rows against the formula: half a step of bf16 and the exponentials' 2^-17 of the terms' sizes
    zn = z.double().cpu().numpy()
    for t in (0, 2, 30, 51, T - 1):
        if masked and t % 4 == 1:
            assert logp[t] == 0 and entropy[t] == 0 and (out[t] == 0).all()
            continue
        lp, _, H = preference.logp_row(zn[t], int(tokens[t]), tau)
        assert abs(logp[t].item() - lp) <= 2.0 ** -18 * max(1.0, abs(lp)) and abs(entropy[t].item() - H) <= 2.0 ** -16 * max(1.0, H)
        w = preference.logp_grad_row(zn[t], int(tokens[t]), tau, dlogp[t].item(), dent[t].item())
        logq = preference.log_softmax(zn[t], tau)
        terms = np.exp(logq) * (abs(dlogp[t].item()) + abs(dent[t].item()) * (np.abs(logq) + H)) / tau
        terms[int(tokens[t])] += abs(dlogp[t].item()) / tau
        assert np.all(np.abs(out[t].double().cpu().numpy() - w) <= 2.0 ** -8 * np.abs(w) + 2.0 ** -17 * terms + 2.0 ** -120)
