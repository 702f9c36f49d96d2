"""pods_logp_chunk and pods_logp_grad_chunk against the fp64 oracle.

Tolerances.  An exponential is off by 2^-22 relative (two units of ex2.approx) plus ln 2 times the rounding of its exponent:
2^-24 of the exponent z c - R (at most 10 above 0 in the kernel's scale, and below 0 its weight falls faster than its error
grows: |d| 2^d <= 0.54), and 2^-24 of |z - z_max| / temperature from rounding c.  fp32 partial sums of n terms add at most n 2^-24;
a thread adds at most 2048 / 8 blocks' sums in the longest row tested, mostly far fewer and of random sign.  REL = 2^-19 covers them
(2^-22 + 10 * 2^-24 + 2^-21 and the partial sums); log-probabilities add their own rounding."""
import numpy as np
import pytest
import torch

from oracle import preference

pytestmark = pytest.mark.gpu
REL = 2.0 ** -19
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def rows(T, V, dtype, seed=0, pad=0, scale=3.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.zeros((T, V + pad), dtype=TYPES[dtype])
    wide[:, :V] = torch.randn((T, V), generator=g) * scale + shift
    wide = wide.cuda()
    return wide[:, :V], torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()


def check_forward(z, tok, tau, got, skip=()):
    logp, lse, H = (x.cpu().numpy() if x is not None else None for x in got)
    zn, tok = z.double().cpu().numpy(), tok.cpu().numpy()
    for t in range(z.shape[0]):
        if t in skip:
            continue
        lp, ls, h = preference.logp_row(zn[t], tok[t], tau)
        spread = np.abs(zn[t][np.isfinite(zn[t])] - zn[t].max()).max() / tau if np.isfinite(zn[t].max()) else 0.0
        tol = REL + 2.0 ** -23 * min(spread, 100.0)
        if np.isnan(lp):
            assert np.isnan(logp[t])
        elif lp == -np.inf:
            assert logp[t] == -np.inf
        else:
            assert abs(logp[t] - lp) <= tol + 2.0 ** -23 * abs(lp), (t, logp[t], lp)
        if lse is not None:
            assert (np.isnan(ls) and np.isnan(lse[t])) or lse[t] == ls or abs(lse[t] - ls) <= tol + 2.0 ** -24 * abs(ls), (t, lse[t], ls)
        if H is not None:
            assert (np.isnan(h) and np.isnan(H[t])) or abs(H[t] - h) <= 4 * tol * max(1.0, h) + 2.0 ** -23 * h, (t, H[t], h)


def check_gradient(z, tok, tau, dlogp, dent, out, dtype):
    zn, tok, out = z.double().cpu().numpy(), tok.cpu().numpy(), out.double().cpu().numpy()
    a = dlogp.double().cpu().numpy()
    b = dent.double().cpu().numpy() if dent is not None else np.zeros_like(a)
    # exponentials below 2^-126, the smallest normal number, are 0 in the kernel; with coefficients of at most 2^6 here that takes
    # at most 2^-120 off a value.  fp16: half of its smallest step
    tiny = 2.0 ** -25 if dtype == "fp16" else 2.0 ** -120
    for t in range(z.shape[0]):
        want = preference.logp_grad_row(zn[t], tok[t], tau, a[t], b[t])
        H = preference.logp_row(zn[t], tok[t], tau)[2]
        logq = preference.log_softmax(zn[t], tau)
        p = np.exp(logq)
        logs = np.where(p > 0, np.abs(logq), 0.0)
        part = p * (abs(a[t]) + abs(b[t]) * (logs + H)) / tau
        tol = HALF_STEP[dtype] * np.abs(want) + part * (REL + 2.0 ** -23 * np.minimum(logs, 100.0) + 2.0 ** -22) + tiny
        tol[tok[t]] += 2.0 ** -23 * abs(a[t]) / tau
        bad = np.abs(out[t] - want) > tol * 1.001
        assert not bad.any(), (t, np.nonzero(bad)[0][:4], out[t][bad][:4], want[bad][:4])


SHAPES = [(1, 1, 0), (3, 7, 0), (5, 31, 1), (9, 256, 0), (37, 1000, 0), (4, 4096, 3), (11, 4103, 0), (3, 8200, 8), (2, 20011, 0),
          (600, 17000, 0), (2, 151936, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,V,pad", SHAPES)
def test_forward_and_gradient(binding, dtype, T, V, pad):
    tau = 1.0 if V % 2 else 0.7
    z, tok = rows(T, V, dtype, seed=V, pad=pad)
    status = binding.new_status()
    got = binding.pods_logp_chunk(z, tok, temperature=tau, want_lse=True, want_entropy=True, status=status)
    tau = float(np.float32(tau))
    some = slice(0, min(T, 37))
    check_forward(z[some], tok[some], tau, [x[some] for x in got])
    plain = binding.pods_logp_chunk(z, tok, temperature=tau)
    assert plain[1] is None and plain[2] is None and torch.allclose(plain[0], got[0], rtol=0, atol=4e-6)
    g = torch.Generator().manual_seed(3)
    dlogp, dent = torch.randn(T, generator=g).cuda(), torch.randn(T, generator=g).cuda()
    for d in (None, dent):
        out = binding.pods_logp_grad_chunk(z, tok, got[1], dlogp, entropy=got[2] if d is not None else None, dentropy=d, temperature=tau, status=status)
        assert out.shape == z.shape and out.is_contiguous()
        check_gradient(z[some], tok[some], tau, dlogp[some], None if d is None else d[some], out[some], dtype)
    assert binding.read_status(status) == 0


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [1003, 33000])
def test_in_place_and_other_alignments(binding, dtype, V):
    z, tok = rows(6, V, dtype, seed=5, pad=5)
    lse = binding.pods_logp_chunk(z, tok, want_lse=True)[1]
    dlogp = torch.randn(6, generator=torch.Generator().manual_seed(1)).cuda()
    want = binding.pods_logp_grad_chunk(z, tok, lse, dlogp)
    for off in (0, 1, 3, 4):
        wide = torch.full((6, V + 16), 7.0, dtype=z.dtype, device="cuda")
        out = wide[:, off:off + V]
        binding.pods_logp_grad_chunk(z, tok, lse, dlogp, dlogits=out)
        assert torch.equal(out, want)
        assert (wide[:, :off] == 7).all() and (wide[:, off + V:] == 7).all()
    beyond = z.as_strided((6, 5), (V + 5, 1), V).clone()
    assert binding.pods_logp_grad_chunk(z, tok, lse, dlogp, dlogits=z) is z
    assert torch.equal(z, want) and torch.equal(z.as_strided((6, 5), (V + 5, 1), V), beyond)


@pytest.mark.parametrize("V", [65, 5000, 40000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_that_defeat_a_first_guess(binding, dtype, V):
    """Rising and falling rows, huge offsets, -inf entries, one heavy id at either end, equal logits."""
    big = 60000.0 if dtype == "fp16" else 3.0e5
    base = torch.linspace(-1, 1, V)
    made = [base * 40, -base * 40, base * 0 + big, base * 0 - big, base + big, torch.where(torch.arange(V) == V - 1, 300.0, -300.0),
            torch.where(torch.arange(V) == 0, 300.0, -300.0), torch.where(torch.arange(V) % 3 == 1, -torch.inf, base * 5),
            torch.where(torch.arange(V) < V - 1, -torch.inf, 2.0), torch.where(torch.arange(V) % 2 == 0, torch.finfo(TYPES[dtype]).min, base),
            base * big, torch.full((V,), torch.finfo(TYPES[dtype]).min)]
    z = torch.stack(made).to(TYPES[dtype]).cuda()
    T = z.shape[0]
    for place in (0, V // 3, V - 1):
        tok = torch.full((T,), place, dtype=torch.int32, device="cuda")
        status = binding.new_status()
        got = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True, status=status)
        assert binding.read_status(status) == 0
        check_forward(z, tok, 1.0, got)
        dlogp = torch.full((T,), 0.5, device="cuda")
        out = binding.pods_logp_grad_chunk(z, tok, got[1], dlogp, entropy=got[2], dentropy=dlogp * 0.1)
        check_gradient(z, tok, 1.0, dlogp, dlogp * 0.1, out, dtype)


@pytest.mark.parametrize("V", [50, 30000])
def test_fp32_logits_and_temperatures_out_of_all_proportion(binding, V):
    z = torch.randn((4, V), generator=torch.Generator().manual_seed(2)) * torch.tensor([[1e9], [1e20], [3e38 / 6], [1.0]])
    z[1] = -z[1].abs()
    z = z.cuda()
    tok = z.argmax(1).to(torch.int32)
    logp, lse, H = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True)
    check_forward(z, tok, 1.0, (logp, lse, H))
    tok2 = z.argmin(1).to(torch.int32)
    logp2, _, _ = binding.pods_logp_chunk(z[3:], tok2[3:], temperature=1e-30)
    assert logp2.item() < -1e29
    hot, _, H = binding.pods_logp_chunk(z[3:], tok2[3:], temperature=1e30, want_entropy=True)
    assert abs(hot.item() + np.log(V)) < 2e-6 and abs(H.item() - np.log(V)) < 2e-5
    out = binding.pods_logp_grad_chunk(z, tok, lse, torch.ones(4, device="cuda"))
    check_gradient(z, tok, 1.0, torch.ones(4), None, out, "fp32")


@pytest.mark.parametrize("V", [40, 9000])
def test_rows_without_a_distribution(binding, V):
    z, tok = rows(7, V, "bf16", seed=9)
    z[1] = -torch.inf
    z[2, V // 2] = torch.nan
    z[3, V - 1] = torch.inf
    z[4, tok[4].long()] = -torch.inf
    tok[5] = V
    tok[6] = -1
    status = binding.new_status()
    logp, lse, H = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True, status=status)
    assert binding.read_status(status) == binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT | binding.STATUS_TOKEN_RANGE
    tok0 = tok.clone()
    tok0[5:] = 0
    check_forward(z, tok0, 1.0, (logp, lse, H))
    assert logp[4] == -torch.inf and torch.isfinite(lse[4]) and torch.isfinite(H[4])
    out = binding.pods_logp_grad_chunk(z, tok, lse, torch.ones(7, device="cuda"))
    assert torch.isnan(out[1]).all() and torch.isnan(out[2]).all() and torch.isnan(out[3]).all() and torch.isfinite(out[4:]).all()
    check_gradient(z[4:], tok0[4:], 1.0, torch.ones(3), None, out[4:], "bf16")
    # of no consequence where nothing is asked of the row
    zero = torch.ones(7, device="cuda")
    zero[1:4] = 0
    out = binding.pods_logp_grad_chunk(z, tok, lse, zero, entropy=H, dentropy=zero * 0.5)
    assert (out[1:4] == 0).all() and torch.isfinite(out).all()


def test_masked_rows_are_left_alone(binding):
    z, tok = rows(20, 9000, "fp16", seed=4)
    mask = (torch.arange(20) % 3 != 0).to(torch.uint8).cuda()
    z[mask == 0] = torch.nan
    out = [torch.full((20,), 5.0, device="cuda"), torch.full((20,), 5.0, dtype=torch.float64, device="cuda"), torch.full((20,), 5.0, device="cuda")]
    status = binding.new_status()
    got = binding.pods_logp_chunk(z, tok, mask=mask, logp=out[0], lse=out[1], entropy=out[2], status=status)
    assert binding.read_status(status) == 0
    for a, b in zip(got, out):
        assert a is b and (a[mask == 0] == 5).all() and torch.isfinite(a).all()
    check_forward(z, tok, 1.0, got, skip=set(range(0, 20, 3)))
    made = binding.pods_logp_chunk(z, tok, mask=mask, want_lse=True)
    assert (made[0][mask == 0] == 0).all() and torch.equal(made[0][mask == 1], got[0][mask == 1])


def test_no_rows_and_views(binding):
    z, tok = rows(0, 100, "bf16")
    logp, lse, H = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True)
    assert logp.numel() == lse.numel() == H.numel() == 0
    assert binding.pods_logp_grad_chunk(z, tok, lse, logp).shape == (0, 100)
    z, tok = rows(8, 3000, "bf16", seed=8)
    part = binding.pods_logp_chunk(z[::2], tok[::2].contiguous(), want_lse=True)
    assert torch.equal(part[0], binding.pods_logp_chunk(z, tok)[0][::2])
    with pytest.raises(binding.PodsError, match="contiguous"):
        binding.pods_logp_chunk(z[:, ::2], tok)
    with pytest.raises(binding.PodsError, match="contiguous"):
        binding.pods_logp_chunk(z, torch.stack((tok, tok), 1)[:, 0])
    with pytest.raises(binding.PodsError, match="overlap"):
        binding.pods_logp_chunk(z[:1].expand(8, 3000), tok)


def test_rows_more_than_2_to_the_32_elements_apart(binding):
    V, pitch = 1000, (1 << 31) + 8
    wide = torch.zeros(2 * pitch + V, dtype=torch.bfloat16, device="cuda")
    z = wide.as_strided((3, V), (pitch, 1))
    z.copy_(torch.randn((3, V), generator=torch.Generator().manual_seed(1)))
    tok = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    logp, lse, _ = binding.pods_logp_chunk(z, tok, want_lse=True)
    near = z.contiguous()
    assert torch.equal(logp, binding.pods_logp_chunk(near, tok)[0])
    ones = torch.ones(3, device="cuda")
    want = binding.pods_logp_grad_chunk(near, tok, lse, ones)
    assert torch.equal(binding.pods_logp_grad_chunk(z, tok, lse, ones), want)
    assert torch.equal(binding.pods_logp_grad_chunk(z, tok, lse, ones, dlogits=z), want)


def test_the_same_bits_every_time_on_two_streams_and_in_a_graph(binding):
    z, tok = rows(40, 30000, "bf16", seed=3)
    first = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True)
    d = torch.randn(40, generator=torch.Generator().manual_seed(1)).cuda()
    grad = binding.pods_logp_grad_chunk(z, tok, first[1], d, entropy=first[2], dentropy=d)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for k in range(6):
        with torch.cuda.stream(streams[k % 2]):
            f = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True)
            got.append((f, binding.pods_logp_grad_chunk(z, tok, f[1], d, entropy=f[2], dentropy=d)))
    torch.cuda.synchronize()
    for f, g in got:
        assert all(torch.equal(a, b) for a, b in zip(f, first)) and torch.equal(g, grad)
    out = torch.empty_like(grad)
    bufs = [torch.empty_like(x) for x in first]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.pods_logp_chunk(z, tok, logp=bufs[0], lse=bufs[1], entropy=bufs[2])
        binding.pods_logp_grad_chunk(z, tok, bufs[1], d, entropy=bufs[2], dentropy=d, dlogits=out)
    z.copy_(rows(40, 30000, "bf16", seed=33)[0])
    graph.replay()
    f = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True)
    assert all(torch.equal(a, b) for a, b in zip(f, bufs))
    assert torch.equal(out, binding.pods_logp_grad_chunk(z, tok, f[1], d, entropy=f[2], dentropy=d))
