"""pods_sample and pods_topk against the fp64 oracle.

Tokens and ids are equal, not near: a case whose draw lies within EDGE of a boundary between tokens would be decided by
rounding (an fp64 sum over V <= 2^19 terms is off by at most 2^19 * 2^-53 < 6e-11 of itself), so such draws are not asked for.

log-probabilities: fp64 up to the row's sum of exponentials, which the kernel takes from fp32 exponentials within 1.6e-6 of
itself: exponent argument (2^-24 + 2^-25) of its size, whose mean under the row's distribution is at most log2 V <= 19
(entropy bound), hardware exponential 2^-22.5, three roundings of 2^-24 in the sums of eight.  Then one rounding to fp32."""
import numpy as np
import pytest
import torch

from oracle import rollout
from paper_2504_13818_b200 import binding

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EDGE = 1e-10
SUM_RTOL = 1.6e-6


def log_tol(x):
    return SUM_RTOL + 2.0 ** -24 * np.abs(np.where(np.isfinite(x), x, 0.0))


def make(T, V, dtype, seed, kind="normal", pad=0, offset=0):
    """Rows of pitch V + pad that start `offset` elements into their storage."""
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn((T, V), generator=gen) * 3.0
    if kind == "peaked":
        n = min(V, 20)
        at = torch.randperm(V, generator=gen)[:n]
        z[:, at] += 12.0 - 0.5 * torch.arange(n)
    elif kind == "ties":
        z = torch.round(z / 2.0) * 0.5
    elif kind == "constant":
        z = torch.full((T, V), 1.25)
    elif kind == "holes":
        z[torch.rand((T, V), generator=gen) < 0.7] = -np.inf
        z[:, V // 2] = 0.5
    flat = torch.full((offset + T * (V + pad) + 16,), 7.0e4 if dtype != "fp16" else 6.0e4, dtype=DT[dtype])
    rows = flat.cuda()[offset:offset + T * (V + pad)].view(T, V + pad)[:, :V]
    rows.copy_(z.to(DT[dtype]))
    return rows


def check_sample(z, u, tau=1.0, top_k=0, top_p=1.0, min_p=0.0, expect_status=0):
    T = z.shape[0]
    status = binding.new_status()
    tokens, logp, logq = binding.pods_sample(z, u, temperature=tau, top_k=top_k, top_p=top_p, min_p=min_p, want_logq=True, status=status)
    torch.cuda.synchronize()
    assert binding.read_status(status) == expect_status
    rows = z.double().cpu().numpy()

    def per_row(x, as_type):
        return [as_type(v) for v in (x.cpu().numpy() if isinstance(x, torch.Tensor) else np.full(T, np.float32(x)))]

    taus, ks, ps, ms = per_row(tau, float), per_row(top_k, int), per_row(top_p, float), per_row(min_p, float)
    tok, lp, lq, un = tokens.cpu().numpy(), logp.cpu().numpy().astype(np.float64), logq.cpu().numpy().astype(np.float64), u.cpu().numpy()
    for t in range(T):
        want = rollout.sample_row(rows[t], float(un[t]), taus[t], ks[t], ps[t], ms[t])
        if want["edge"] <= EDGE:
            continue
        assert tok[t] == want["token"], (t, tok[t], want["token"], want["edge"], len(want["kept"]))
        assert abs(lp[t] - want["logp"]) <= log_tol(want["logp"]) or (lp[t] == want["logp"]) or (np.isnan(lp[t]) and np.isnan(want["logp"]))
        assert abs(lq[t] - want["logq"]) <= log_tol(want["logq"]) or (lq[t] == want["logq"]) or (np.isnan(lq[t]) and np.isnan(want["logq"]))
    return tokens, logp, logq


FILTERS = [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=50, top_p=0.9), dict(top_k=700), dict(top_p=0.1), dict(top_p=0.9),
           dict(top_p=0.999), dict(top_p=0.0), dict(min_p=0.01), dict(min_p=1.0), dict(min_p=1e-6),
           dict(top_p=0.95, min_p=0.001), dict(top_k=300, top_p=0.99, min_p=1e-4), dict(top_k=40, min_p=0.02)]


def uniform(T, seed):
    return torch.rand(T, generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,pad,offset", [(1, 0, 0), (2, 3, 1), (7, 0, 3), (9, 0, 0), (255, 1, 5), (1000, 8, 0), (5003, 0, 7), (32000, 0, 0)])
def test_lengths_alignments_and_filters(dtype, V, pad, offset):
    for i, kind in enumerate(["normal", "peaked", "ties"]):
        z = make(6, V, dtype, seed=V + i, kind=kind, pad=pad, offset=offset)
        for j, f in enumerate(FILTERS):
            check_sample(z, uniform(6, 100 * i + j), tau=[1.0, 0.7, 1.9][j % 3], **f)


@pytest.mark.parametrize("dtype,V", [("bf16", 151936), ("fp32", 151936), ("fp16", 50257), ("bf16", 300001), ("fp32", 524288)])
@pytest.mark.parametrize("kind", ["normal", "peaked", "ties"])
def test_long_rows(dtype, V, kind):
    z = make(3, V, dtype, seed=V, kind=kind)
    for j, f in enumerate(FILTERS):
        check_sample(z, uniform(3, j), tau=[1.0, 0.6][j % 2], **f)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [37, 5003, 151936])
def test_equal_logits_and_masked_ids(dtype, V):
    for kind in ("constant", "holes"):
        z = make(3, V, dtype, seed=V, kind=kind)
        for j, f in enumerate(FILTERS):
            check_sample(z, uniform(3, j), **f)


def test_first_and_last_random_number():
    z = make(4, 5003, "bf16", seed=1)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 2.0 ** -24, 0.5]).cuda()
    for f in FILTERS:
        check_sample(z, u, **f)


@pytest.mark.parametrize("V", [1000, 20000, 143193])
def test_zero_takes_the_lowest_kept_id_however_little_its_weight(V):
    """Rows that rise with the id at a cold temperature: the first ids weigh e^-700 and less."""
    z = (torch.randn((3, V), generator=torch.Generator().manual_seed(1)) * 10).sort(1).values.to(torch.bfloat16).cuda()
    z[1, : V // 3] = -np.inf
    u = torch.zeros(3).cuda()
    for f in (dict(), dict(top_k=400), dict(top_k=700), dict(top_p=0.99999), dict(min_p=1e-30), dict(top_p=0.5)):
        check_sample(z, u, tau=0.01, **f)
    many = z[:1].expand(34 * 10 ** 6 // V, V).contiguous()      # rows enough for the pipeline
    got = binding.pods_sample(many, torch.zeros(many.shape[0]).cuda(), temperature=0.01)
    assert (got[0] == 0).all() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("V", [4000, 60000])
@pytest.mark.parametrize("tau", [1.0, 0.01])
def test_logits_where_exponents_of_two_run_out_of_fractions(V, tau):
    """Maxima of a row's parts lie on both sides of the exponent 2^23, where references change their form."""
    at = -2.0 ** 23 * np.log(2.0) * tau
    for seed in range(4):
        z = torch.randn((8, V), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * (2 * tau)
        z = (z - z.max(1, keepdim=True).values + at + 0.5 * tau * torch.arange(8)[:, None]).to(torch.float32).cuda()
        u = torch.rand(8, generator=torch.Generator().manual_seed(100 + seed)).cuda()
        check_sample(z, u, tau=tau)
        check_sample(z, u, tau=tau, top_k=100)
        check_sample(z, u, tau=tau, top_p=0.8)


@pytest.mark.parametrize("V,dtype", [(1000, "fp32"), (151936, "bf16")])
def test_each_row_has_its_own_settings(V, dtype):
    T = 24
    z = make(T, V, dtype, seed=5, kind="peaked")
    g = torch.Generator().manual_seed(1)
    tau = (torch.rand(T, generator=g) * 1.5)
    tau[::5] = 0.0
    tau[1] = 2.0 ** -21
    k = torch.randint(-2, 80, (T,), generator=g, dtype=torch.int32)
    k[7] = V + 5
    p = 0.5 + 0.6 * torch.rand(T, generator=g)
    m = 0.1 * torch.rand(T, generator=g) - 0.05
    m[3] = 2.0
    check_sample(z, uniform(T, 3), tau=tau.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=m.cuda())


def test_cold_and_hot_temperatures():
    z = make(4, 5003, "fp32", seed=2)
    for tau in (0.0, 2.0 ** -20, 1e-3, 50.0, 1e30):
        for f in (dict(), dict(top_k=5), dict(top_p=0.5), dict(min_p=0.5)):
            check_sample(z, uniform(4, 9), tau=tau, **f)


def test_rows_without_a_distribution_and_settings_out_of_range():
    z = make(6, 1000, "fp32", seed=3)
    z[0] = -np.inf
    z[2, 999] = np.nan
    z[4, 0] = np.inf
    bits = binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT
    for f in FILTERS:
        check_sample(z, uniform(6, 1), expect_status=bits, **f)
    z = make(4, 1000, "bf16", seed=4)
    nan = float("nan")
    status = binding.new_status()
    base = uniform(4, 2)
    got = binding.pods_sample(z, base, temperature=torch.tensor([-1.0, nan, np.inf, 1.0]).cuda(), status=status)
    assert binding.read_status(status) == binding.STATUS_PARAM_RANGE
    want = binding.pods_sample(z, base)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for u, as_if in (([nan, -0.5, 1.0, 7.0], [0.0, 0.0, 1 - 2.0 ** -24, 1 - 2.0 ** -24]),):
        status = binding.new_status()
        got = binding.pods_sample(z, torch.tensor(u).cuda(), status=status)
        assert binding.read_status(status) == binding.STATUS_PARAM_RANGE
        assert torch.equal(got[0], binding.pods_sample(z, torch.tensor(as_if).cuda())[0])
    for name in ("top_p", "min_p"):
        status = binding.new_status()
        got = binding.pods_sample(z, base, status=status, **{name: torch.full((4,), nan).cuda()})
        assert binding.read_status(status) == binding.STATUS_PARAM_RANGE and torch.equal(got[0], want[0])


def test_masked_rows_are_left_as_they_were():
    T, V = 9, 5003
    z = make(T, V, "bf16", seed=6)
    mask = torch.tensor([1, 0, 1, 1, 0, 0, 1, 0, 1], dtype=torch.uint8).cuda()
    z[mask == 0] = float("nan")                            # not read: no status bit
    status = binding.new_status()
    tokens = torch.full((T,), 12345, dtype=torch.int32).cuda()
    logp = torch.full((T,), 3.5).cuda()
    u = uniform(T, 4)
    binding.pods_sample(z, u, mask=mask, tokens=tokens, logp=logp, top_p=0.9, status=status)
    ids, values, lse = binding.pods_topk(z, 5, mask=mask, status=status)
    assert binding.read_status(status) == 0
    live = mask.bool()
    assert (tokens[~live] == 12345).all() and (logp[~live] == 3.5).all()
    assert (ids[~live] == -1).all() and (values[~live] == 0).all() and (lse[~live] == 0).all()
    alone = binding.pods_sample(z[live].contiguous(), u[live].contiguous(), top_p=0.9)
    # V is odd: packed without the masked rows, a row starts at another 16-byte offset and its sum is grouped differently,
    # so the two log-probs agree as two values that are each within log_tol of the exact one
    assert torch.equal(tokens[live], alone[0])
    both = logp[live].double().cpu().numpy(), alone[1].double().cpu().numpy()
    assert (np.abs(both[0] - both[1]) <= 2 * log_tol(both[0])).all()


def test_frequencies_follow_the_distribution():
    """2^18 draws from one row: counts within six standard deviations of the probabilities."""
    V, n = 64, 1 << 18
    row = make(1, V, "fp32", seed=8)
    z = row.expand(n, V).contiguous()
    tokens, _, _ = binding.pods_sample(z, uniform(n, 5), top_k=20, temperature=1.3)
    p = torch.softmax(row[0].double() / np.float32(1.3), 0)
    keep = torch.zeros(V, dtype=torch.bool).cuda()
    keep[row[0].topk(20).indices] = True
    p = torch.where(keep, p, 0.0)
    p = (p / p.sum()).cpu().numpy()
    count = np.bincount(tokens.cpu().numpy(), minlength=V)
    assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p)) + 1e-9).all()


def test_many_rows_and_the_same_bits_twice():
    z = make(1500, 1003, "bf16", seed=9, kind="peaked", pad=2)
    u = uniform(1500, 6)
    for f in (dict(), dict(top_p=0.9), dict(top_k=700, top_p=0.99)):
        a = check_sample(z, u, **f)
        b = binding.pods_sample(z, u, want_logq=True, **f)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_another_stream_and_a_captured_graph():
    z = make(8, 50257, "bf16", seed=10, kind="peaked")
    u = uniform(8, 7)
    want = binding.pods_sample(z, u, top_p=0.9)[:2] + binding.pods_topk(z, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.pods_sample(z, u, top_p=0.9)[:2] + binding.pods_topk(z, 12)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    tokens, logp = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    ids, values, lse = (torch.zeros_like(x) for x in want[2:])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.pods_sample(z, u, top_p=0.9, tokens=tokens, logp=logp)
        binding.pods_topk(z, 12, ids=ids, values=values, lse=lse)
    for seed in (11, 12):
        z.copy_(make(8, 50257, "bf16", seed=seed, kind="peaked"))
        u.copy_(uniform(8, seed))
        graph.replay()
        want = binding.pods_sample(z, u, top_p=0.9)[:2] + binding.pods_topk(z, 12)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((tokens, logp, ids, values, lse), want))


def far_apart(rows, pitch):
    """The rows in a storage of 9 GB: offsets past 2^32 elements."""
    T, V = rows.shape
    flat = torch.empty(T * pitch, dtype=rows.dtype, device="cuda")
    out = flat.view(T, pitch)[:, :V]
    out.copy_(rows)
    return out


def test_rows_far_apart():
    z = far_apart(make(224, 151936, "bf16", seed=2), 20_000_003)         # rows enough for the pipeline
    u = uniform(224, 4)
    check_sample(z, u)
    check_sample(z[200:], u[200:], top_k=40, top_p=0.9)
    check_sample(z[200:], u[200:], top_p=0.95)
    check_topk(z[200:], 100)


# ---- pods_topk ------------------------------------------------------------------------------------------------------

def check_topk(z, K, tau=1.0, expect_status=0):
    status = binding.new_status()
    ids, values, lse = binding.pods_topk(z, K, temperature=tau, status=status)
    torch.cuda.synchronize()
    assert binding.read_status(status) == expect_status
    rows = z.double().cpu().numpy()
    ids, values, lse = ids.cpu().numpy(), values.cpu().numpy(), lse.cpu().numpy().astype(np.float64)
    for t in range(z.shape[0]):
        want = rollout.topk_row(rows[t], K, float(np.float32(tau)))
        assert np.array_equal(ids[t], want["ids"]), t
        assert np.array_equal(values[t].astype(np.float64), want["values"], equal_nan=True)
        assert abs(lse[t] - want["lse"]) <= log_tol(want["lse"]) or lse[t] == want["lse"] or np.isnan(lse[t]) and np.isnan(want["lse"])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,pad,offset", [(1, 0, 0), (7, 2, 3), (255, 1, 5), (1000, 8, 0), (5003, 0, 7), (32000, 0, 0), (151936, 0, 0)])
def test_topk(dtype, V, pad, offset):
    for kind in ("normal", "peaked", "ties", "constant", "holes"):
        z = make(3, V, dtype, seed=V, kind=kind, pad=pad, offset=offset)
        for K in sorted({1, min(V, 3), min(V, 20), min(V, 64), min(V, 257), min(V, 1000), min(V, 1024)}):
            check_topk(z, K, tau=1.0 if K % 2 else 1.6)


def test_topk_of_rows_sorted_by_id_and_the_longest_row():
    """All of the top in one stretch of ids: one CTA's share."""
    V = 524288
    z = torch.arange(V, dtype=torch.float32).mul_(1e-4)[None].repeat(2, 1).cuda()
    z[1] = z[1].flip(0)
    for K in (1, 100, 1024):
        check_topk(z, K)
    check_sample(z, uniform(2, 3), top_k=300)
    check_sample(z, uniform(2, 3), top_p=0.5)


def test_topk_of_rows_without_a_distribution():
    z = make(4, 1000, "fp16", seed=3)
    z[0] = -np.inf
    z[1, 5] = np.nan
    z[3, 0] = np.inf
    check_topk(z, 17, expect_status=binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT)


def test_empty_batches():
    z = torch.zeros((0, 100), device="cuda")
    assert binding.pods_sample(z, torch.zeros(0, device="cuda"))[0].numel() == 0
    assert binding.pods_topk(z, 5)[0].shape == (0, 5)


@pytest.mark.parametrize("dtype,T,V,pad", [("bf16", 1100, 32001, 0), ("fp32", 3500, 5003, 1), ("fp16", 230, 151936, 0), ("bf16", 34000, 1000, 8),
                                            ("fp32", 130, 151936, 0)])
def test_many_rows_without_filters(dtype, T, V, pad):
    """Enough rows that each cluster takes several in a row (slots of the ring used more than once), rows that fp64 decides,
    rows without a distribution among them."""
    z = make(T, V, dtype, seed=T, kind="normal", pad=pad)
    z[5] = -np.inf
    z[T // 2, V - 1] = np.nan
    u = uniform(T, 13)
    status = binding.new_status()
    tokens, logp, logq = binding.pods_sample(z, u, temperature=1.5, want_logq=True, status=status)
    again = binding.pods_sample(z, u, temperature=1.5, want_logq=True)
    torch.cuda.synchronize()
    assert binding.read_status(status) == binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT
    assert all(torch.equal(a, b) or (torch.isnan(a) == torch.isnan(b)).all() for a, b in zip((tokens, logp, logq), again))
    rows = sorted({0, 1, 5, T // 2, T - 1} | set(range(0, T, max(1, T // 150))))
    sub = z[rows].contiguous()
    want_rows = sub.double().cpu().numpy()
    tok, lp, un = tokens.cpu().numpy(), logp.cpu().numpy().astype(np.float64), u.cpu().numpy()
    for k, t in enumerate(rows):
        want = rollout.sample_row(want_rows[k], float(un[t]), 1.5)
        if want["edge"] <= EDGE:
            continue
        assert tok[t] == want["token"], t
        assert want["token"] < 0 or abs(lp[t] - want["logp"]) <= log_tol(want["logp"])
    # every row against the way for few rows, which takes a mask
    live = torch.ones(T, dtype=torch.uint8, device="cuda")
    other = binding.pods_sample(z, u, temperature=1.5, mask=live)
    assert torch.equal(tokens, other[0])


# ---- random numbers far below the steps of the usual generators ------------------------------------------------------------

def check_small_u(z, u, **settings):
    """The oracle's tokens; that the draws are asked for fairly is a share of the drawn point itself: an fp64 sum of V <= 2^18
    terms in any order is off by at most 2^18 * 2^-53 = 3e-11 of itself."""
    status = binding.new_status()
    tokens, logp, _ = binding.pods_sample(z, u, status=status, **settings)
    torch.cuda.synchronize()
    assert binding.read_status(status) == 0
    rows, un = z.double().cpu().numpy(), u.cpu().numpy().astype(np.float64)
    for t in range(z.shape[0]):
        want = rollout.sample_row(rows[t], un[t], min_p=float(np.float32(settings.get("min_p", 0.0))), top_k=settings.get("top_k", 0))
        run = np.cumsum(np.exp(rows[t] - rows[t].max())[np.sort(want["kept"])])
        target = un[t] * run[-1]
        assert np.abs(run[:-1] - target).min() > 1e-9 * target
        assert int(tokens[t]) == want["token"], (t, un[t], int(tokens[t]), want["token"])
        assert abs(float(logp[t]) - want["logp"]) <= log_tol(want["logp"])


@pytest.mark.parametrize("V,dtype", [(600, "fp32"), (5003, "bf16"), (5003, "fp32"), (151936, "bf16")])
def test_weights_that_fp32_flushes_can_be_drawn(V, dtype):
    """The ids ahead of the maximum weigh 2 to 4e-39 of it, below the normal numbers of fp32: u = 1e-39 draws the first of them,
    u = 1e-38 the fourth."""
    z = torch.full((8, V), -30.0)
    z[:, 0] = -88.5
    z[:, 1:7] = -89.0
    z[:, 7] = 0.0
    z[:, V - 1] = -95.0                                    # what top_k = V - 1 leaves out
    z = z.to(DT[dtype]).cuda()
    u = torch.tensor([1e-39, 4.5e-39, 1e-38, 1e-20, 1.5e-13, 1e-7, 0.5, 1e-45]).cuda()
    check_small_u(z, u)
    check_small_u(z, u, min_p=1e-44)                       # a floor below every id: by list at V = 600, by threshold above
    check_small_u(z, u, top_k=V - 1)
    T = (64 << 20) // (V * z.element_size()) + 1           # rows enough for the pipeline
    many = binding.pods_sample(z.repeat(T // 8 + 1, 1), u.repeat(T // 8 + 1))
    few = binding.pods_sample(z, u)
    assert (many[0].view(-1, 8) == few[0]).all()


@pytest.mark.parametrize("V,dtype", [(600, "fp32"), (5003, "bf16"), (50257, "fp32"), (151936, "bf16")])
def test_light_ids_ahead_of_a_heavy_one_are_told_apart(V, dtype):
    """Ids of about 1e-20 of the row's mass, one that holds the rest somewhere behind them, and points drawn among the last of the
    light ones: what lies ahead of the heavy id must not be rounded off by it (2^-53 of it is ten thousand of them)."""
    heavy = sorted({4, 9, 40, 130, 333, 590, V // 3, V // 2 + 5, V - 300, V - 2})
    T = 2 * len(heavy)
    z = -46.0 + torch.randn((T, V), generator=torch.Generator().manual_seed(V))
    for t in range(T):
        z[t, heavy[t // 2]] = 0.0
    z = z.to(DT[dtype])
    e = np.exp(z.double().numpy())
    u = torch.zeros(T)
    for t in range(T):
        last = heavy[t // 2] - 1 - t % 2                   # half way into the last light id ahead, or the one before it
        u[t] = (e[t, :last].sum() + 0.5 * e[t, last]) / e[t].sum()
    z, u = z.cuda(), u.cuda()
    check_small_u(z, u)
    check_small_u(z, u, min_p=1e-30)                       # a floor below every id: by list at V = 600, by threshold above
    n = (64 << 20) // (T * V * z.element_size()) + 1       # rows enough for the pipeline
    many = binding.pods_sample(z.repeat(n, 1), u.repeat(n))
    few = binding.pods_sample(z, u)
    assert (many[0].view(n, T) == few[0]).all()


def test_top_k_of_any_size_is_off_above_the_row():
    z = make(16, 1000, "fp32", seed=12)
    u = uniform(16, 8)
    want = binding.pods_sample(z, u, want_logq=True)
    for k in (0, -1, 1000, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 40 + 3, -2 ** 31, -2 ** 32 + 2, np.int64(2 ** 33 + 1)):
        got = binding.pods_sample(z, u, top_k=k, want_logq=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def same_bits(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b)) if a.is_floating_point() else a == b).all())


@pytest.mark.parametrize("dtype,T,V,pad", [("bf16", 1100, 32001, 0), ("fp16", 230, 151936, 8), ("bf16", 34000, 1000, 0), ("fp32", 130, 151936, 1)])
def test_many_rows_without_filters_the_same_bits_every_time_and_under_a_mask(dtype, T, V, pad):
    """The pipeline's ring, marks and numbers leave nothing to the order in which its warps come: the same bits each time, rows
    without a distribution among them.  Then half of the rows masked: those are left as they were, the others are as before."""
    z = make(T, V, dtype, seed=T + 1, kind="normal", pad=pad)
    z[3] = -np.inf
    z[T // 3, 0] = np.nan
    u = uniform(T, 14)
    status = binding.new_status()
    first = binding.pods_sample(z, u, temperature=1.3, want_logq=True, status=status)
    assert binding.read_status(status) == binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT
    for _ in range(4):
        again = binding.pods_sample(z, u, temperature=1.3, want_logq=True)
        assert all(same_bits(a, b) for a, b in zip(first, again))
    tok, lp, lq = (x.cpu().numpy().astype(np.float64) for x in first)
    un = u.cpu().numpy()
    for t in sorted({0, 1, 3, T // 3, T - 1} | set(range(0, T, max(1, T // 40)))):
        want = rollout.sample_row(z[t].double().cpu().numpy(), float(un[t]), float(np.float32(1.3)))
        if want["edge"] <= EDGE:
            continue
        assert tok[t] == want["token"], t
        if want["token"] >= 0:
            assert abs(lp[t] - want["logp"]) <= log_tol(want["logp"]) and abs(lq[t] - want["logq"]) <= log_tol(want["logq"])
        else:
            assert np.array_equal([lp[t], lq[t]], [want["logp"], want["logq"]], equal_nan=True)
    mask = (torch.arange(T, device="cuda") % 7 < 4).to(torch.uint8)
    live = mask.bool()
    z[~live] = float("nan")                                # not read
    z[3], z[T // 3] = 0.0, 0.0
    given = [torch.full((T,), 77, dtype=torch.int32, device="cuda"), torch.full((T,), 2.5, device="cuda"), torch.full((T,), -3.5, device="cuda")]
    status = binding.new_status()
    binding.pods_sample(z, u, temperature=1.3, mask=mask, tokens=given[0], logp=given[1], logq=given[2], status=status)
    assert binding.read_status(status) == 0
    assert (given[0][~live] == 77).all() and (given[1][~live] == 2.5).all() and (given[2][~live] == -3.5).all()
    live[3] = live[T // 3] = False                         # other rows now
    assert torch.equal(given[0][live], first[0][live])
    for x, y in zip(given[1:], first[1:]):                 # two kernels: each within log_tol of the exact value
        x, y = x[live].double().cpu().numpy(), y[live].double().cpu().numpy()
        assert (np.abs(x - y) <= 2 * log_tol(y)).all()
