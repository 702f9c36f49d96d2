"""pods_distill_chunk against the fp64 oracle.

Sums of exponentials carry SUM_RTOL (see test_gpu_sample.py).  kl = H - A + Q log Z + r (log r - log S2 + log Z): the two
sums enter through logarithms with factors Q, r and r, then one rounding to fp32.  A gradient entry is a sum of terms (the
oracle's `terms` is the sum of their absolute values): each carries SUM_RTOL, the exponent's own error of 9e-8 per unit of
|z - max| / tau ((2^-24 + 2^-25), natural units), 2^-22.5 of the exponential and three fp32 roundings; the entry is then
rounded to the logits' type, half a step: eps / 2 of the value, or half the smallest subnormal.  A bf16 entry outside the list
may be the product of an exponential that was itself kept as bf16, half a step more."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rollout
from paper_2504_13818_b200 import binding

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SUM_RTOL = 1.6e-6
# the smallest step that an entry can be off by: half the smallest fp16; where the type reaches as far as fp32, what the
# exponential loses by giving 0 below 2^-126 (e <= 1 scales with a factor of at most g)
HALF_SUBNORMAL = {"bf16": 2.0 ** -126, "fp16": 2.0 ** -25, "fp32": 2.0 ** -126}


def make(T, V, K, dtype, seed, pad=0, offset=0, M=3, holes=False, sharp=False):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((T, V), generator=g) * 3.0
    if sharp:
        z[:, 0] += 60.0
    if holes and V > 2:
        z[torch.rand((T, V), generator=g) < 0.5] = -np.inf
        z[:, V // 2] = 0.25
    flat = torch.full((offset + T * (V + pad) + 16,), 6.0e4, dtype=DT[dtype]).cuda()
    rows = flat[offset:offset + T * (V + pad)].view(T, V + pad)[:, :V]
    rows.copy_(z.to(DT[dtype]))
    teacher = torch.randn((T, V), generator=g) * 2.0 + torch.where(torch.isfinite(z), z, torch.zeros(())) * 0.7
    values, ids = teacher.topk(K, dim=1)
    cuts = np.linspace(0, T, M + 1).astype(np.int64)
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8)
    return dict(z=rows, teacher=teacher, ids=ids.to(torch.int32).cuda(), values=values.cuda(), cu=torch.from_numpy(cuts).cuda(),
                mask=mask.cuda(), dtype=dtype)


def run(b, tau=1.0, rest=False, lse=True, mask=True, grad_scale=1.0, want_grad=True, dlogits=None, expect_status=0):
    L = torch.logsumexp(b["teacher"].double() / np.float32(tau), 1).float().cuda() if lse else None
    m = b["mask"] if mask else None
    weight = binding.grpo_seq_weights(m, b["cu"])
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    status = binding.new_status()
    kl, dl = binding.pods_distill_chunk(b["z"], b["ids"], b["values"], L, weight, b["cu"], 0, m, acc, temperature=tau, rest=rest,
                                        want_grad=want_grad, grad_scale=grad_scale, dlogits=dlogits, status=status)
    torch.cuda.synchronize()
    assert binding.read_status(status) == expect_status
    return dict(kl=kl.cpu().numpy().astype(np.float64), dl=None if dl is None else dl, loss=float(acc.item()), L=L,
                weight=weight.cpu().numpy(), mask=np.ones(b["z"].shape[0], np.uint8) if m is None else m.cpu().numpy())


def check(b, got, tau=1.0, rest=False, grad_scale=1.0, z=None):
    z = (b["z"] if z is None else z).double().cpu().numpy()
    T = z.shape[0]
    ids, values = b["ids"].cpu().numpy(), b["values"].cpu().numpy()
    L = None if got["L"] is None else got["L"].cpu().numpy().astype(np.float64)
    row = oracle.seq_of_rows(b["cu"].cpu().numpy())
    tau = float(np.float32(tau))
    dl = None if got["dl"] is None else got["dl"].double().cpu().numpy()
    half = torch.finfo(DT[b["dtype"]]).eps / 2
    loss, loss_tol = 0.0, 1e-12
    for t in range(T):
        w = got["weight"][row[t]] * (got["mask"][t] != 0)
        if w == 0:
            assert got["kl"][t] == 0 and (dl is None or (dl[t] == 0).all())
            continue
        want = rollout.distill_row(z[t], ids[t], values[t], None if L is None else L[t], tau, rest)
        if not np.isfinite(want["kl"]):
            assert np.isnan(got["kl"][t]) == np.isnan(want["kl"]) and (np.isnan(want["kl"]) or got["kl"][t] == want["kl"])
            loss = np.nan
        else:
            tol = (want["Q"] + 2 * want["r"]) * SUM_RTOL + 1e-11          # 1e-11: fp64 sums of terms of up to 1e3
            assert abs(got["kl"][t] - want["kl"]) <= tol + 2.0 ** -24 * abs(want["kl"]), (t, got["kl"][t], want["kl"], tol)
            loss += w * want["kl"]
            loss_tol += w * tol
        if dl is not None:
            if np.isnan(want["kl"]):
                assert np.isnan(dl[t]).all()
                continue
            g = grad_scale * w / tau
            depth = np.where(np.isfinite(z[t]), z[t].max() - z[t], 0.0) / tau
            err = np.abs(dl[t] - g * want["grad"])
            bar = g * want["terms"] * (SUM_RTOL + 9e-8 * depth + 2.0 ** -22.5 + 3 * 2.0 ** -24)
            steps = np.ones(z.shape[1])
            if b["dtype"] == "bf16":
                # fl(fl(e) c): (1 + half)^2 - 1 of the value; a listed id's entry is computed apart and rounded once
                steps[:] = 2 + half
                steps[ids[t][(ids[t] >= 0) & (ids[t] < z.shape[1])]] = 1
            bar = bar * (1 + half) + half * steps * np.abs(g * want["grad"]) + HALF_SUBNORMAL[b["dtype"]] * max(1.0, g)
            assert (err <= bar).all(), (t, int(np.argmax(err - bar)), float((err - bar).max()))
    if np.isfinite(loss):
        assert abs(got["loss"] - loss) <= loss_tol
    else:
        assert not np.isfinite(got["loss"])


MODES = [dict(rest=False, lse=False), dict(rest=False, lse=True), dict(rest=True, lse=True)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,K,pad,offset", [(1, 1, 0, 0), (7, 3, 2, 3), (9, 9, 0, 0), (255, 17, 1, 5), (1000, 300, 8, 0), (5003, 64, 0, 7), (32000, 1024, 0, 0)])
def test_lengths_alignments_and_modes(dtype, V, K, pad, offset):
    b = make(10, V, K, dtype, seed=V + K, pad=pad, offset=offset)
    for i, mode in enumerate(MODES):
        for tau in (1.0, 2.5, 0.4):
            got = run(b, tau=tau, mask=i != 1, grad_scale=[1.0, 0.5, 64.0][i], **mode)
            check(b, got, tau=tau, rest=mode["rest"], grad_scale=[1.0, 0.5, 64.0][i])


@pytest.mark.parametrize("dtype,V", [("bf16", 151936), ("fp32", 151936), ("fp16", 50257), ("bf16", 300001), ("fp32", 524288)])
def test_long_rows(dtype, V):
    b = make(5, V, 50, dtype, seed=V)
    for mode in MODES:
        check(b, run(b, tau=1.3, **mode), tau=1.3, rest=mode["rest"])


def test_rows_far_apart():
    """Offsets past 2^32 elements, the gradient in place; rows enough for the pipeline."""
    T, V, pitch = 112, 151936, 40_000_003
    b = make(T, V, 30, "bf16", seed=3)
    z = b["z"]
    flat = torch.empty(T * pitch, dtype=torch.bfloat16, device="cuda")
    b["z"] = flat.view(T, pitch)[:, :V]
    b["z"].copy_(z)
    check(b, run(b, rest=True, dlogits=b["z"]), rest=True, z=z)


@pytest.mark.parametrize("sign", [1, -1])
def test_logits_where_exponents_of_two_run_out_of_fractions(sign):
    """Maxima of a row's parts lie on both sides of the exponent 2^23, where references change their form."""
    T, V = 520, 17001
    b = make(T, V, 20, "fp32", seed=4)
    z = b["z"].double() + sign * 2.0 ** 23 * np.log(2.0) + torch.linspace(-12, 6, T, device="cuda", dtype=torch.float64)[:, None]
    b["z"].copy_(z.float())
    for t in (T, 5):                                                     # the pipeline, and the kernel for few rows
        part = dict(b, z=b["z"][:t], ids=b["ids"][:t], values=b["values"][:t], teacher=b["teacher"][:t], mask=b["mask"][:t],
                    cu=torch.tensor([0, t // 2, t], device="cuda"))
        for mode in MODES:
            check(part, run(part, **mode), rest=mode["rest"])


@pytest.mark.parametrize("V", [9, 1000, 50257])
def test_holes_and_sure_policies(V):
    """-inf logits inside and outside the list (kl +inf, gradient finite); a policy with all but e^-60 on one id, where 1 - s
    as a difference would be zero."""
    b = make(6, V, 5, "fp32", seed=V, holes=True)
    for mode in MODES:
        check(b, run(b, **mode), rest=mode["rest"])
    b = make(6, V, 5, "fp32", seed=V, sharp=True)
    b["ids"][:, 4] = 0
    b["ids"][:, :4] = torch.arange(1, 5, dtype=torch.int32)
    for mode in MODES:
        check(b, run(b, **mode), rest=mode["rest"])


def test_ids_twice_unused_and_out_of_range():
    b = make(8, 1000, 40, "fp32", seed=1)
    for mode in MODES:
        b["ids"][1, 7] = b["ids"][1, 30]
        b["ids"][2, :] = 5
        b["ids"][3, 10:] = -1
        b["ids"][4, :] = -1
        check(b, run(b, mask=False, **mode), rest=mode["rest"])
        b["ids"][5, 0] = 1000
        b["ids"][6, 3] = -7
        check(b, run(b, mask=False, expect_status=binding.STATUS_TOKEN_RANGE, **mode), rest=mode["rest"])
        b["ids"][5, 0], b["ids"][6, 3] = 1, 1


def test_list_holding_the_whole_row():
    b = make(4, 64, 64, "fp32", seed=2)
    for mode in MODES:
        check(b, run(b, mask=False, **mode), rest=mode["rest"])


def test_rows_without_a_distribution():
    b = make(6, 1000, 8, "bf16", seed=3)
    b["mask"][:] = 1
    b["z"][0] = -np.inf
    b["z"][2, 999] = np.nan
    b["z"][4, int(b["ids"][4, 0])] = np.inf
    for mode in MODES:
        check(b, run(b, expect_status=binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT, **mode), rest=mode["rest"])
    b["mask"][::2] = 0                                      # under the mask none of it counts
    for mode in MODES:
        got = run(b, **mode)
        check(b, got, rest=mode["rest"])
        assert np.isfinite(got["loss"])


@pytest.mark.parametrize("pad", [0, 3, 8])
def test_in_place_loss_alone_and_a_pitched_gradient(pad):
    b = make(9, 5003, 20, "bf16", seed=4, pad=pad)
    got = run(b, rest=True)
    alone = run(b, rest=True, want_grad=False)
    assert alone["dl"] is None and np.array_equal(alone["kl"], got["kl"]) and alone["loss"] == got["loss"]
    wide = torch.full((9, 5003 + 13), 5.0, dtype=torch.bfloat16, device="cuda")
    pitched = run(b, rest=True, dlogits=wide[:, 4:5007])
    assert torch.equal(pitched["dl"], got["dl"]) and (wide[:, :4] == 5.0).all() and (wide[:, 5007:] == 5.0).all()
    before = b["z"].clone()
    behind = b["z"].as_strided((9, pad), b["z"].stride(), b["z"].storage_offset() + 5003).clone() if pad else None
    inplace = run(b, rest=True, dlogits=b["z"])
    assert torch.equal(b["z"], got["dl"]) and np.array_equal(inplace["kl"], got["kl"])
    if pad:
        assert torch.equal(b["z"].as_strided((9, pad), b["z"].stride(), b["z"].storage_offset() + 5003), behind)
    check(b, got, rest=True, z=before)


def test_chunks_add_up_and_weights_follow_the_rollouts():
    b = make(40, 1000, 12, "bf16", seed=5, M=7)
    whole = run(b, rest=True)
    weight = binding.grpo_seq_weights(b["mask"], b["cu"])
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    for lo, hi in ((0, 13), (13, 14), (14, 40)):
        kl, dl = binding.pods_distill_chunk(b["z"][lo:hi], b["ids"][lo:hi], b["values"][lo:hi], whole["L"][lo:hi], weight, b["cu"],
                                            lo, b["mask"][lo:hi], acc, rest=True)
        assert np.array_equal(kl.cpu().numpy(), whole["kl"][lo:hi].astype(np.float32)) and torch.equal(dl, whole["dl"][lo:hi])
    assert abs(float(acc.item()) - whole["loss"]) <= 1e-12 * max(1.0, abs(whole["loss"]))


def test_many_rollouts_find_their_weights():
    """5000 rollouts of 0 to 3 tokens: the row-to-rollout search over more than two levels of 32."""
    rng = np.random.default_rng(6)
    lengths = rng.integers(0, 4, 5000)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    T = int(cu[-1])
    g = torch.Generator().manual_seed(6)
    z = torch.randn((T, 16), generator=g).cuda()
    values, ids = torch.randn((T, 16), generator=g).topk(3, dim=1)
    weight = torch.arange(1, 5001, dtype=torch.float64).cuda()
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    kl, _ = binding.pods_distill_chunk(z, ids.to(torch.int32).cuda(), values.cuda(), None, weight, torch.from_numpy(cu).cuda(), 0, None, acc)
    want = (weight.cpu().numpy()[oracle.seq_of_rows(cu)] * kl.double().cpu().numpy()).sum()
    assert abs(float(acc.item()) - want) <= 2.0 ** -23 * abs(want)      # kl is rounded to fp32, the sum is not


def test_gradient_agrees_with_differences_of_the_loss():
    V = 50
    b = make(4, V, 6, "fp32", seed=7)
    got = run(b, tau=1.5, rest=True, mask=False)
    z0 = b["z"].clone()
    h = 0.05
    for t, v in ((0, int(b["ids"][0, 0])), (1, int(b["ids"][1, 5])), (2, 17), (3, 33)):
        losses = []
        for step in (h, -h):
            b["z"].copy_(z0)
            b["z"][t, v] += step
            losses.append(run(b, tau=1.5, rest=True, mask=False)["loss"])
        slope = (losses[0] - losses[1]) / (2 * h)
        w = got["weight"][oracle.seq_of_rows(b["cu"].cpu().numpy())[t]]
        # h^2 / 6 of a third derivative below 2 w, and the two losses' own errors of 4e-6 w over 2 h
        assert abs(slope - float(got["dl"][t, v])) <= w * (2 * h * h / 6 + 4 * SUM_RTOL / (2 * h) * 2 + 1e-6)
    b["z"].copy_(z0)


def test_another_stream_a_captured_graph_and_the_same_bits_twice():
    b = make(30, 50257, 33, "bf16", seed=8, M=4)
    want = run(b, rest=True)
    again = run(b, rest=True)
    assert torch.equal(want["dl"], again["dl"]) and np.array_equal(want["kl"], again["kl"]) and want["loss"] == again["loss"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run(b, rest=True)
    assert torch.equal(want["dl"], other["dl"]) and want["loss"] == other["loss"]
    weight = binding.grpo_seq_weights(b["mask"], b["cu"])
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    kl, dl = torch.zeros(30, device="cuda"), torch.zeros_like(want["dl"])
    ws = torch.empty(binding.pods_distill_chunk_workspace_bytes(30), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        acc.zero_()
        binding.pods_distill_chunk(b["z"], b["ids"], b["values"], want["L"], weight, b["cu"], 0, b["mask"], acc, kl=kl, dlogits=dl,
                                   workspace=ws, rest=True)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dl, want["dl"]) and float(acc.item()) == want["loss"]


def test_rollout_teacher_list_distillation_and_objective_in_one_run():
    """As they are used: tokens drawn from the policy with their log-probs, the teacher's lists, the divergence's gradient and
    the policy objective on the drawn tokens, whose ratio is 1 on the first step."""
    T, V, K, M = 48, 32000, 32, 4
    g = torch.Generator().manual_seed(9)
    policy = (torch.randn((T, V), generator=g) * 2.5).to(torch.bfloat16).cuda()
    teacher = (policy.float() + torch.randn((T, V), generator=g).cuda()).to(torch.bfloat16)
    u = torch.rand(T, generator=g).cuda()
    status = binding.new_status()
    tokens, old_logp, _ = binding.pods_sample(policy, u, status=status)
    ids, values, lse = binding.pods_topk(teacher, K, status=status)
    cu = torch.arange(0, T + 1, T // M, dtype=torch.int64).cuda()
    weight = binding.grpo_seq_weights(None, cu)
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    kl, dl = binding.pods_distill_chunk(policy, ids, values, lse, weight, cu, 0, None, acc, rest=True, status=status)
    adv = torch.tensor([1.0, -1.0, 0.5, -0.5]).cuda()
    loss, logp, dpolicy = binding.grpo_loss_fwd_bwd(policy, tokens, old_logp, None, adv, None, 0.2, 0.0, cu, status=status)
    torch.cuda.synchronize()
    assert binding.read_status(status) == 0
    assert (logp - old_logp).abs().max() <= 1e-5             # both are log softmax(policy)[token], to 2 sums and 2 roundings at 16
    z = policy.double().cpu().numpy()
    teacher_rows = teacher.double().cpu().numpy()
    for t in range(0, T, 7):
        assert int(tokens[t]) == rollout.sample_row(z[t], float(u[t]))["token"]
        want = rollout.topk_row(teacher_rows[t], K)
        assert np.array_equal(ids[t].cpu().numpy(), want["ids"])
        ref = rollout.distill_row(z[t], want["ids"], want["values"], float(lse[t]), rest=True)
        assert abs(float(kl[t]) - ref["kl"]) <= 3 * SUM_RTOL + 2.0 ** -24 * ref["kl"]
    assert torch.isfinite(dpolicy.float()).all() and torch.isfinite(dl.float()).all() and float(acc.item()) > 0


def test_empty_chunk():
    z = torch.zeros((0, 100), device="cuda")
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    kl, dl = binding.pods_distill_chunk(z, torch.zeros((0, 4), dtype=torch.int32, device="cuda"), torch.zeros((0, 4), device="cuda"), None,
                                        torch.ones(1, dtype=torch.float64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"),
                                        0, None, acc)
    assert kl.numel() == 0 and dl.shape == (0, 100) and float(acc.item()) == 0.0


@pytest.mark.parametrize("dtype,T,V,K,pad,offset", [("bf16", 600, 32000, 64, 0, 0), ("fp32", 500, 17001, 128, 3, 1), ("fp16", 3500, 5003, 33, 8, 5),
                                                    ("bf16", 120, 151936, 8, 0, 0), ("bf16", 17000, 1000, 5, 0, 0), ("fp32", 130, 100003, 20, 0, 0),
                                                    ("fp32", 64, 151936, 128, 1, 0), ("bf16", 60, 300001, 64, 0, 3)])
def test_many_rows(dtype, T, V, K, pad, offset):
    """Enough rows that each cluster takes several in a row (every stage and slot used more than once), with masked rows, ids
    twice, unused entries and rows without a distribution among them; in every mode, with the gradient at another alignment
    than the logits and in place."""
    b = make(T, V, K, dtype, seed=V, pad=pad, offset=offset, M=17)
    b["ids"][3, K - 1] = b["ids"][3, 0]
    b["ids"][T // 2, K // 2:] = -1
    b["ids"][T - 1, :] = -1
    b["mask"][3] = b["mask"][T // 2] = b["mask"][T - 1] = 1
    for i, mode in enumerate(MODES):
        got = run(b, tau=1.7, grad_scale=0.5, **mode)
        check(b, got, tau=1.7, rest=mode["rest"], grad_scale=0.5)
        alone = run(b, tau=1.7, want_grad=False, **mode)
        assert np.array_equal(alone["kl"], got["kl"]) and alone["loss"] == got["loss"]
    b["mask"][5] = b["mask"][7] = 1
    b["mask"][8] = 0
    b["z"][5] = -np.inf
    b["z"][7, V - 1] = np.nan
    b["z"][8, 0] = np.nan
    bits = binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT
    got = run(b, rest=True, expect_status=bits)
    check(b, got, rest=True)
    wide = torch.full((T, V + 13), 5.0, dtype=DT[dtype], device="cuda")
    pitched = run(b, rest=True, dlogits=wide[:, 4:V + 4], expect_status=bits)
    same = lambda x, y: bool(((x == y) | (torch.isnan(x) & torch.isnan(y))).all())  # noqa: E731
    # at another alignment than the logits a bf16 entry is rounded once, not twice, and an fp32 exponential is taken relative
    # to another maximum, which rounds its exponent elsewhere: held to the oracle, not to the bits of `got`
    check(b, pitched, rest=True)
    assert (dtype != "fp16" or same(pitched["dl"], got["dl"])) and (wide[:, :4] == 5.0).all() and (wide[:, V + 4:] == 5.0).all()
    z = b["z"].clone()
    inplace = run(b, rest=True, dlogits=b["z"], expect_status=bits)
    check(b, inplace, rest=True, z=z)
    # the bits of `got` where its rows lie as the logits' do; elsewhere see above
    assert (dtype != "fp16" and (pad, offset) != (0, 0)) or same(inplace["dl"], got["dl"])
    assert np.array_equal(inplace["kl"], got["kl"], equal_nan=True)


@pytest.mark.parametrize("dtype,T,V,K", [("bf16", 12, 1000, 20), ("fp32", 12, 5003, 300), ("bf16", 120, 151936, 20), ("fp32", 520, 17001, 128)])
def test_rollouts_of_weight_zero_leave_no_trace(dtype, T, V, K):
    """Rows that are not masked but whose rollout weighs nothing: ids out of range, NaN in the lists and in the logits raise no
    bit and leave a loss of 0 and a row of zeros; the other rows are as ever."""
    b = make(T, V, K, dtype, seed=11, M=4)
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    weight = torch.tensor([0.25, 0.0, 0.25, 0.0], dtype=torch.float64, device="cuda")
    L = torch.logsumexp(b["teacher"].double(), 1).float().cuda()
    of_row = oracle.seq_of_rows(b["cu"].cpu().numpy())
    dead = torch.from_numpy(np.isin(of_row, (1, 3))).cuda()
    want_acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    want_kl, want_dl = binding.pods_distill_chunk(b["z"], b["ids"], b["values"], L, weight, b["cu"], 0, mask, want_acc, rest=True)
    b["ids"][dead, 0] = V
    b["ids"][dead, K // 2] = -9
    b["values"][dead, 1] = float("nan")
    b["z"][dead, V - 1] = float("nan")
    b["z"][dead, 0] = float("inf")
    for m in (mask, None):
        acc = torch.zeros(1, dtype=torch.float64, device="cuda")
        status = binding.new_status()
        kl, dl = binding.pods_distill_chunk(b["z"], b["ids"], b["values"], L, weight, b["cu"], 0, m, acc, rest=True, status=status)
        torch.cuda.synchronize()
        assert binding.read_status(status) == 0
        assert (kl[dead] == 0).all() and (dl[dead] == 0).all()
        assert torch.equal(kl, want_kl) and torch.equal(dl, want_dl) and torch.equal(acc, want_acc)
    # where a row weighs something, the same id counts
    b["ids"][int((~dead).nonzero()[0]), 0] = V
    status = binding.new_status()
    binding.pods_distill_chunk(b["z"], b["ids"], b["values"], L, weight, b["cu"], 0, mask, acc, rest=True, status=status)
    assert binding.read_status(status) == binding.STATUS_TOKEN_RANGE


@pytest.mark.parametrize("dtype,T,V,K,pad,offset", [("bf16", 260, 100003, 200, 0, 0), ("fp32", 330, 50257, 300, 1, 3), ("fp16", 420, 60000, 129, 8, 5),
                                                    ("bf16", 400, 70001, 1024, 0, 1), ("bf16", 180, 90001, 60, 3, 0)])
def test_several_rows_a_cluster_without_the_pipeline(dtype, T, V, K, pad, offset):
    """Lists above the pipeline's longest, and 32 MB of logits not reached: clusters of several CTAs that take more than one row,
    so the segment, the load barrier and the exchange are used again; masked rows and rows without a distribution among them."""
    b = make(T, V, K, dtype, seed=V, pad=pad, offset=offset, M=9)
    b["mask"][[4, 6, T // 2]] = 1
    b["mask"][[5, T // 2 + 1]] = 0
    b["z"][4] = -np.inf
    b["z"][5] = np.nan
    b["z"][T // 2, V - 1] = np.nan
    b["ids"][6, K - 1] = b["ids"][6, 0]
    b["ids"][T - 1, K // 2:] = -1
    bits = binding.STATUS_EMPTY_ROW | binding.STATUS_NONFINITE_LOGIT
    got = run(b, tau=1.4, rest=True, expect_status=bits)
    # some of the rows against the oracle, as if each were a rollout with the weight of its own
    some = np.unique(np.r_[0:8, T // 2 - 1:T // 2 + 2, T - 2:T, np.arange(0, T, 23)])
    at = torch.from_numpy(some).cuda()
    row = oracle.seq_of_rows(b["cu"].cpu().numpy())
    part = dict(b, z=b["z"][at], ids=b["ids"][at], values=b["values"][at], mask=b["mask"][at], cu=torch.arange(len(some) + 1, device="cuda"))
    check(part, dict(kl=got["kl"][some], dl=got["dl"][at], loss=np.nan, L=got["L"][at], weight=got["weight"][row[some]], mask=got["mask"][some]),
          tau=1.4, rest=True)
    # every row against calls of so few rows that each has a cluster to itself: kl is within (Q + 2 r) SUM_RTOL and half a step of
    # the exact value in both
    acc = torch.zeros(1, dtype=torch.float64, device="cuda")
    weight = binding.grpo_seq_weights(b["mask"], b["cu"])
    for lo in range(0, T, 40):
        hi = min(T, lo + 40)
        kl, dl = binding.pods_distill_chunk(b["z"][lo:hi], b["ids"][lo:hi], b["values"][lo:hi], got["L"][lo:hi], weight, b["cu"], lo,
                                            b["mask"][lo:hi], acc, temperature=1.4, rest=True)
        assert np.allclose(kl.cpu().numpy(), got["kl"][lo:hi], rtol=2.0 ** -23, atol=4 * SUM_RTOL, equal_nan=True)
        assert ((kl == 0).cpu().numpy() == (got["kl"][lo:hi] == 0)).all()
    again = run(b, tau=1.4, rest=True, expect_status=bits)
    assert np.array_equal(again["kl"], got["kl"], equal_nan=True)
    assert bool(((again["dl"] == got["dl"]) | (torch.isnan(again["dl"]) & torch.isnan(got["dl"]))).all())


def test_pipelines_side_by_side_and_in_a_captured_graph():
    """Sampling and distillation at sizes that take their pipelines, on two streams at once and replayed on new inputs: the bits of
    the calls alone."""
    T, V, K = 520, 70001, 40
    b = make(T, V, K, "bf16", seed=21, M=6)
    u = torch.rand(T, generator=torch.Generator().manual_seed(3)).cuda()
    L = torch.logsumexp(b["teacher"].double(), 1).float().cuda()
    weight = binding.grpo_seq_weights(b["mask"], b["cu"])
    ws = [torch.empty(binding.pods_distill_chunk_workspace_bytes(T), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def outputs():
        return dict(tokens=torch.zeros(T, dtype=torch.int32, device="cuda"), logp=torch.zeros(T, device="cuda"), kl=torch.zeros(T, device="cuda"),
                    dl=torch.zeros((T, V), dtype=torch.bfloat16, device="cuda"), acc=torch.zeros(1, dtype=torch.float64, device="cuda"))

    def sample(o):
        binding.pods_sample(b["z"], u, tokens=o["tokens"], logp=o["logp"])

    def distill(o, w):
        o["acc"].zero_()
        binding.pods_distill_chunk(b["z"], b["ids"], b["values"], L, weight, b["cu"], 0, b["mask"], o["acc"], kl=o["kl"], dlogits=o["dl"],
                                   workspace=w, rest=True)

    def alone():
        o = outputs()
        sample(o)
        distill(o, ws[0])
        torch.cuda.synchronize()
        return o

    want = alone()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [outputs() for _ in streams]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                (sample(got[k]), distill(got[k], ws[k])) if k == 0 else (distill(got[k], ws[k]), sample(got[k]))
    torch.cuda.synchronize()
    for o in got:
        assert all(torch.equal(o[n], want[n]) for n in want)
    graph = torch.cuda.CUDAGraph()
    o = outputs()
    with torch.cuda.graph(graph):
        sample(o)
        distill(o, ws[1])
    for seed in (22, 23):
        b["z"].copy_(make(T, V, K, "bf16", seed=seed)["z"])
        u.copy_(torch.rand(T, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        want = alone()
        assert all(torch.equal(o[n], want[n]) for n in want)
