"""pods_grad_norm and pods_adamw against the fp64 oracle.

Tolerances.  m and v: two products and a sum in fp32, the gradient scaled once before: 3 * 2^-24 of the magnitudes added (4 for v,
whose square doubles the gradient's error).  The parameter: its own product and difference, 2^-23 of it, and the update, whose m and
sqrt(v), quotient and scalars are off by less than 16 * 2^-24 together, half a step more for its own type.
8-bit states: the code is the one the random bits choose from the fp64 value, or the next one where a value lies within 2^-16 of
a code of the border, once the value's own error (that of m, half that of v and the root's rounding) is counted."""
import math

import numpy as np
import pytest
import torch

from oracle import adamw

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
SET = dict(beta1=0.9, beta2=0.95, eps=1e-8)


def f32(x):
    return float(np.float32(x))


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def make(binding, sizes, param="fp32", grad="fp32", bits=32, copy=None, seed=0, decay=0.1, lr_scale=1.0, offset=0, warm=True):
    """A table whose states are those of some steps already taken.  offset: elements between the buffers' starts and their use."""
    g = torch.Generator().manual_seed(seed)
    def tensor(n, dtype, scale):
        x = torch.zeros(n + offset, dtype=dtype)
        x[offset:] = torch.randn(n, generator=g) * scale
        return x.cuda()[offset:]
    params = [tensor(n, TYPES[param], 0.05) for n in sizes]
    grads = [tensor(n, TYPES[grad], 0.01) for n in sizes]
    states = []
    for n in sizes:
        if bits == 32:
            m, v = tensor(n, torch.float32, 0.003), tensor(n, torch.float32, 0.01).square_()
            states.append((m, v))
        else:
            blocks = (n + 31) // 32
            code = torch.randint(0, 127, (2, n + offset), generator=g, dtype=torch.uint8)
            sign = torch.randint(0, 2, (n + offset,), generator=g, dtype=torch.uint8) * 128
            scale = torch.randint(100, 116, (2, blocks), generator=g, dtype=torch.uint8)
            states.append(((code[0] | sign).cuda()[offset:], scale[0].cuda(), code[1].cuda()[offset:], scale[1].cuda()))
        if not warm:
            states[-1] = binding.new_adamw_state(params[len(states) - 1], bits)
    copies = [torch.zeros(n, dtype=TYPES[copy], device="cuda") for n in sizes] if copy else None
    return binding.pods_adamw_table(params, grads, states, copies=copies, weight_decay=decay, lr_scale=lr_scale)


def host(t):
    return t.double().cpu().numpy().reshape(-1)


def snapshot(table):
    return [(host(p), host(g), [s.cpu().numpy().copy() for s in st]) for p, g, st in zip(table.params, table.grads, table.states)]


def values(state):
    """fp64 m and second moment."""
    if len(state) == 2:
        return state[0].astype(np.float64), state[1].astype(np.float64)
    return adamw.decode(state[0], state[1]), adamw.decode(state[2], state[3]) ** 2


def check_codes(codes, scales, value, error, bits16, positive):
    size = np.abs(value)
    least, most = np.maximum(size - error, 0.0), size + error
    assert np.all((scales >= adamw.block_exponents(least)) & (scales <= adamw.block_exponents(most)))
    k = scales.astype(np.int64)
    word = (bits16.astype(np.float64) + 0.5) / 65536
    lo, hi = np.floor(adamw.place_on_grid(least, k) + word - 2.0 ** -16), np.floor(adamw.place_on_grid(most, k) + word + 2.0 ** -16)
    if positive:
        lo, hi = np.where(value > 0, np.maximum(lo, 1), lo), np.where(value > 0, np.maximum(hi, 1), hi)
    got = (codes & 127).astype(np.float64)
    bad = (got < lo) | (got > hi)
    assert not bad.any(), (got[bad][:5], lo[bad][:5], hi[bad][:5])
    assert len(lo) < 1000 or np.mean(lo != hi) < 1e-2
    assert not positive or not (codes & 128).any()
    moved = size > error
    assert positive or np.array_equal(((codes & 128) != 0)[moved], (value < 0)[moved])


def check_step(table, before, step, lr, seed=0, stochastic=False, norm=None, max_norm=0.0, grad_scale=1.0, beta1=0.9, beta2=0.95, eps=1e-8):
    first = 0
    b1, b2, eps, lr = f32(beta1), f32(beta2), f32(eps), f32(lr)
    for i, (p0, g0, st) in enumerate(before):
        e = table.entries[i]
        n = p0.size
        m0, v0 = values(st)
        rate = lr * e.lr_scale
        p, m, v = adamw.step(p0, g0, m0, v0, step, rate, b1, b2, eps, decay=e.weight_decay, grad_scale=f32(grad_scale), norm=norm, max_norm=max_norm)
        c = f32(grad_scale) * (max_norm / norm if max_norm > 0 and norm > max_norm else 1.0)
        now = table.states[i]
        bits = adamw.random_bits(seed, step, first, n)
        off_m = 4 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * c * g0)) + 1e-44
        if len(st) == 2:
            assert np.all(np.abs(host(now[0]) - m) <= off_m)
            assert np.all(np.abs(host(now[1]) - v) <= 6 * U * v + 1e-44)
        else:
            ck = [x.cpu().numpy() for x in now]
            check_codes(ck[0], ck[1], m, off_m, bits[1], False)
            check_codes(ck[2], ck[3], np.sqrt(v), 4 * U * np.sqrt(v), bits[2], True)
        # where m is a small difference of larger terms its error counts relative to them
        update = rate / (1 - b1 ** step) * (np.abs(b1 * m0) + np.abs((1 - b1) * c * g0)) / (np.sqrt(v) / math.sqrt(1 - b2 ** step) + eps)
        tol = 3 * U * np.abs(p0) + 16 * U * update
        if table.copies[i] is not None:
            kind = {torch.bfloat16: "bf16", torch.float16: "fp16", torch.float32: "fp32"}[table.copies[i].dtype]
            assert np.all(np.abs(host(table.copies[i]) - p) <= tol + HALF_STEP[kind] * (np.abs(p) + tol) + 2.0 ** -25)
        kind = {torch.bfloat16: "bf16", torch.float16: "fp16", torch.float32: "fp32"}[table.params[i].dtype]
        got = host(table.params[i])
        if stochastic and kind == "bf16":
            grid = np.exp2(np.floor(np.log2(np.maximum(np.abs(p), 2.0 ** -120))) - 7)
            lo = np.floor((np.abs(p) - tol) / grid + bits[0].astype(np.float64) / 65536) * grid
            hi = np.floor((np.abs(p) + tol) / grid + bits[0].astype(np.float64) / 65536) * grid
            sure = (np.abs(p) > 4 * tol) & (np.floor(np.log2(np.abs(p) + tol + 1e-300)) == np.floor(np.log2(np.maximum(np.abs(p) - tol, 1e-300))))
            assert np.all(((np.abs(got) >= lo * (1 - 1e-9)) & (np.abs(got) <= hi * (1 + 1e-9)))[sure])
            assert np.all(np.abs(got - p)[~sure] <= 2 * grid[~sure] + tol[~sure])
        else:
            assert np.all(np.abs(got - p) <= tol + HALF_STEP[kind] * (np.abs(p) + tol) + (2.0 ** -25 if kind == "fp16" else 0))
        first += (n + 31) // 32 * 32


SIZES = [1, 31, 32, 33, 1000, 0, 4096, 4097, 70001, 5]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param,grad,copy", [("fp32", "fp32", None), ("bf16", "fp32", None), ("bf16", "bf16", None), ("fp32", "bf16", "bf16"),
                                             ("fp16", "fp16", None), ("fp32", "fp16", "fp16"), ("bf16", "fp16", "fp32")])
def test_one_step(binding, bits, param, grad, copy):
    n = len(SIZES)
    table = make(binding, SIZES, param, grad, bits, copy, seed=bits, decay=[0.1 * (i % 2) for i in range(n)], lr_scale=[1.0 + 0.5 * (i % 3) for i in range(n)])
    before = snapshot(table)
    norm = binding.pods_grad_norm(table)
    total = math.sqrt(sum((g * g).sum() for _, g, _ in before))
    assert abs(norm.item() - total) <= 4 * U * total
    stochastic = param == "bf16" and grad != "bf16"
    status = binding.new_status()
    binding.pods_adamw(table, 7, 1e-3, norm=norm, max_norm=0.5, stochastic=stochastic, seed=(3 << 40) + 11, status=status, **SET)
    assert binding.read_status(status) == 0
    check_step(table, before, 7, 1e-3, seed=(3 << 40) + 11, stochastic=stochastic, norm=norm.item(), max_norm=0.5)


@pytest.mark.parametrize("bits", [8, 32])
def test_first_step_from_nothing(binding, bits):
    table = make(binding, [100, 5000], "fp32", "fp32", bits, warm=False)
    table.grads[0].zero_()
    table.grads[1][::3] = 0
    before = snapshot(table)
    binding.pods_adamw(table, 1, 0.01, **SET)
    check_step(table, before, 1, 0.01)
    if bits == 8:
        assert (table.states[0][0] == 0).all() and (table.states[0][2] == 0).all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("offset", [1, 2, 4])
def test_tensors_off_the_vectors_boundaries(binding, bits, offset):
    for param, grad in (("fp32", "bf16"), ("bf16", "fp32")):
        table = make(binding, [5, 9000, 64], param, grad, bits, seed=1, offset=offset)
        before = snapshot(table)
        binding.pods_adamw(table, 3, 1e-3, **SET)
        check_step(table, before, 3, 1e-3)
        norm = binding.pods_grad_norm(table.grads, scale=-2.0).item()
        total = 2 * math.sqrt(sum((g * g).sum() for _, g, _ in before))
        assert abs(norm - total) <= 4 * U * total


@pytest.mark.parametrize("count", [24, 25, 352, 353, 433, 700, 1300])
def test_many_tensors(binding, count):
    """Sets that fill one table of either size exactly, and more."""
    rng = np.random.default_rng(count)
    table = make(binding, rng.integers(0, 300, count).tolist(), "bf16", "bf16", 8, seed=count)
    before = snapshot(table)
    norm = binding.pods_grad_norm(table)
    total = math.sqrt(sum((g * g).sum() for _, g, _ in before))
    assert abs(norm.item() - total) <= 4 * U * total
    binding.pods_adamw(table, 2, 1e-2, stochastic=True, seed=5, **SET)
    check_step(table, before, 2, 1e-2, seed=5, stochastic=True)


def test_states_of_both_kinds_in_one_table(binding):
    a, b = make(binding, [5000, 77], "fp32", "fp32", 32), make(binding, [6000, 33], "bf16", "fp32", 8, seed=2)
    both = binding.pods_adamw_table(a.params + b.params, a.grads + b.grads, a.states + b.states)
    before = snapshot(both)
    binding.pods_adamw(both, 4, 1e-3, **SET)
    check_step(both, before, 4, 1e-3)


@pytest.mark.parametrize("grad", ["fp32", "bf16"])
def test_moments_are_those_of_single_roundings_bit_for_bit(binding, grad):
    """Operations of g, m and v rounded one by one: elementary fp32 operations give the same bits, over enough elements to meet every
    last place, and so 8-bit states do not depend on how a product and a sum were put together."""
    n = 1 << 22
    table = make(binding, [n], "fp32", grad, 32, seed=8)
    (m, v), g = table.states[0], table.grads[0].float()
    norm = binding.pods_grad_norm(table)
    assert norm.item() == torch.sqrt(g.double().square().sum()).float().item()
    b1, b2 = f32(0.9), f32(0.95)
    x = g * (1.0 / norm)                               # 1 is max_norm
    want_m = b1 * m + (1.0 - b1) * x
    want_v = b2 * v + (1.0 - b2) * (x * x)
    binding.pods_adamw(table, 3, 1e-3, norm=norm, max_norm=1.0, **SET)
    assert norm.item() > 1 and torch.equal(m, want_m) and torch.equal(v, want_v)


def test_steps_far_below_half_a_unit_keep_their_average(binding):
    """bf16 parameters at 1 (units of 2^-7 above, 2^-8 below) that lose 1e-5 a step: nearest rounding leaves them, random bits keep the
    average.  Of n elements each rounds down with probability 1e-5 * 2^8; six standard deviations."""
    n = 1 << 20
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(n, device="cuda")
    for stochastic in (False, True):
        p.fill_(1.0)
        table = binding.pods_adamw_table([p], [g], [binding.new_adamw_state(p)])
        for step in range(1, 11):
            binding.pods_adamw(table, step, 1e-5, eps=0.0, stochastic=stochastic, seed=1)
        lost = (1 - p.double()).mean().item()
        if not stochastic:
            assert lost == 0
        else:
            q = 1e-5 * 256
            assert abs(lost - 1e-4) < 6 / 256 * math.sqrt(10 * q / n)


def test_8_bit_moments_keep_their_average(binding):
    """n equal elements: after each step the mean of their decoded m is the exact one, within six standard deviations of roundings
    to one of two neighbours (an eighth of a power apart, so at most 2^-4 of the value each, fading with beta)."""
    n, steps = 1 << 18, 40
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.3, device="cuda")
    st = binding.new_adamw_state(p, bits=8)
    table = binding.pods_adamw_table([p], [g], [st])
    m = 0.0
    for step in range(1, steps + 1):
        binding.pods_adamw(table, step, 1e-3, beta1=0.9, beta2=0.99, seed=9)
        m = 0.9 * m + 0.1 * f32(0.3)
        # blocks share a scale, which follows the largest of 32: still every rounding is even in the mean
        mean = float(adamw.decode(st[0].cpu().numpy(), st[1].cpu().numpy()).mean())
        assert abs(mean - m) <= 6 * 0.0625 * 0.3 / math.sqrt(n) * math.sqrt(1 / (1 - 0.81)) + 1e-6, step


def test_a_norm_that_is_no_number_leaves_everything(binding):
    for bad in (float("nan"), float("inf"), -float("inf")):
        for bits in (8, 32):
            table = make(binding, [300, 5000], "bf16", "fp32", bits, copy="fp32")
            table.grads[1][4321] = bad
            kept = [t.clone() for t in table.params + table.copies + [s for st in table.states for s in st]]
            status = binding.new_status()
            norm = binding.pods_grad_norm(table, status=status)
            assert not math.isfinite(norm.item()) and binding.read_status(status) == binding.STATUS_NONFINITE_GRAD
            status.zero_()
            binding.pods_adamw(table, 1, 0.1, norm=norm, max_norm=1.0, status=status, **SET)
            assert binding.read_status(status) == binding.STATUS_NONFINITE_GRAD
            now = table.params + table.copies + [s for st in table.states for s in st]
            assert all(torch.equal(a, b) for a, b in zip(now, kept))
    # without a norm the element is lost, and in 8 bits its block's states, no more
    table = make(binding, [5000], "fp32", "fp32", 8)
    table.grads[0][100] = float("nan")
    binding.pods_adamw(table, 1, 0.1, **SET)
    p, m = table.params[0], adamw.decode(table.states[0][0].cpu().numpy(), table.states[0][1].cpu().numpy())
    assert torch.isnan(p).sum() == 1 and torch.isnan(p[100]) and np.isnan(m[96:128]).all() and np.isfinite(np.delete(m, np.s_[96:128])).all()


@pytest.mark.parametrize("scale", [1e-25, 1e-12, 1.0, 1e12, 1e18])
def test_norms_of_tiny_and_huge_gradients(binding, scale):
    g = [torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda() * scale for n in (10, 5000, 33333)]
    want = math.sqrt(sum(float((x.double() ** 2).sum()) for x in g))
    assert abs(binding.pods_grad_norm(g).item() - want) <= 4 * U * want


@pytest.mark.parametrize("bits", [8, 32])
def test_gradients_whose_square_overflows_or_vanishes(binding, bits):
    """v infinite: the step is 0; v 0 beside a first moment: the step is the moment over eps."""
    table = make(binding, [4096 + 64], "fp32", "fp32", bits, warm=False, decay=0.0)
    p, g = table.params[0], table.grads[0]
    g[5], g[4100] = 1e20, -3e30
    g[64:96] = 1e-30
    before = p.clone()
    binding.pods_adamw(table, 1, 1e-2, beta1=0.5, beta2=0.5, eps=1e-8)
    assert p[5] == before[5] and p[4100] == before[4100] and torch.isfinite(p).all()
    # m-hat = 1e-30 over eps: 1e-24 of a step
    assert torch.equal(p[64:96], before[64:96])
    moved = torch.ones(p.numel(), dtype=torch.bool)
    moved[[5, 4100]] = False
    moved[64:96] = False
    assert ((p - before).abs()[moved.cuda()] <= 1.001e-2).all() and ((p - before).abs()[moved.cuda()] > 0.9e-2).float().mean() > 0.99
    if bits == 32:
        m, v = table.states[0]
        assert m[5].item() == f32(0.5e20) and v[5] == torch.inf and (v[64:96] == 0).all()


def test_norm_of_nothing(binding):
    assert binding.pods_grad_norm([]).item() == 0
    assert binding.pods_grad_norm([torch.zeros(0, device="cuda"), torch.zeros(7, device="cuda", dtype=torch.float16)]).item() == 0
    binding.pods_adamw(binding.pods_adamw_table([], [], []), 1, 0.1)


def test_settings_read_on_the_device_in_a_replayed_graph(binding):
    eager, held = (make(binding, [333, 20000], "bf16", "fp32", 8, seed=4) for _ in range(2))
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-3, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(binding.load().pods_grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    kept = [t.clone() for t in held.params + [s for st in held.states for s in st]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        binding.pods_grad_norm(held, norm=norm, workspace=ws)
        binding.pods_adamw(held, step, lr, norm=norm, max_norm=0.1, stochastic=True, seed=6, **SET)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, held.params + [s for st in held.states for s in st]))
    for k in range(1, 4):
        lr.fill_(1e-3 / k)
        for t in (eager, held):
            t.grads[1].mul_(1.25)
        graph.replay()
        binding.pods_adamw(eager, k, float(lr.item()), norm=binding.pods_grad_norm(eager), max_norm=0.1, stochastic=True, seed=6, **SET)
        assert all(torch.equal(a, b) for a, b in zip(eager.params + [s for st in eager.states for s in st],
                                                     held.params + [s for st in held.states for s in st])), k


def test_two_tables_on_two_streams(binding):
    tables = [make(binding, [100, 300000], "fp32", "bf16", 8, seed=s) for s in (1, 2)]
    again = [make(binding, [100, 300000], "fp32", "bf16", 8, seed=s) for s in (1, 2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for k in range(1, 5):
        for s, t in zip(streams, tables):
            with torch.cuda.stream(s):
                binding.pods_adamw(t, k, 1e-3, norm=binding.pods_grad_norm(t), max_norm=1.0)
    torch.cuda.synchronize()
    for t in again:
        for k in range(1, 5):
            binding.pods_adamw(t, k, 1e-3, norm=binding.pods_grad_norm(t), max_norm=1.0)
    for a, b in zip(tables, again):
        assert all(torch.equal(x, y) for x, y in zip(a.params + [s for st in a.states for s in st], b.params + [s for st in b.states for s in st]))


def test_other_gradients_and_refusals(binding):
    table = make(binding, [64, 1000], "fp32", "fp32", 32)
    before = snapshot(table)
    new = [torch.randn(64, device="cuda").half(), torch.randn((10, 100), device="cuda").bfloat16()]
    table.set_grads(new)
    binding.pods_adamw(table, 1, 1e-3, **SET)
    check_step(table, [(p, host(g), s) for (p, _, s), g in zip(before, new)], 1, 1e-3)
    for bad in ([new[0]], [new[0], new[1][:5]], [new[0], new[1].t()], [new[0], new[1].double()], [new[0], new[1].cpu()]):
        with pytest.raises(binding.PodsError):
            table.set_grads(bad)
    p = torch.zeros(64, device="cuda")
    with pytest.raises(binding.PodsError, match="shares memory"):
        binding.pods_adamw_table([p, p], [new[0]] * 2, [binding.new_adamw_state(p) for _ in range(2)])
    with pytest.raises(binding.PodsError, match="norm"):
        binding.pods_adamw(table, 1, 1e-3, max_norm=1.0)
    with pytest.raises(binding.PodsError, match="invalid argument"):
        binding.pods_adamw(table, 0, 1e-3)
    with pytest.raises(binding.PodsError, match="made by"):
        binding.pods_adamw([p], 1, 1e-3)


def test_elements_beyond_2_to_the_32(binding):
    n = (1 << 32) + 5000
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    st = binding.new_adamw_state(p, bits=8)
    tail = slice(n - 4999, n)
    g[tail] = torch.randn(4999, generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    table = binding.pods_adamw_table([p], [g], [st])
    norm = binding.pods_grad_norm(table).item()
    want = float(g[tail].double().norm())
    assert abs(norm - want) <= 4 * U * want
    binding.pods_adamw(table, 1, 0.1, stochastic=True, seed=3, **SET)
    assert (p[:n - 4999] == 0).all()
    lo = (n - 4999) // 32 * 32                         # the oracle's blocks begin where the kernel's do
    bits = adamw.random_bits(3, 1, lo, n - lo)
    gd = host(g[lo:])
    m, r = (1 - f32(0.9)) * gd, np.sqrt((1 - f32(0.95)) * gd * gd)
    check_codes(st[0][lo:].cpu().numpy(), st[1][lo // 32:].cpu().numpy(), m, 4 * U * np.abs(m), bits[1], False)
    check_codes(st[2][lo:].cpu().numpy(), st[3][lo // 32:].cpu().numpy(), r, 4 * U * r, bits[2], True)

@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** 126])
def test_the_ends_of_eps(binding, bits, eps):
    """Elements without a gradient stay where they are; the others move by lr at the smallest eps, by less than 2^-100 at the largest."""
    table = make(binding, [4096 + 64], "fp32", "fp32", bits, warm=False, decay=0.0)
    p, g = table.params[0], table.grads[0]
    g.fill_(0.25)
    g[1::2] = 0.0
    before = p.clone()
    binding.pods_adamw(table, 1, 1e-2, eps=eps)
    assert torch.equal(p[1::2], before[1::2])
    want = before[::2].double() - (f32(1e-2) if eps < 1.0 else 0.0)
    assert ((p[::2].double() - want).abs() <= 16 * U * 1e-2 + 2 * U * before[::2].double().abs()).all()
