"""pods_logp_chunk at the sizes that take its kernels for many rows, every row of a batch against fp64: references carried from row to
row, sums' slots used again, more rows of a walk than one look at the mask covers, and rows without a distribution, or out of fp32's
range, ahead of plain ones."""
import pytest
import torch

from logp_plain import compare, rows64

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

# (kernel and CTAs of a cluster on 148 SMs, which test_row_plan.py checks; type, T, V, elements between rows)
SHAPES = [
    ("rows", "bf16", 1300, 1000, 0), ("rows", "bf16", 30000, 1000, 0), ("rows", "fp16", 9001, 1003, 2), ("rows", "fp32", 7200, 2051, 1),
    ("rows", "bf16", 2500, 5, 0), ("rows", "bf16", 4000, 8199, 1), ("rows", "fp32", 1200, 4096, 0),
    ("pipe4", "bf16", 3000, 16000, 0), ("pipe4", "fp16", 2500, 20011, 3), ("pipe4", "fp32", 4800, 17003, 0),
    ("pipe16", "bf16", 5000, 70001, 0), ("pipe16", "fp16", 700, 50257, 7), ("pipe16 x2", "bf16", 2369, 524288, 0),
    ("pipe16 x4", "bf16", 297, 166692, 0), ("pipe16 x8", "fp32", 166, 470531, 0),
]


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def mixed_rows(dtype, T, V, pad, seed):
    """Plain rows and, one in three, one of ten kinds that are not: (logits, tokens, kinds)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.zeros((T, V + pad), dtype=TYPES[dtype], device="cuda")[:, :V]
    kind = torch.randint(0, 30, (T,), generator=g, device="cuda")
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    place = torch.randint(0, V, (T,), generator=g, device="cuda")
    ids = torch.arange(V, device="cuda")
    big = 60000.0 if dtype == "fp16" else 3.0e5
    step = max(1, (1 << 25) // V)
    for a in range(0, T, step):
        x = torch.randn((min(step, T - a), V), generator=g, device="cuda") * 3.0
        k, p = kind[a:a + step, None], place[a:a + step, None]
        x = torch.where((k == 0) & (ids == p), torch.nan, x)
        x = torch.where(k == 1, -torch.inf, x)
        x = torch.where(k == 2, x * (3000.0 if dtype == "fp16" else 1e7), x)       # exponents that fp32 has no fractions for, but in fp16
        x = torch.where(k == 3, x + big, x)
        x = torch.where(k == 4, x - big, x)
        x = torch.where((k == 5) & (ids == p), 300.0, x)
        x = torch.where((k == 6) & (ids == p), torch.inf, x)
        x = torch.where((k == 7) & (ids == tok[a:a + step, None]), -torch.inf, x)
        x = torch.where((k == 8) & (ids <= p), -torch.inf, x)
        x = torch.where(k == 9, ids * (80.0 / V), x)
        z[a:a + step] = x.to(z.dtype)
    return z, tok, kind


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("kernel,dtype,T,V,pad", SHAPES)
def test_every_row(binding, kernel, dtype, T, V, pad, masked):
    z, tok, kind = mixed_rows(dtype, T, V, pad, seed=V + masked)
    mask = live = None
    if masked:
        mask = (torch.rand(T, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") < 0.7).to(torch.uint8)
        if T > 20000:
            mask[T // 3:T // 3 + 6000] = 0             # whole batches of rows without work
        live = mask != 0
        z[~live, V // 2] = torch.nan
    want = rows64(z, tok, 1.0)
    rows = torch.ones(T, dtype=torch.bool, device="cuda") if live is None else live
    status = binding.new_status()

    def call(entropy):
        out = [torch.full((T,), 5.0, device="cuda"), torch.full((T,), 5.0, dtype=torch.float64, device="cuda"),
               torch.full((T,), 5.0, device="cuda") if entropy else None]
        binding.pods_logp_chunk(z, tok, mask=mask, logp=out[0], lse=out[1], entropy=out[2], status=status)
        return out

    flags = 0
    top = z.amax(1)
    if (rows & ~(top < torch.inf)).any():
        flags |= binding.STATUS_NONFINITE_LOGIT
    if (rows & (top == -torch.inf)).any():
        flags |= binding.STATUS_EMPTY_ROW
    for entropy in (False, True):
        got = call(entropy)
        assert binding.read_status(status) == flags
        compare(got, want, rows)
        for x in got:
            assert x is None or (x[~rows] == 5.0).all()
        again = call(entropy)
        assert all(a is None or torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype,T,V", [("bf16", 1300, 1000), ("fp16", 3000, 16000), ("bf16", 700, 70001), ("bf16", 300, 151936)])
def test_rows_behind_the_last_rollout(binding, dtype, T, V):
    """The same kernels where the call leaves out masked rows and rows behind the last rollout, which get 0."""
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn((T, V), generator=g, device="cuda") * 2.0).to(TYPES[dtype])
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8)
    cu = torch.tensor([0, T // 5, T // 2, T - T // 7], device="cuda")
    pairs = torch.tensor([[0, 1], [2, 1]], dtype=torch.int32, device="cuda")
    live = (mask != 0) & (torch.arange(T, device="cuda") < cu[-1])
    want = rows64(z, tok, 1.0)
    z[~live] = torch.nan
    status = binding.new_status()
    _, logp, dlogits, _, _ = binding.pods_preference_fwd_bwd(z, tok, None, mask, cu, pairs, 0.1, status=status)
    assert binding.read_status(status) == 0
    compare((logp, None, None), want, live)
    assert (logp[~live] == 0).all() and (dlogits[~live] == 0).all() and torch.isfinite(dlogits.float()).all()
