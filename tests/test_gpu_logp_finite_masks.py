"""pods_logp_chunk on rows whose ids are ruled out by a large negative number in place of -inf: the values, and what they cost."""
import pytest
import torch

from logp_plain import compare, rows64

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def fills(dtype):
    least = torch.finfo(TYPES[dtype]).min
    return (least, least / 2, -2.0e4, -3.0e3) if dtype == "fp16" else (least, -1e30, -1e9, -6e6, -4e6, -3e6, -2.5e6, -1e6, -1e4)


# the kernels for few rows, for many short ones, the pipeline in groups and whole, on clusters of one CTA and of two
SHAPES = [(24, 5000), (1300, 1000), (2400, 16500), (160, 70001), (300, 151936)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,V", SHAPES)
def test_values(binding, dtype, T, V):
    """Allowed ids in one stretch, at either end only, spread, and none; their logits around 0, and far below it where the type has
    room, so that they lie on both sides of what fp32 exponents resolve and next to the mask's number."""
    g = torch.Generator(device="cuda").manual_seed(V)
    ids = torch.arange(V, device="cuda")
    some = fills(dtype)
    z = torch.empty((T, V), dtype=TYPES[dtype], device="cuda")
    low = (0.0, -5e4, 0.0) if dtype == "fp16" else (0.0, -1.4e6, -1.46e6, -2.0e6, -2.89e6, -2.92e6, -3.5e6, 0.0, -2e5)
    for t in range(T):
        x = torch.randn(V, generator=g, device="cuda") * 3.0 + low[(t // 5) % len(low)]
        allowed = (((ids >= V // 3) & (ids < V // 3 + V // 10)), ids == V - 1, ids < 3, ids % 97 == 5, ids < 0)[t % 5]
        z[t] = torch.where(allowed, x, some[(t // 3) % len(some)]).to(z.dtype)
    # a plain row, and one of -inf but for one id, among them
    z[T // 2] = torch.randn(V, generator=g, device="cuda").to(z.dtype)
    z[T // 2 + 1] = torch.where(ids == V // 2, 1.0, -torch.inf).to(z.dtype)
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    tok[::2] = z[::2].float().argmax(1).to(torch.int32)
    want = rows64(z, tok, 1.0)
    status = binding.new_status()
    got = binding.pods_logp_chunk(z, tok, want_lse=True, want_entropy=True, status=status)
    compare(got, want)
    compare(binding.pods_logp_chunk(z, tok, want_lse=True, status=status), want)
    assert binding.read_status(status) == 0


def shortest(f, n=12):
    """Device time of a call, the shortest of n."""
    f()
    times = []
    for _ in range(n):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("where", ["spread", "at the end"])
@pytest.mark.parametrize("T,V", [(592, 151936), (3000, 32000), (20000, 8000), (1000, 16000)])
@pytest.mark.parametrize("fill", [-1e9, "least"])
def test_cost(binding, T, V, fill, where):
    """Nine ids in ten ruled out, so that many threads see nothing else at first: less than twice the call without a mask.  Rows that
    are taken in fp64 for it cost 2.8 (few rows) to 70 times as much."""
    g = torch.Generator(device="cuda").manual_seed(1)
    z = (torch.randn((T, V), generator=g, device="cuda") * 2.0).to(torch.bfloat16)
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    logp = torch.empty(T, device="cuda")
    plain = shortest(lambda: binding.pods_logp_chunk(z, tok, logp=logp))
    fill = torch.finfo(z.dtype).min if fill == "least" else fill
    if where == "spread":
        z.masked_fill_(torch.rand((T, V), generator=g, device="cuda", dtype=torch.float16) < 0.9, fill)
    else:
        z[:, :V - V // 10] = fill
    assert shortest(lambda: binding.pods_logp_chunk(z, tok, logp=logp)) < 2.0 * plain
