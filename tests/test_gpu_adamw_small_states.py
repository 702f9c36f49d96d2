"""8-bit states whose blocks lie so low that their scale, times a beta, is no normal number: the operations of the moments are still those of
the header, each rounded by itself, and the codes those of elementary fp32 operations, every one."""
import numpy as np
import pytest
import torch

from oracle import adamw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2504_13818_b200 import binding as b
    b.load()
    return b


def encode(x, scales, bits16, root):
    """Codes of fp32 numbers (at least 0) in blocks of these scales: a number times 2^(7 - k) has e4m3's code above its lowest 20 bits, where 16
    random bits and a half are added."""
    y = x * np.exp2(7.0 - np.repeat(scales.astype(np.float64), 32)[:x.size]).astype(np.float32)
    code = (y.view(np.uint32).astype(np.uint64) + (bits16 << np.uint64(4)) + np.uint64(8)) >> np.uint64(20)
    return np.where(x > 0, np.maximum(code, 1), 0) if root else code


@pytest.mark.parametrize("beta", [0.9, 0.25, 1e-3])
@pytest.mark.parametrize("scale", [1, 2, 3, 9])
def test_first_moment(binding, beta, scale):
    n = 1 << 18
    rng = np.random.default_rng(scale)
    codes = rng.integers(0, 127, n).astype(np.uint8) | (rng.integers(0, 2, n).astype(np.uint8) << 7)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = binding.new_adamw_state(p, bits=8)
    state[0].copy_(torch.from_numpy(codes))
    state[1].fill_(scale)
    table = binding.pods_adamw_table([p], [g], [state])
    binding.pods_adamw(table, 3, 1e-3, beta1=beta, seed=5)
    m = np.float32(beta) * adamw.decode(codes, np.full(n // 32, scale)).astype(np.float32)
    k = adamw.block_exponents(m.astype(np.float64))
    assert np.array_equal(state[1].cpu().numpy(), k)
    got = state[0].cpu().numpy()
    want = encode(np.abs(m), k, adamw.random_bits(5, 3, 0, n)[1], False)
    assert np.array_equal(got & 127, want.astype(np.uint8))
    assert np.array_equal((got & 128)[m != 0], (codes & 128)[m != 0])
    assert (state[2] == 0).all()


@pytest.mark.parametrize("beta", [0.95, 0.2, 1e-3])
@pytest.mark.parametrize("scale", [64, 65, 66, 67, 71])
def test_second_moment(binding, beta, scale):
    n = 1 << 18
    rng = np.random.default_rng(scale)
    codes = rng.integers(0, 127, n).astype(np.uint8)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = binding.new_adamw_state(p, bits=8)
    state[2].copy_(torch.from_numpy(codes))
    state[3].fill_(scale)
    table = binding.pods_adamw_table([p], [g], [state])
    binding.pods_adamw(table, 3, 1e-3, beta2=beta, seed=5)
    old = adamw.decode(codes, np.full(n // 32, scale)).astype(np.float32)
    v = np.float32(beta) * (old * old)
    root = np.sqrt(v)
    k = adamw.block_exponents(root.astype(np.float64))
    assert np.array_equal(state[3].cpu().numpy(), k)
    got, bits = state[2].cpu().numpy(), adamw.random_bits(5, 3, 0, n)[2]
    # a root is the nearest fp32 number or, one in ten million, the one next to it, which turns a code where its neighbours' differ
    near = [encode(np.nextafter(root, np.float32(d)) if d is not None else root, k, bits, True) for d in (None, 0.0, np.inf)]
    assert np.isin(got.astype(np.int64) - near[0].astype(np.int64), (-1, 0, 1)).all()
    off = got != near[0]
    assert off.sum() <= 2 and ((got == near[1]) | (got == near[2]))[off].all()
    assert (state[0] == 0).all() and (p == 0).all()
