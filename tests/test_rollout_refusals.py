"""What pods_sample, pods_topk and pods_distill_chunk refuse on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2504_13818_b200 import binding

fake = C.c_void_p(256)          # non-null, never dereferenced: every check comes first
INF, NAN = float("inf"), float("nan")


def sample(logits=fake, ldl=100, dtype=0, T=4, V=100, u=fake, tau_row=None, tau=1.0, k_row=None, k=0, p_row=None, p=1.0, m_row=None,
           m=0.0, tokens=fake):
    return binding.load().pods_sample(logits, ldl, dtype, T, V, u, tau_row, tau, k_row, k, p_row, p, m_row, m, None, tokens, None, None,
                                      None, None)


def test_sample_refusals():
    assert sample(T=0) == 0 and sample(T=0, logits=None, u=None, tokens=None) == 0
    assert sample(dtype=3) == 2 and sample(dtype=-1) == 2
    assert sample(V=524289, ldl=524289) == 2
    for bad in (dict(T=-1), dict(V=0), dict(ldl=99), dict(logits=None), dict(u=None), dict(tokens=None), dict(tau=-1.0), dict(tau=INF),
                dict(tau=NAN), dict(p=NAN), dict(m=NAN), dict(logits=C.c_void_p(257)), dict(dtype=2, logits=C.c_void_p(258))):
        assert sample(**bad) == 1, bad


def topk(logits=fake, ldl=100, dtype=0, T=4, V=100, K=5, tau=1.0, ids=fake, values=fake):
    return binding.load().pods_topk(logits, ldl, dtype, T, V, K, tau, None, ids, values, None, None, None)


def test_topk_refusals():
    assert topk(T=0) == 0
    assert topk(dtype=7) == 2 and topk(V=524289, ldl=524289) == 2 and topk(V=2000, ldl=2000, K=1025) == 2
    for bad in (dict(K=0), dict(K=101), dict(tau=0.0), dict(tau=-1.0), dict(tau=1e-39), dict(tau=NAN), dict(tau=INF), dict(ids=None), dict(values=None),
                dict(logits=None), dict(ldl=5), dict(T=-3)):
        assert topk(**bad) == 1, bad


def distill(logits=fake, ldl=100, dtype=0, ids=fake, values=fake, ldk=8, K=8, lse=None, M=1, row0=0, T=4, V=100, tau=1.0, flags=0,
            scale=1.0, loss=fake, kl=fake, dl=C.c_void_p(4096), ldd=100, ws=fake, ws_bytes=1 << 16):
    return binding.load().pods_distill_chunk(logits, ldl, dtype, ids, values, ldk, K, lse, fake, fake, M, row0, None, T, V, tau, flags,
                                             scale, loss, kl, dl, ldd, ws, ws_bytes, None, None)


def test_distill_refusals():
    assert distill(T=0) == 0
    assert distill(dtype=3) == 2 and distill(V=524289, ldl=524289, ldd=524289) == 2 and distill(K=1025, ldk=1025) == 2
    assert distill(flags=2) == 2
    for bad in (dict(K=0), dict(ldk=7), dict(M=0), dict(row0=-1), dict(T=-1), dict(V=0), dict(ldl=99), dict(ldd=99), dict(tau=0.0),
                dict(tau=1e-39), dict(tau=NAN), dict(scale=NAN), dict(flags=1), dict(logits=None), dict(ids=None), dict(values=None), dict(loss=None),
                dict(kl=None), dict(dl=C.c_void_p(4097)), dict(dl=fake, ldd=104), dict(loss=C.c_void_p(260))):
        assert distill(**bad) == 1, bad
    need = binding.pods_distill_chunk_workspace_bytes(4)
    assert need >= 32 and binding.pods_distill_chunk_workspace_bytes(-1) == 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=C.c_void_p(264))):
        assert distill(**bad) == 3, bad


def test_the_binding_checks_shapes_types_and_devices():
    T, V = 6, 50
    z = torch.zeros((T, V))
    u = torch.zeros(T)
    for bad in (dict(u=torch.zeros(T - 1)), dict(mask=torch.ones(T + 1, dtype=torch.uint8)), dict(tokens=torch.zeros(3, dtype=torch.int32)),
                dict(logp=torch.zeros(T - 1)), dict(logq=torch.zeros(1)), dict(temperature=torch.ones(T - 1)),
                dict(top_k=torch.ones(2, dtype=torch.int32)), dict(top_p=torch.ones(T + 1)), dict(min_p=torch.ones(1))):
        with pytest.raises(binding.PodsError, match="must hold"):
            binding.pods_sample(**{"logits": z, "u": u, **bad})
    for wrong in (torch.zeros(T), torch.zeros((T, V, 1)), torch.zeros((T, 0))):
        with pytest.raises(binding.PodsError, match=r"\[T,V\]|column"):
            binding.pods_sample(wrong, u)
    with pytest.raises(binding.PodsError, match="bfloat16, float16 or float32"):
        binding.pods_sample(z.double(), u)
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_sample(z, u)
    with pytest.raises(binding.PodsError, match="at most"):
        binding.pods_sample(torch.zeros((1, 1)).expand(1, 524289), torch.zeros(1))
    for K in (0, V + 1, 2000):
        with pytest.raises(binding.PodsError, match="1 <= K"):
            binding.pods_topk(z, K)
    for bad in (dict(ids=torch.zeros((T, 4), dtype=torch.int32)), dict(values=torch.zeros((T - 1, 5)))):
        with pytest.raises(binding.PodsError, match="must have the shape"):
            binding.pods_topk(z, 5, **bad)
    with pytest.raises(binding.PodsError, match="must hold"):
        binding.pods_topk(z, 5, lse=torch.zeros(T + 1))

    def args(**over):
        a = dict(logits=z, ids=torch.zeros((T, 4), dtype=torch.int32), values=torch.zeros((T, 4)), teacher_lse=torch.zeros(T),
                 seq_weight=torch.zeros(2, dtype=torch.float64), cu_seqlens=torch.zeros(3, dtype=torch.int64), row0=0,
                 mask=torch.ones(T, dtype=torch.uint8), loss_acc=torch.zeros(1, dtype=torch.float64))
        a.update(over)
        return a

    for bad in (dict(ids=torch.zeros((T - 1, 4), dtype=torch.int32)), dict(values=torch.zeros((T, 5))), dict(teacher_lse=torch.zeros(T - 1)),
                dict(seq_weight=torch.zeros(3, dtype=torch.float64)), dict(mask=torch.ones(1, dtype=torch.uint8)), dict(kl=torch.zeros(T + 2)),
                dict(loss_acc=torch.zeros(2, dtype=torch.float64)), dict(dlogits=torch.zeros((T, V - 1))),
                dict(dlogits=torch.zeros((T, V), dtype=torch.bfloat16)), dict(ids=torch.zeros((T, 0), dtype=torch.int32)),
                dict(teacher_lse=None, rest=True)):
        with pytest.raises(binding.PodsError, match="must hold|must have|must be|1 <= K|needs"):
            binding.pods_distill_chunk(**args(**bad))
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_distill_chunk(**args())


def test_misaligned_pointers_are_refused():
    """Every array, off its element's boundary by half an element or a byte: refused on the host, nothing is launched."""
    lib = binding.load()
    off = {1: None, 4: [C.c_void_p(256 + d) for d in (1, 2, 3)], 8: [C.c_void_p(256 + d) for d in (1, 4)]}

    def refused(call, good, arrays):
        for at, size in arrays.items():
            for bad in off[size]:
                args = list(good)
                args[at] = bad
                assert call(*args) == 1, (at, bad)

    #            logits ldl dt T  V    u     tau_row tau  k_row k  p_row p    m_row m    mask  tokens logp logq status stream
    refused(lib.pods_sample, (fake, 100, 2, 4, 100, fake, fake, 1.0, fake, 0, fake, 1.0, fake, 0.0, None, fake, fake, fake, fake, None),
            {0: 4, 5: 4, 6: 4, 8: 4, 10: 4, 12: 4, 15: 4, 16: 4, 17: 4, 18: 4})
    #          logits ldl dt T  V    K  tau  mask  ids   values lse status stream
    refused(lib.pods_topk, (fake, 100, 2, 4, 100, 5, 1.0, None, fake, fake, fake, fake, None), {0: 4, 8: 4, 9: 4, 10: 4, 11: 4})
    #                   logits ldl dt ids  values ldk K lse  weight  cu   M  row0 mask T  V   tau flags scale loss kl  dlogits ldd ws bytes status stream
    refused(lib.pods_distill_chunk, (fake, 100, 2, fake, fake, 8, 8, fake, fake, fake, 1, 0, None, 4, 100, 1.0, 0, 1.0, fake, fake, C.c_void_p(4096), 100,
                                     fake, 1 << 16, fake, None), {0: 4, 3: 4, 4: 4, 7: 4, 8: 8, 9: 8, 18: 8, 19: 4, 20: 4, 24: 4})
