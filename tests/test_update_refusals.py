"""Refusals of pods_logp_chunk, pods_logp_grad_chunk, pods_preference, pods_preference_fwd_bwd, pods_grad_norm and pods_adamw: the
host says no before anything is launched, so all of it runs without a GPU."""
import ctypes as C
import re

import pytest
import torch

from paper_2504_13818_b200 import binding
from paper_2504_13818_b200.csrc import build as cuda_build

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
F = C.c_void_p(4096)                                   # never read: everything comes back before a launch


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return binding.load()


def at(offset):
    return C.c_void_p(4096 + offset)


def logp(lib, logits=F, ldl=16, dtype=0, tokens=F, mask=None, T=4, V=16, temperature=1.0, logp=F, lse=F, entropy=None):
    return lib.pods_logp_chunk(logits, ldl, dtype, tokens, mask, T, V, temperature, logp, lse, entropy, None, None)


def grad(lib, logits=F, ldl=16, dtype=0, tokens=F, lse=F, dlogp=F, entropy=None, dentropy=None, T=4, V=16, temperature=1.0,
         dlogits=at(65536), ldd=16):
    return lib.pods_logp_grad_chunk(logits, ldl, dtype, tokens, lse, dlogp, entropy, dentropy, T, V, temperature, dlogits, ldd, None, None)


def pref(lib, logp=F, cu=F, M=2, T=4, pairs=F, P=1, kind=0, flags=0, beta=0.1, smoothing=0.0, margin=0.0, nll=0.0, scale=1.0,
         loss=F, dlogp=F, ws=F, ws_bytes=1 << 20):
    return lib.pods_preference(logp, None, None, cu, M, T, pairs, None, P, kind, flags, beta, smoothing, None, margin, nll, scale,
                               loss, dlogp, None, None, ws, ws_bytes, None, None)


def whole(lib, logits=F, ldl=16, dtype=0, tokens=F, T=4, V=16, temperature=1.0, M=2, P=1, loss=F, logp=F, dlogits=at(65536), ldd=16,
          ws=F, ws_bytes=1 << 20, beta=0.1):
    return lib.pods_preference_fwd_bwd(logits, ldl, dtype, tokens, None, None, F, M, T, V, temperature, F, None, P, 0, 0, beta, 0.0, None,
                                       0.0, 0.0, 1.0, loss, logp, dlogits, ldd, None, None, ws, ws_bytes, None, None)


nan, inf = float("nan"), float("inf")


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(ldl=15)), (INVALID, dict(V=0)), (INVALID, dict(T=-1)), (INVALID, dict(logits=None)), (INVALID, dict(tokens=None)),
    (INVALID, dict(temperature=0.0)), (INVALID, dict(temperature=nan)), (INVALID, dict(temperature=inf)), (INVALID, dict(temperature=-1.0)),
    (INVALID, dict(logits=at(1))), (INVALID, dict(dtype=2, logits=at(2))), (INVALID, dict(tokens=at(2))), (INVALID, dict(lse=at(4))),
    (INVALID, dict(logp=None)), (INVALID, dict(entropy=at(1))), (UNSUPPORTED, dict(dtype=3)), (UNSUPPORTED, dict(dtype=-1)),
    (UNSUPPORTED, dict(V=524289, ldl=524289)), (UNSUPPORTED, dict(T=(1 << 24) + 1)), (0, dict(T=0)), (0, dict(T=0, logits=None))])
def test_logp_refuses_on_the_host(lib, want, kw):
    assert logp(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(ldl=15)), (INVALID, dict(ldd=15)), (INVALID, dict(dlogits=None)), (INVALID, dict(dlogits=F, ldl=32, ldd=16)),
    (INVALID, dict(dentropy=F)), (INVALID, dict(lse=None)), (INVALID, dict(dlogp=None)), (INVALID, dict(lse=at(4))),
    (INVALID, dict(dlogits=at(65537))), (INVALID, dict(temperature=nan)), (UNSUPPORTED, dict(dtype=7)), (0, dict(T=0))])
def test_logp_grad_refuses_on_the_host(lib, want, kw):
    assert grad(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(M=0)), (INVALID, dict(P=-1)), (INVALID, dict(T=-1)), (INVALID, dict(beta=0.0)), (INVALID, dict(beta=-1.0)),
    (INVALID, dict(beta=nan)), (INVALID, dict(beta=inf)), (INVALID, dict(smoothing=0.5)), (INVALID, dict(smoothing=-0.1)),
    (INVALID, dict(smoothing=nan)), (INVALID, dict(kind=1, smoothing=0.1)), (INVALID, dict(nll=-1.0)), (INVALID, dict(margin=nan)),
    (INVALID, dict(scale=inf)), (INVALID, dict(pairs=None)), (INVALID, dict(cu=None)), (INVALID, dict(loss=None)),
    (INVALID, dict(loss=at(4))), (INVALID, dict(logp=None)), (INVALID, dict(pairs=at(2))), (UNSUPPORTED, dict(kind=3)),
    (UNSUPPORTED, dict(kind=-1)), (UNSUPPORTED, dict(flags=2)), (UNSUPPORTED, dict(M=1 << 31)), (WORKSPACE, dict(ws=None)),
    (WORKSPACE, dict(ws_bytes=16)), (WORKSPACE, dict(ws=at(8)))])
def test_preference_refuses_on_the_host(lib, want, kw):
    assert pref(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(ldl=15)), (INVALID, dict(ldd=15)), (INVALID, dict(loss=None)), (INVALID, dict(beta=0.0)), (INVALID, dict(M=0)),
    (INVALID, dict(dlogits=F, ldl=32)), (INVALID, dict(tokens=None)), (INVALID, dict(logp=None)), (UNSUPPORTED, dict(dtype=4)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=64)), (WORKSPACE, dict(ws=at(8)))])
def test_preference_fwd_bwd_refuses_on_the_host(lib, want, kw):
    assert whole(lib, **kw) == want


def entry(**over):
    e = binding._AdamWEntry()
    for k, v in dict(param=4096, grad=4096, m=4096, v=4096, n=10, param_type=2, grad_type=2, state_bits=32, lr_scale=1.0).items():
        setattr(e, k, v)
    for k, v in over.items():
        setattr(e, k, v)
    return e


def adamw(lib, e=None, n=1, step=1, lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, scale=1.0, norm=None, max_norm=0.0, flags=0, step_dev=None):
    table = (binding._AdamWEntry * 1)(e or entry())
    return lib.pods_adamw(table if n >= 0 else None, abs(n), step, step_dev, lr, None, beta1, beta2, eps, scale, norm, max_norm, flags, 0, None, None)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n=-1)), (INVALID, dict(step=0)), (INVALID, dict(lr=nan)), (INVALID, dict(beta1=1.0)), (INVALID, dict(beta2=-0.1)),
    (INVALID, dict(beta1=nan)), (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=inf)), (INVALID, dict(eps=1e-38)), (INVALID, dict(eps=1e38)), (INVALID, dict(scale=inf)), (INVALID, dict(max_norm=1.0)),
    (INVALID, dict(max_norm=-1.0)), (INVALID, dict(max_norm=nan, norm=F)), (INVALID, dict(norm=at(2))), (INVALID, dict(step_dev=at(4))),
    (UNSUPPORTED, dict(flags=2)), (0, dict(n=0)), (0, dict(n=0, eps=0.0)), (0, dict(n=0, eps=2.0 ** -126)), (0, dict(n=0, eps=2.0 ** 126))])
def test_adamw_refuses_settings_on_the_host(lib, want, kw):
    assert adamw(lib, **kw) == want


@pytest.mark.parametrize("want,over", [
    (INVALID, dict(n=-1)), (INVALID, dict(param=None)), (INVALID, dict(grad=None)), (INVALID, dict(m=None)), (INVALID, dict(v=None)),
    (INVALID, dict(param=4098)), (INVALID, dict(param_type=0, param=4097)), (INVALID, dict(grad=4098)), (INVALID, dict(m=4098)),
    (INVALID, dict(state_bits=8)), (INVALID, dict(weight_decay=-1.0)), (INVALID, dict(weight_decay=nan)), (INVALID, dict(lr_scale=inf)),
    (INVALID, dict(copy=4097, copy_type=0)), (UNSUPPORTED, dict(state_bits=16)), (UNSUPPORTED, dict(param_type=3)),
    (UNSUPPORTED, dict(grad_type=-1)), (UNSUPPORTED, dict(copy=4096, copy_type=9)), (UNSUPPORTED, dict(n=(1 << 42) + 1)), (0, dict(n=0, param=None))])
def test_adamw_refuses_tensors_on_the_host(lib, want, over):
    assert adamw(lib, e=entry(**over)) == want


def test_the_entry_is_the_struct_of_the_header(request):
    assert C.sizeof(binding._AdamWEntry) == 88
    text = (request.config.rootpath / "include" / "pods.h").read_text()
    body = text[:text.index("} pods_adamw_tensor;")].rsplit("typedef struct {", 1)[1]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"(\w+)[,;]", body) == [n for n, _ in binding._AdamWEntry._fields_]


def test_norm_refuses_on_the_host(lib):
    table = (binding._AdamWEntry * 1)(entry())
    need = lib.pods_grad_norm_workspace_bytes(1)
    assert need > 0 and lib.pods_grad_norm_workspace_bytes(-1) == 0
    assert lib.pods_grad_norm(table, 1, 1.0, None, F, need, None, None) == INVALID
    assert lib.pods_grad_norm(table, 1, nan, F, F, need, None, None) == INVALID
    assert lib.pods_grad_norm(table, 1, 1.0, F, F, need - 1, None, None) == WORKSPACE
    assert lib.pods_grad_norm(table, 1, 1.0, F, None, need, None, None) == WORKSPACE
    assert lib.pods_grad_norm(table, -1, 1.0, F, F, need, None, None) == INVALID


def test_binding_refuses_before_marshalling():
    bf, i32 = torch.zeros((4, 16), dtype=torch.bfloat16), torch.int32
    tok, cu, pairs = torch.zeros(4, dtype=i32), torch.tensor([0, 2, 4]), torch.zeros((1, 2), dtype=i32)
    with pytest.raises(binding.PodsError, match="must be \\[T,V\\]"):
        binding.pods_logp_chunk(bf[0], tok)
    with pytest.raises(binding.PodsError, match="at least one column"):
        binding.pods_logp_chunk(bf[:, :0], tok)
    with pytest.raises(binding.PodsError, match="tokens must hold"):
        binding.pods_logp_chunk(bf, tok[:3])
    with pytest.raises(binding.PodsError, match="bfloat16, float16 or float32"):
        binding.pods_logp_chunk(bf.double(), tok)
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_logp_chunk(bf, tok)
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_logp_grad_chunk(bf, tok, torch.zeros(4, dtype=torch.float64), torch.zeros(4))
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_preference_fwd_bwd(bf, tok, None, None, cu, pairs, 0.1)
    with pytest.raises(binding.PodsError, match="logp must be"):
        binding.pods_preference(torch.zeros((2, 2)), None, None, cu, pairs, 0.1, torch.zeros(1, dtype=torch.float64))
    p = [torch.zeros(8)]
    for bad in (dict(grads=[]), dict(states=[]), dict(copies=[]), dict(weight_decay=[0.0, 1.0]), dict(lr_scale=[])):
        with pytest.raises(binding.PodsError, match="one entry a parameter"):
            binding.pods_adamw_table(**{**dict(params=p, grads=p, states=[binding.new_adamw_state(p[0])]), **bad})
    with pytest.raises(binding.PodsError, match="CUDA"):
        binding.pods_adamw_table(p, p, [binding.new_adamw_state(p[0])])
    with pytest.raises(binding.PodsError, match="8 or 32"):
        binding.new_adamw_state(p[0], bits=4)
    assert [t.numel() for t in binding.new_adamw_state(torch.zeros(33), bits=8)] == [33, 2, 33, 2]
