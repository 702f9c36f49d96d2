"""Token log-probabilities with their gradient, pair losses on packed rollouts, and the optimiser's step over many tensors:
cases, plain forms, exact values.

Plain forms hold V-wide work in fp32 and sums, row and rollout terms in fp64.  The optimiser's tensors are views of flat
buffers, each beginning at a multiple of 32 elements with zeros between them, so that its plain form is a handful of
operations on the flat buffers."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ESIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
MASKED = 0.05                    # share of the tokens that a mask leaves out


def listed():
    return [
        # one short answer of a toy vocabulary: latency
        dict(name="logp_37_small", op="logp", T=37, V=1024, dtype="bf16", temperature=1.0, entropy=False, pad=0),
        # a chunk of kept tokens under the reference policy, whose logits are at hand
        dict(name="logp_2048_reference", op="logp", T=2048, V=151936, dtype="bf16", temperature=1.0, entropy=False, pad=0),
        # log-probability and entropy of sampled tokens, a ragged vocabulary whose rows have a pitch of their own
        dict(name="logp_700_entropy_odd", op="logp", T=700, V=50257, dtype="fp16", temperature=0.8, entropy=True, pad=7),
        # the gradient of a user's objective on token log-probabilities with an entropy bonus
        dict(name="logp_grad_2048_entropy", op="logp_grad", T=2048, V=151936, dtype="bf16", temperature=1.0, entropy=True, pad=0),
        # the same without the bonus, fp32 rows of an odd length
        dict(name="logp_grad_400_fp32_odd", op="logp_grad", T=400, V=50257, dtype="fp32", temperature=1.0, entropy=False, pad=0),
        # two pairs of short answers, a toy vocabulary: latency
        dict(name="pair_2_small", op="pair", T=61, V=1024, dtype="bf16", M=4, shared=0, loss="sigmoid", smoothing=0.0, average=False, nll=0.0, reference=True),
        # eight pairs, chosen beside rejected, of some 250 tokens each
        dict(name="pair_8_sigmoid", op="pair", T=4096, V=151936, dtype="bf16", M=16, shared=0, loss="sigmoid", smoothing=0.1, average=False, nll=0.0, reference=True),
        # the kept rollouts of four prompts, every better one against every worse one, length-averaged, with the chosen's likelihood
        dict(name="pair_64_shared", op="pair", T=6007, V=32000, dtype="fp16", M=32, shared=8, loss="squared", smoothing=0.0, average=True, nll=0.2, reference=True),
        # the output projection alone: bf16 weights, the fp32 gradient that its fused objective accumulates, 8-bit states
        dict(name="adamw_head_8bit", op="adamw", shapes="head", vocab=151936, d=2048, param="bf16", grad="fp32", bits=8, copy="", clip=True),
        # a whole small model with fp32 weights, their bf16 copy and fp32 states
        dict(name="adamw_model_fp32", op="adamw", shapes="layers", layers=24, vocab=32000, d=1024, kv=256, ff=2816, param="fp32", grad="bf16", bits=32, copy="bf16", clip=True),
        # low-rank adapters: hundreds of small tensors
        dict(name="adamw_adapters", op="adamw", shapes="adapters", layers=28, rank=8, d=2048, kv=256, ff=11008, param="fp32", grad="fp32", bits=32, copy="", clip=True),
        # a handful of tensors of odd sizes, down to one element
        dict(name="adamw_odd_8bit", op="adamw", shapes="odd", seed=1, count=12, most=70000, param="bf16", grad="fp16", bits=8, copy="", clip=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "logp_grad", "pair", "pair", "adamw", "adamw", "adamw"])
    if op == "adamw":
        c = dict(op=op, param=rng.choice(["fp32", "bf16"]), grad=rng.choice(["fp32", "bf16", "fp16"]), bits=rng.choice([8, 32]),
                 copy="", clip=rng.random() < 0.7)
        if c["param"] == "fp32":
            c["copy"] = rng.choice(["", "bf16", "fp16"])
        c["shapes"] = rng.choice(["odd", "odd", "layers", "adapters", "head"])
        if c["shapes"] == "odd":
            c.update(seed=rng.randrange(1 << 20), count=_log_int(rng, 1, 500), most=_log_int(rng, 100, 2_000_000))
            while c["count"] * c["most"] > 300_000_000:
                c["count"] //= 2
        elif c["shapes"] == "head":
            c.update(vocab=_log_int(rng, 1000, 151936), d=8 * _log_int(rng, 16, 192))
        else:
            c.update(layers=rng.randint(1, 16), d=64 * rng.randint(2, 16), kv=64 * rng.randint(1, 4), ff=32 * rng.randint(8, 88))
            c.update(dict(vocab=_log_int(rng, 1000, 32000)) if c["shapes"] == "layers" else dict(rank=rng.choice([4, 8, 16, 64])))
        return c
    V = rng.choice([_log_int(rng, 1000, 160000), _log_int(rng, 1000, 160000), 32000, 50257, 128256, 151936])
    c = dict(op=op, V=V, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    most = 2048 * 151936 * 2 // ESIZE[c["dtype"]]
    c["T"] = _log_int(rng, 16, max(17, min(6000, most // V)))
    if op != "pair":
        c.update(temperature=round(rng.uniform(0.5, 1.5), 3), entropy=rng.random() < 0.5, pad=rng.choice([0, 0, 3, 8]))
    else:
        c["shared"] = rng.choice([0, 0, 2, 5, 8])
        c["M"] = max(2, c["shared"]) * rng.randint(1, max(1, min(16, c["T"] // 16)))
        c["M"] -= c["M"] % 2 if not c["shared"] else 0
        c.update(loss=rng.choice(["sigmoid", "hinge", "squared"]), smoothing=0.0, average=rng.random() < 0.5, nll=rng.choice([0.0, 0.2]), reference=rng.random() < 0.7)
        if c["loss"] == "sigmoid":
            c["smoothing"] = rng.choice([0.0, 0.1])
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _logits(gen, T, V):
    """fp32 [T,V] as a trained model's rows look: N(0,2^2) with a few ids well above the rest."""
    dev = torch.device("cuda")
    z = torch.randn((T, V), generator=gen, device=dev)
    z *= 2.0
    at = torch.randint(0, V, (T, 4), generator=gen, device=dev)
    up = torch.tensor([9.0, 7.5, 6.5, 6.0], device=dev) * (0.6 + 0.8 * torch.rand((T, 1), generator=gen, device=dev))
    z.scatter_add_(1, at, up)
    return z, at


def _cuts(T, M):
    """Rollouts of about T / M tokens, some longer and some shorter."""
    even = T // M
    return torch.tensor([0] + [T * i // M + (7919 * i) % max(1, even // 2) for i in range(1, M)] + [T], dtype=torch.int64)


def _pairs(M, shared):
    if not shared:
        return [(2 * p, 2 * p + 1) for p in range(M // 2)]
    best = (shared + 1) // 2     # of every `shared` rollouts of a prompt the first half are the better ones
    return [(g + a, g + b) for g in range(0, M, shared) for a in range(best) for b in range(best, shared)]


def _sizes(c):
    """(elements, takes weight decay) of every tensor."""
    if c["shapes"] == "head":
        return [(c["vocab"] * c["d"], True)]
    if c["shapes"] == "odd":
        x, got = c["seed"] * 2 + 1, []
        for _ in range(c["count"]):
            x = (x * 6364136223846793005 + 1442695040888963407) % (1 << 64)
            got.append((max(1, int(c["most"] ** ((x >> 40) / float(1 << 24)))), (x >> 39) & 1 == 1))
        return got
    d, kv, ff = c["d"], c["kv"], c["ff"]
    shapes = [(d, d), (d, kv), (d, kv), (d, d), (d, ff), (d, ff), (ff, d)]
    if c["shapes"] == "adapters":
        return [(n * c["rank"], True) for _ in range(c["layers"]) for s in shapes for n in s]
    return [(c["vocab"] * d, True)] + [s for _ in range(c["layers"]) for s in [(a * b, True) for a, b in shapes] + [(d, False), (d, False)]]


def _prepare_adamw(case, gen):
    dev = torch.device("cuda")
    sizes = _sizes(case)
    starts, N = [], 0
    for n, _ in sizes:
        starts.append(N)
        N += (n + 31) // 32 * 32
    held = torch.zeros(N, dtype=torch.bool, device=dev)
    decay = torch.zeros(N, dtype=torch.float32, device=dev)
    s = dict(op="adamw", case=case, N=N, lr=_f32(3e-4), beta1=_f32(0.9), beta2=_f32(0.95), eps=_f32(1e-8), step=1000, seed=20250413,
             max_norm=_f32(1.0) if case["clip"] else 0.0, decay=decay, stochastic=case["param"] == "bf16")
    wd = _f32(0.1)
    for a, (n, d) in zip(starts, sizes):
        held[a:a + n] = True
        if d:
            decay[a:a + n] = wd

    def normal(scale):
        x = torch.randn(N, generator=gen, device=dev)
        x *= scale
        x *= held
        return x

    s["p"] = normal(0.02).to(DTYPES[case["param"]])
    s["g"] = normal(1e-3).to(DTYPES[case["grad"]])
    if case["copy"]:
        s["copy"] = s["p"].to(DTYPES[case["copy"]])
    m, r = normal(3e-4), normal(1e-3).abs_()
    if case["bits"] == 32:
        s["m"], s["v"] = m, r * r
    else:                                              # states as earlier steps left them
        for key, x in (("m", m), ("r", r)):
            top = x.view(-1, 32).abs().amax(1)
            k = torch.where(top > 0, torch.ceil(torch.log2(top.double().clamp(min=1e-300) / 448.0)), torch.full_like(top, -126).double()).clamp(min=-126)
            code = (x.view(-1, 32).double() * torch.exp2(-k)[:, None]).clamp(-448, 448).float().to(torch.float8_e4m3fn)
            s[key] = code.view(torch.uint8).reshape(-1)
            s[key + "_scale"] = (k + 127).to(torch.uint8)
    if own:
        from paper_2504_13818_b200 import binding

        def views(flat, per=1):
            return [flat[a // per:a // per + (n + per - 1) // per] for a, (n, _) in zip(starts, sizes)]

        state = (views(s["m"]), views(s["v"])) if case["bits"] == 32 else (views(s["m"]), views(s["m_scale"], 32), views(s["r"]), views(s["r_scale"], 32))
        s["table"] = binding.pods_adamw_table(views(s["p"]), views(s["g"]), list(zip(*state)), copies=views(s["copy"]) if case["copy"] else None,
                                              weight_decay=[wd if d else 0.0 for _, d in sizes])
    return s


def _f32(x):
    """Settings are fp32 numbers, as the entry points take them."""
    return torch.tensor(x, dtype=torch.float32).item()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen)
    T, V = case["T"], case["V"]
    z, at = _logits(gen, T, V)
    pad = case.get("pad", 0)
    wide = torch.zeros((T, V + pad), dtype=DTYPES[case["dtype"]], device=dev)
    wide[:, :V] = z
    z = wide[:, :V]
    likely = torch.rand(T, generator=gen, device=dev) < 0.8
    tokens = torch.where(likely, at[:, 0], torch.randint(0, V, (T,), generator=gen, device=dev)).to(torch.int32)
    s = dict(op=case["op"], case=case, logits=z, tokens=tokens, temperature=_f32(case.get("temperature", 1.0)))
    if case["op"] == "logp":
        return s
    rows = torch.arange(0, T, 256, device=dev).tolist() + [T]
    logp, lse, entropy = (torch.empty(T, dtype=torch.float64, device=dev) for _ in range(3))
    for a, b in zip(rows[:-1], rows[1:]):              # what the forward pass left behind; a reference policy near the policy
        y = z[a:b].double() / s["temperature"]
        lse[a:b] = torch.logsumexp(y, 1)
        logp[a:b] = y.gather(1, tokens[a:b, None].long())[:, 0] - lse[a:b]
        if case["op"] == "logp_grad" and case["entropy"]:
            entropy[a:b] = lse[a:b] - (torch.exp(y - lse[a:b, None]) * y).sum(1)
    mask = torch.rand(T, generator=gen, device=dev) >= MASKED
    if case["op"] == "logp_grad":
        s.update(lse=lse, dlogp=torch.randn(T, generator=gen, device=dev) * mask / T)
        if case["entropy"]:
            s.update(entropy=entropy.float(), dentropy=torch.full((T,), -0.01 / T, device=dev) * mask)
        return s
    cuts = _cuts(T, case["M"])
    away = 0.02 * torch.randn(case["M"], generator=gen, device=dev, dtype=torch.float64)
    ref = (logp + away.repeat_interleave((cuts[1:] - cuts[:-1]).to(dev)) + 0.1 * torch.randn(T, generator=gen, device=dev, dtype=torch.float64)).float()
    s.update(ref_logp=ref if case["reference"] else None, mask=mask.to(torch.uint8), cu_seqlens=cuts.to(dev),
             pairs=torch.tensor(_pairs(case["M"], case["shared"]), dtype=torch.int32, device=dev), beta=_f32(0.1), margin=_f32(0.05),
             smoothing=_f32(case["smoothing"]), nll=_f32(case["nll"]))
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------------


def _logp_plain(z, tokens, tau, entropy):
    z = z.float()
    top = z.max(1, keepdim=True).values
    d = (z - top) / tau
    e = torch.exp(d)
    total = e.sum(1, dtype=torch.float64)
    lse = top[:, 0].double() / tau + torch.log(total)
    logp = z.gather(1, tokens.long()[:, None])[:, 0].double() / tau - lse
    H = None
    if entropy:
        e *= d
        H = torch.log(total) - e.sum(1, dtype=torch.float64) / total
    return logp, lse, H


def _grad_plain(z, tokens, tau, lse, dlogp, entropy, dentropy):
    y = z.float() / tau
    top = y.max(1, keepdim=True).values
    d = y - top
    d -= (lse[:, None] - top.double()).float()
    p = torch.exp(d)
    if dentropy is not None:
        d += entropy[:, None]
        d *= dentropy[:, None]
        d += dlogp[:, None]
        p *= -d
    else:
        p *= -dlogp[:, None]
    at = tokens.long()[:, None]
    p.scatter_add_(1, at, dlogp[:, None])
    p /= tau
    return p.to(z.dtype)


def _pair_plain(s):
    c = s["case"]
    logp, lse, _ = _logp_plain(s["logits"], s["tokens"], 1.0, False)
    live = s["mask"] != 0
    logp32 = torch.where(live, logp, torch.zeros_like(logp)).float()
    cu = s["cu_seqlens"]
    row = torch.searchsorted(cu[1:], torch.arange(c["T"], device=cu.device), right=True)
    diff = logp32.double() - (s["ref_logp"].double() if s["ref_logp"] is not None else 0.0)
    diff = torch.where(live, diff, torch.zeros_like(diff))
    zeros = torch.zeros(c["M"], dtype=torch.float64, device=cu.device)
    n = zeros.index_add(0, row, live.double())
    per = 1.0 / n.clamp(min=1.0) if c["average"] else torch.ones_like(n)
    score = zeros.index_add(0, row, diff) * per
    best, worst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    h = s["beta"] * (score[best] - score[worst]) - s["margin"]
    loss, slope = _pair_terms(h, c["loss"], s["smoothing"], s["beta"])
    likely = zeros.index_add(0, row, torch.where(live, -logp32.double(), torch.zeros_like(diff))) / n.clamp(min=1.0)
    loss = loss + s["nll"] * likely[best]
    w = 1.0 / len(best)
    coef = zeros.index_add(0, best, w * s["beta"] * slope).index_add(0, worst, -w * s["beta"] * slope) * per
    coef = coef - zeros.index_add(0, best, torch.full_like(slope, w * s["nll"])) / n.clamp(min=1.0)
    dlogp = torch.where(live, coef[row], torch.zeros_like(diff))
    dlogits = _grad_plain(s["logits"], s["tokens"], 1.0, lse, dlogp.float(), None, None)
    return dict(loss=(w * loss).sum().reshape(1).float(), logp=logp32, dlogits=dlogits, reward=(s["beta"] * score).float(), pair_loss=loss.float())


def _pair_terms(h, kind, smoothing, beta):
    """The loss of a pair and its slope in h."""
    if kind == "sigmoid":
        down, up = torch.log1p(torch.exp(-h.abs())) + torch.relu(-h), torch.log1p(torch.exp(-h.abs())) + torch.relu(h)
        return (1.0 - smoothing) * down + smoothing * up, smoothing - 1.0 / (1.0 + torch.exp(h))
    if kind == "hinge":
        return torch.relu(1.0 - h), -(h < 1.0).double()
    return ((h - 0.5) / beta) ** 2, 2.0 * (h - 0.5) / beta ** 2


def _mix(x):
    """32 bits to 32 bits, one to one, every input bit turning every output bit half of the time."""
    x = x ^ (x >> 16)
    x = (x * 0x888EC647) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x246CE511) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _word(x):
    return _mix(torch.tensor([x & 0xFFFFFFFF], dtype=torch.int64)).item()


def _random_bits(N, seed, step, dev):
    """Three numbers of 16 bits for each element of the flat buffers: those that round p, m and r."""
    key = _word(_word(_word(seed + 0x9E3779B9) ^ (seed >> 32)) ^ step)
    i = torch.arange(N, dtype=torch.int64, device=dev)
    x = i & 0xFFFFFFFF
    if N > 1 << 32:
        x ^= _mix((key + (i >> 32)) & 0xFFFFFFFF)
    else:
        x ^= _word(key)
    x = _mix(x)
    return x & 0xFFFF, x >> 16, ((x * 0x9E3779B1) & 0xFFFFFFFF) >> 16


def _to_8_bits(x, bits16, positive):
    """Blocks of 32 under the smallest power of two that keeps them within 448 -> (codes, scales), stochastically rounded."""
    top = x.view(-1, 32).abs().amax(1)
    k = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    y = (x.abs().view(-1, 32) * ((254 - k) << 23).view(torch.float32)[:, None]).view(-1)
    low = y < 2.0 ** -6
    b = torch.where(low, y + 2.0 ** -6, y).view(torch.int32)
    code = ((b + (bits16.to(torch.int32) << 4) + 8) >> 20) - 960 - 8 * low.to(torch.int32)
    if positive:
        code = torch.where(x > 0, code.clamp(min=1), code)
    else:
        code = code | ((x.view(torch.int32) >> 24) & 0x80)
    return code.to(torch.uint8), k.to(torch.uint8)


def _from_8_bits(code, scale):
    x = code.view(torch.float8_e4m3fn).float()
    return (x.view(-1, 32) * (scale.to(torch.int32) << 23).view(torch.float32)[:, None]).view(-1)


def _adamw_plain(s):
    c = s["case"]
    s["step"] += 1
    out = dict()
    g = s["g"].float()
    if s["max_norm"]:
        norm = torch.sqrt(g.double().square().sum()).float().reshape(1)
        out["norm"] = norm
        g = g * torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _from_8_bits(s["m"], s["m_scale"]), _from_8_bits(s["r"], s["r_scale"]).square()
    m = s["beta1"] * m + (1.0 - s["beta1"]) * g
    v = s["beta2"] * v + (1.0 - s["beta2"]) * (g * g)
    r = torch.sqrt(v)
    if s["stochastic"] or c["bits"] == 8:
        bits_p, bits_m, bits_r = _random_bits(s["N"], s["seed"], s["step"], g.device)
    p = s["p"].float()
    p = p * (1.0 - s["lr"] * s["decay"])
    p = p - (s["lr"] / (1.0 - s["beta1"] ** s["step"])) * (m / (r / math.sqrt(1.0 - s["beta2"] ** s["step"]) + s["eps"]))
    if s["stochastic"]:
        b = (p.view(torch.int32) + bits_p.to(torch.int32)) & -65536
        s["p"].copy_(b.view(torch.float32))
    else:
        s["p"].copy_(p)
    if c["copy"]:
        s["copy"].copy_(p)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for key, x, bits in (("m", m, bits_m), ("r", r, bits_r)):
            code, scale = _to_8_bits(x, bits, key == "r")
            s[key].copy_(code)
            s[key + "_scale"].copy_(scale)
    return out


def _adamw_outputs(s, out):
    """The updated buffers; what is held in 8 bits as the numbers it stands for: codes, and the powers of two above them."""
    out["p"] = s["p"]
    if s["case"]["copy"]:
        out["copy"] = s["copy"]
    if s["case"]["bits"] == 32:
        out.update(m=s["m"], v=s["v"])
    else:
        for key in ("m", "r"):
            out[key] = s[key].view(torch.float8_e4m3fn)
            out[key + "_scale"] = s[key + "_scale"].view(torch.float8_e8m0fnu)
    return out


def run(s):
    c = s["case"]
    if not own:
        if s["op"] == "adamw":
            return _adamw_outputs(s, _adamw_plain(s))
        if s["op"] == "pair":
            return _pair_plain(s)
        if s["op"] == "logp":
            logp, lse, H = _logp_plain(s["logits"], s["tokens"], s["temperature"], c["entropy"])
            return [logp.float()] + ([H.float()] if H is not None else [])
        return _grad_plain(s["logits"], s["tokens"], s["temperature"], s["lse"], s["dlogp"], s.get("entropy"), s.get("dentropy"))
    from paper_2504_13818_b200 import binding
    if s["op"] == "adamw":
        s["step"] += 1
        out = dict()
        if s["max_norm"]:
            out["norm"] = binding.pods_grad_norm(s["table"])
        binding.pods_adamw(s["table"], s["step"], s["lr"], beta1=s["beta1"], beta2=s["beta2"], eps=s["eps"], norm=out.get("norm"),
                           max_norm=s["max_norm"], stochastic=s["stochastic"], seed=s["seed"])
        return _adamw_outputs(s, out)
    if s["op"] == "pair":
        got = binding.pods_preference_fwd_bwd(s["logits"], s["tokens"], s["ref_logp"], s["mask"], s["cu_seqlens"], s["pairs"], s["beta"],
                                              kind=c["loss"], label_smoothing=s["smoothing"], margin=s["margin"], average=c["average"], nll=s["nll"])
        return dict(zip(("loss", "logp", "dlogits", "reward", "pair_loss"), got))
    if s["op"] == "logp":
        got = binding.pods_logp_chunk(s["logits"], s["tokens"], temperature=s["temperature"], want_entropy=c["entropy"])
        return [x for x in got if x is not None]
    return binding.pods_logp_grad_chunk(s["logits"], s["tokens"], s["lse"], s["dlogp"], entropy=s.get("entropy"), dentropy=s.get("dentropy"),
                                        temperature=s["temperature"])


def work(case):
    if case["op"] == "adamw":
        N = sum(n for n, _ in _sizes(case))
        state = 16 if case["bits"] == 32 else 4 * (1 + 1 / 32)
        return dict(bytes=N * (2 * ESIZE[case["param"]] + ESIZE[case["grad"]] + state + (ESIZE[case["copy"]] if case["copy"] else 0)), flops=(17 if case["clip"] else 14) * N)
    T, V, b = case["T"], case["V"], ESIZE[case["dtype"]]
    if case["op"] == "logp":
        return dict(bytes=T * V * b + T * (20 if case["entropy"] else 16), flops=(5 if case["entropy"] else 3) * T * V)
    if case["op"] == "logp_grad":
        return dict(bytes=(2 - MASKED) * T * V * b + T * (24 if case["entropy"] else 16), flops=(5 if case["entropy"] else 3) * T * V)
    pairs = len(_pairs(case["M"], case["shared"]))
    return dict(bytes=(2 - MASKED) * T * V * b + T * (13 if case["reference"] else 9) + 12 * pairs, flops=6 * T * V)


# ---- exact values -------------------------------------------------------------------------------------------------------


def _exact_rows(z, tokens, tau, step=256):
    """(log-probability, log-normaliser, entropy) of rows, some at a time."""
    got = []
    for a in range(0, z.shape[0], step):
        logq = torch.log_softmax(z[a:a + step].to(torch.float64) / tau, 1)
        q = torch.exp(logq)
        i = tokens[a:a + step].long()[:, None]
        own_logp = logq.gather(1, i)[:, 0]
        got.append((own_logp, z[a:a + step].gather(1, i)[:, 0].to(torch.float64) / tau - own_logp, torch.special.entr(q).sum(1)))
    return [torch.cat(x) for x in zip(*got)]


def _exact_slope(z, tokens, tau, dlogp, dentropy, step=256):
    out = torch.empty(z.shape, dtype=torch.float64, device=z.device)
    for a in range(0, z.shape[0], step):
        logq = torch.log_softmax(z[a:a + step].to(torch.float64) / tau, 1)
        q = torch.exp(logq)
        g = dlogp[a:a + step, None].double()
        slope = torch.zeros_like(q).scatter_(1, tokens[a:a + step].long()[:, None], g) - g * q
        if dentropy is not None:
            mean = (q * logq).sum(1, keepdim=True)
            slope -= dentropy[a:a + step, None].double() * q * (logq - mean)
        out[a:a + step] = slope / tau
    return out


def _exact_pair(s):
    c = s["case"]
    logp, _, _ = _exact_rows(s["logits"], s["tokens"], 1.0)
    cuts, chosen, rejected = s["cu_seqlens"].tolist(), *(s["pairs"].T.tolist())
    keep = s["mask"].bool()
    logp = torch.where(keep, logp, torch.zeros_like(logp))
    gain = logp if s["ref_logp"] is None else logp - torch.where(keep, s["ref_logp"].to(torch.float64), torch.zeros_like(logp))
    tokens = [max(1, int(keep[a:b].sum())) for a, b in zip(cuts[:-1], cuts[1:])]
    total = [float(gain[a:b].sum()) for a, b in zip(cuts[:-1], cuts[1:])]
    like = [float(logp[a:b].sum()) / n for a, b, n in zip(cuts[:-1], cuts[1:], tokens)]
    div = tokens if c["average"] else [1] * c["M"]
    coef, losses = [0.0] * c["M"], []
    for i, j in zip(chosen, rejected):
        x = s["beta"] * (total[i] / div[i] - total[j] / div[j]) - s["margin"]
        if c["loss"] == "sigmoid":
            sig = 1.0 / (1.0 + math.exp(-x)) if x > -700 else 0.0
            log_up, log_down = (-math.log1p(math.exp(-x)), -x - math.log1p(math.exp(-x))) if x >= 0 else (x - math.log1p(math.exp(x)), -math.log1p(math.exp(x)))
            e = s["smoothing"]
            loss, d = -(1.0 - e) * log_up - e * log_down, -(1.0 - e) * (1.0 - sig) + e * sig
        elif c["loss"] == "hinge":
            loss, d = max(0.0, 1.0 - x), -1.0 if x < 1.0 else 0.0
        else:
            loss, d = ((x - 0.5) / s["beta"]) ** 2, 2.0 * (x - 0.5) / s["beta"] ** 2
        losses.append(loss - s["nll"] * like[i])
        coef[i] += (d * s["beta"] / div[i] - s["nll"] / tokens[i]) / len(chosen)
        coef[j] -= d * s["beta"] / div[j] / len(chosen)
    slope = torch.cat([torch.full((b - a,), k, dtype=torch.float64) for a, b, k in zip(cuts[:-1], cuts[1:], coef)]).to(logp.device) * keep
    dev = logp.device
    losses = torch.tensor(losses, dtype=torch.float64, device=dev)
    return dict(loss=losses.mean().reshape(1), logp=logp, dlogits=_exact_slope(s["logits"], s["tokens"], 1.0, slope, None),
                reward=torch.tensor([s["beta"] * t / n for t, n in zip(total, div)], dtype=torch.float64, device=dev), pair_loss=losses)


def _exact_adamw(s):
    """fp64 throughout; numbers that are rounded with random bits are rounded from the fp64 result with the same bits."""
    c, N = s["case"], s["N"]
    t = s["step"] + 1
    g = s["g"].to(torch.float64)
    out = dict()
    if s["max_norm"]:
        length = torch.linalg.vector_norm(g)
        out["norm"] = length.reshape(1)
        if float(length) > s["max_norm"]:
            g = g * (s["max_norm"] / length)
    x = dict()
    for key in ("m", "v") if c["bits"] == 32 else ("m", "r"):
        x[key] = s[key].to(torch.float64) if c["bits"] == 32 else s[key].view(torch.float8_e4m3fn).to(torch.float64) * torch.exp2(s[key + "_scale"].to(torch.float64) - 127.0).repeat_interleave(32)
    second = x["v"] if c["bits"] == 32 else x["r"] ** 2
    first = x["m"] + (1.0 - s["beta1"]) * (g - x["m"])
    second = second + (1.0 - s["beta2"]) * (g ** 2 - second)
    root = second ** 0.5
    p = s["p"].to(torch.float64)
    p = p - s["lr"] * s["decay"].to(torch.float64) * p - s["lr"] * (first / (1.0 - s["beta1"] ** t)) / ((second / (1.0 - s["beta2"] ** t)) ** 0.5 + s["eps"])
    bits = _random_bits(N, s["seed"], t, g.device)

    def stochastic(value, places, lowest, word, nudge):
        """|value| on the grid of `places` bits behind the leading one, exponents from `lowest`: up where the rest exceeds the word."""
        size = value.abs()
        exponent = torch.floor(torch.log2(size.clamp(min=2.0 ** -400))).clamp(min=lowest)
        grid = torch.exp2(exponent - places)
        return torch.sign(value) * torch.floor(size / grid + (word.to(torch.float64) + nudge) / 65536.0) * grid

    out["p"] = stochastic(p, 7, -126, bits[0], 0.0) if s["stochastic"] else p
    if c["copy"]:
        out["copy"] = p
    if c["bits"] == 32:
        out.update(m=first, v=second)
    else:
        for key, value, word in (("m", first, bits[1]), ("r", root, bits[2])):
            top = value.view(-1, 32).abs().amax(1)
            power = torch.ceil(torch.log2((top / 448.0).clamp(min=2.0 ** -126))).clamp(min=-126.0)
            y = value / torch.exp2(power).repeat_interleave(32)
            code = stochastic(y, 3, -6, word, 0.5)
            out[key] = torch.where((value > 0) & (code == 0), torch.full_like(code, 2.0 ** -9), code) if key == "r" else code
            out[key + "_scale"] = torch.exp2(power)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "pair":
        return _exact_pair(s)
    if case["op"] == "logp":
        logp, _, H = _exact_rows(s["logits"], s["tokens"], s["temperature"])
        return [logp] + ([H] if case["entropy"] else [])
    return _exact_slope(s["logits"], s["tokens"], s["temperature"], s["dlogp"], s.get("dentropy"))
