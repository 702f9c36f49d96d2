"""Sampling from logits, the top of a row of logits, and distillation from such tops: cases, plain forms, exact values.

Plain forms hold the V-wide work of the objective in fp32; the sampler's running sums, whose borders decide which token
is drawn, and the K-wide or one-per-row terms are held in fp64."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ESIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
GREEDY_BELOW = 2.0 ** -20        # temperatures below this are the arg-max


def listed():
    return [
        # one sequence being decoded at the usual serving settings: latency
        dict(name="sample_1_topk_topp", op="sample", T=1, V=151936, dtype="bf16", logits="peaked", temperature=0.7, top_k=50, top_p=0.95, min_p=0.0, per_row=False, pad=0),
        # one prompt's 64 rollouts in flight, fp32 logits, every request with its own settings (greedy ones among them)
        dict(name="sample_64_per_request", op="sample", T=64, V=151936, dtype="fp32", logits="peaked", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=True, pad=0),
        # a step of the rollouts of 8 prompts, drawn from the whole policy as on-policy training asks
        dict(name="sample_512_policy", op="sample", T=512, V=151936, dtype="bf16", logits="spiked", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=False, pad=0),
        # the same step with a nucleus, on rows whose nucleus has thousands of tokens
        dict(name="sample_512_wide_nucleus", op="sample", T=512, V=151936, dtype="bf16", logits="spiked", temperature=1.0, top_k=0, top_p=0.9, min_p=0.0, per_row=False, pad=0),
        # a ragged vocabulary whose rows start off every 16-byte boundary, with a floor under the probabilities
        dict(name="sample_100_minp_odd", op="sample", T=100, V=50257, dtype="fp16", logits="peaked", temperature=1.2, top_k=0, top_p=1.0, min_p=0.05, per_row=False, pad=0),
        # the teacher's top 64 of a chunk of kept tokens
        dict(name="topk_1024_k64", op="topk", T=1024, V=151936, dtype="bf16", logits="spiked", K=64, temperature=1.0, pad=0),
        # a few rows, as for the alternatives reported beside each sampled token
        dict(name="topk_16_k20", op="topk", T=16, V=32000, dtype="fp32", logits="peaked", K=20, temperature=1.0, pad=0),
        # long lists of fp32 rows of an odd vocabulary
        dict(name="topk_300_k500_odd", op="topk", T=300, V=50257, dtype="fp32", logits="spiked", K=500, temperature=2.0, pad=0),
        # a chunk of kept tokens trained towards the teacher's top 64 and the mass of the rest
        dict(name="distill_4096_rest", op="distill", T=4096, V=151936, dtype="bf16", logits="spiked", K=64, temperature=1.0, rest=True, lse=True, grad=True, pad=0),
        # softened, renormalised lists and an fp32 gradient
        dict(name="distill_512_renorm_fp32", op="distill", T=512, V=151936, dtype="fp32", logits="spiked", K=128, temperature=2.0, rest=False, lse=False, grad=True, pad=0),
        # a toy vocabulary: launch latency
        dict(name="distill_37_small", op="distill", T=37, V=1024, dtype="bf16", logits="peaked", K=8, temperature=1.0, rest=True, lse=True, grad=True, pad=0),
        # evaluation: the loss alone, fp16 rows with a pitch of their own
        dict(name="distill_600_eval_odd", op="distill", T=600, V=50257, dtype="fp16", logits="peaked", K=33, temperature=1.0, rest=False, lse=True, grad=False, pad=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "topk", "distill"])
    V = rng.choice([_log_int(rng, 1000, 160000), _log_int(rng, 1000, 160000), 32000, 50257, 128256, 151936])
    c = dict(op=op, V=V, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), logits=rng.choice(["peaked", "spiked"]),
             temperature=round(rng.uniform(0.5, 1.5), 3), pad=rng.choice([0, 0, 3, 8]))
    most = {"sample": 512 * 151936, "topk": 1024 * 151936 // 2, "distill": 2048 * 151936}[op]
    c["T"] = _log_int(rng, 1, max(2, min(2000, most // V)))
    if op == "sample":
        how = rng.choice(["policy", "top_k", "top_p", "min_p", "all", "per_row"])
        c.update(top_k=_log_int(rng, 1, 1000) if how in ("top_k", "all") else 0,
                 top_p=round(rng.uniform(0.5, 0.99), 3) if how in ("top_p", "all") else 1.0,
                 min_p=round(rng.uniform(0.01, 0.2), 3) if how in ("min_p", "all") else 0.0, per_row=how == "per_row")
    elif op == "topk":
        c.update(K=_log_int(rng, 1, 1000))
    else:
        lse = rng.random() < 0.7
        c.update(K=_log_int(rng, 1, 500), lse=lse, rest=lse and rng.random() < 0.7, grad=rng.random() < 0.8)
    return c


def _logits(gen, T, V, kind):
    """fp32 [T,V].  spiked: N(0,3^2), one id raised by 8 in 30 % of the rows.  peaked: N(0,2^2) under a falling head of
    60 ids, as a trained model's rows look."""
    dev = torch.device("cuda")
    z = torch.randn((T, V), generator=gen, device=dev)
    if kind == "spiked":
        z *= 3.0
        at = torch.randint(0, V, (T, 1), generator=gen, device=dev)
        up = 8.0 * (torch.rand((T, 1), generator=gen, device=dev) < 0.3)
        z.scatter_add_(1, at, up)
    else:
        z *= 2.0
        head = min(60, V)
        part = V // head                               # one id in each of `head` stretches: no id twice
        at = torch.randint(0, V, (T, 1), generator=gen, device=dev) + part * torch.arange(head, device=dev)
        at = (at + torch.randint(0, part, (T, head), generator=gen, device=dev)) % V
        slope = 0.1 + 0.5 * torch.rand((T, 1), generator=gen, device=dev)
        top = 14.0 + 6.0 * torch.rand((T, 1), generator=gen, device=dev)
        fall = top - slope * torch.arange(head, device=dev) + torch.randn((T, head), generator=gen, device=dev)
        z.scatter_(1, at, fall)
    return z


def _stored(z, dtype, pad):
    """The rows as a user holds them: dtype, row pitch V + pad."""
    T, V = z.shape
    wide = torch.zeros((T, V + pad), dtype=DTYPES[dtype], device=z.device)
    wide[:, :V] = z
    return wide[:, :V]


def _f32(x):
    """Settings are fp32 numbers, as the entry points take them."""
    return torch.tensor(x, dtype=torch.float32).item()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    T, V = case["T"], case["V"]
    z32 = _logits(gen, T, V, case["logits"])
    s = dict(op=case["op"], logits=_stored(z32, case["dtype"], case["pad"]), T=T, V=V)
    if case["op"] == "sample":
        s["u"] = torch.rand(T, generator=gen, device=dev)
        if case["per_row"]:
            r = torch.rand((4, T), generator=gen, device=dev)
            pick = torch.rand((4, T), generator=gen, device=dev)
            s["temperature"] = torch.where(pick[0] < 0.2, torch.zeros_like(r[0]), 0.5 + 0.8 * r[0])
            s["top_k"] = torch.where(pick[1] < 0.5, torch.zeros_like(r[1]), 1 + 200 * r[1]).to(torch.int32)
            s["top_p"] = torch.where(pick[2] < 0.4, torch.ones_like(r[2]), 0.6 + 0.39 * r[2])
            s["min_p"] = torch.where(pick[3] < 0.6, torch.zeros_like(r[3]), 0.1 * r[3])
        else:
            s.update(temperature=_f32(case["temperature"]), top_k=case["top_k"], top_p=_f32(case["top_p"]), min_p=_f32(case["min_p"]))
    elif case["op"] == "topk":
        s.update(K=min(case["K"], V), temperature=_f32(case["temperature"]))
    else:
        K = min(case["K"], V)
        tau = _f32(case["temperature"])
        ids = torch.empty((T, K), dtype=torch.int32, device=dev)
        vals = torch.empty((T, K), dtype=torch.float32, device=dev)
        lse = torch.empty(T, dtype=torch.float32, device=dev)
        for a in range(0, T, 512):                     # the teacher: the student's rows with some noise
            y = z32[a:a + 512]
            y += 0.5 * torch.randn(y.shape, generator=gen, device=dev)
            v, i = y.topk(K, dim=1)
            ids[a:a + 512], vals[a:a + 512] = i.to(torch.int32), v
            lse[a:a + 512] = torch.logsumexp(y / tau, 1)
        M = max(1, min(T, 1 + T // 250))               # rollouts of about 250 tokens, one token in twenty masked out
        cuts = torch.arange(M + 1, dtype=torch.int64) * T // M
        mask = (torch.rand(T, generator=gen, device=dev) >= 0.05).to(torch.uint8)
        row = torch.repeat_interleave(torch.arange(M), cuts[1:] - cuts[:-1]).to(dev)
        n = torch.zeros(M, dtype=torch.float64, device=dev).index_add_(0, row, mask.double())
        weight = torch.where(n > 0, 1.0 / (M * n.clamp(min=1.0)), torch.zeros_like(n))
        s.update(ids=ids, values=vals, teacher_lse=lse if case["lse"] else None, mask=mask, cu_seqlens=cuts.to(dev),
                 seq_weight=weight, row_weight=weight[row] * mask, temperature=tau, rest=case["rest"], grad=case["grad"],
                 loss_acc=torch.zeros(1, dtype=torch.float64, device=dev))
    return s


def _column(x, T, dev):
    return torch.as_tensor(x, dtype=torch.float64, device=dev).expand(T)[:, None]


def _sample_plain(s):
    z = s["logits"].double()
    T, V = z.shape
    tau = _column(s["temperature"], T, z.device)
    k, p, floor = (_column(s[n], T, z.device) for n in ("top_k", "top_p", "min_p"))
    greedy = tau < GREEDY_BELOW
    tau = torch.where(greedy, torch.ones_like(tau), tau)
    d = (z - z.max(1, keepdim=True).values) / tau
    del z
    e = torch.exp(d)
    if not (isinstance(s["top_k"], int) and s["top_k"] <= 0 and s["top_p"] >= 1.0 and s["min_p"] <= 0.0):
        ds, at = torch.sort(d, dim=1, descending=True, stable=True)       # larger first, then the lower id
        es = torch.exp(ds)
        del ds
        k = torch.where((k <= 0) | (k >= V), torch.full_like(k, V), k)
        keep = torch.arange(V, device=e.device)[None] < k
        run = torch.cumsum(es * keep, 1)
        keep &= (run - es < p * run[:, -1:]) | (p >= 1.0)
        keep &= es >= floor
        keep[:, 0] = True
        del run, es
        weights = e * torch.zeros_like(keep).scatter_(1, at, keep)
        del at, keep
    else:
        weights = e
    run = torch.cumsum(weights, 1)
    total = run[:, -1:]
    target = s["u"].double()[:, None] * total
    token = (run <= target).sum(1, keepdim=True).clamp(max=V - 1)
    first = (d == 0).to(torch.int8).argmax(1, keepdim=True)
    token = torch.where(greedy, first, token)
    dt = d.gather(1, token)
    logp = dt - torch.log(e.sum(1, keepdim=True))
    logq = torch.where(greedy, torch.zeros_like(dt), dt - torch.log(total))
    return token[:, 0].to(torch.int32), logp[:, 0].float(), logq[:, 0].float()


def _topk_plain(s):
    z = s["logits"].float()
    v, i = torch.sort(z, dim=1, descending=True, stable=True)
    ids, vals = i[:, :s["K"]].to(torch.int32), v[:, :s["K"]].clone()
    del v, i
    m = z.max(1, keepdim=True).values.double()
    total = torch.exp((z - m.float()) / s["temperature"]).sum(1, dtype=torch.float64)
    return ids, vals, (m[:, 0] / s["temperature"] + torch.log(total)).float()


def _distill_plain(s):
    tau, ids = s["temperature"], s["ids"].long()
    z = s["logits"].float()
    y = s["values"].double() / tau
    L = s["teacher_lse"].double()[:, None] if s["teacher_lse"] is not None else torch.log(torch.exp(y - y.max(1, keepdim=True).values).sum(1, keepdim=True)) + y.max(1, keepdim=True).values
    lq = y - L
    q = torch.exp(lq)
    Q = q.sum(1, keepdim=True)
    r = (1.0 - Q).clamp(min=0.0) if s["rest"] else torch.zeros_like(Q)
    m = z.max(1, keepdim=True).values
    listed_d = (z.gather(1, ids).double() - m.double()) / tau
    e = torch.exp((z - m) / tau)
    del z
    outside = e.scatter(1, ids, 0.0).sum(1, keepdim=True, dtype=torch.float64)
    listed_e = torch.exp(listed_d)
    Z = outside + listed_e.sum(1, keepdim=True)
    kl = (q * (lq - (listed_d - torch.log(Z)))).sum(1, keepdim=True)
    if s["rest"]:
        kl = kl + torch.where(r > 0, r * (torch.log(r.clamp(min=1e-300)) - torch.log(outside / Z)), torch.zeros_like(r))
    w = s["row_weight"][:, None]
    live = (w != 0)
    kl = torch.where(live, kl, torch.zeros_like(kl))
    out = dict(loss=(w * kl).sum().reshape(1).float(), kl=kl[:, 0].float())
    if s["grad"]:
        g = w / tau
        e *= (g * ((Q + r) / Z - (r / outside if s["rest"] else 0.0))).float()
        e.scatter_(1, ids, (g * ((Q + r) * listed_e / Z - q)).float())
        out["dlogits"] = e.to(s["logits"].dtype)
    return out


def run(s):
    if not own:
        return {"sample": _sample_plain, "topk": _topk_plain, "distill": _distill_plain}[s["op"]](s)
    from paper_2504_13818_b200 import binding
    if s["op"] == "sample":
        return binding.pods_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                   min_p=s["min_p"], want_logq=True)
    if s["op"] == "topk":
        return binding.pods_topk(s["logits"], s["K"], temperature=s["temperature"])
    s["loss_acc"].zero_()
    kl, dlogits = binding.pods_distill_chunk(s["logits"], s["ids"], s["values"], s["teacher_lse"], s["seq_weight"],
                                             s["cu_seqlens"], 0, s["mask"], s["loss_acc"], temperature=s["temperature"],
                                             rest=s["rest"], want_grad=s["grad"])
    out = dict(loss=s["loss_acc"].float(), kl=kl)
    if s["grad"]:
        out["dlogits"] = dlogits
    return out


def work(case):
    T, V, b = case["T"], case["V"], ESIZE[case["dtype"]]
    if case["op"] == "sample":
        return dict(bytes=T * V * b + 16 * T, flops=3 * T * V)
    if case["op"] == "topk":
        return dict(bytes=T * V * b + T * (8 * min(case["K"], V) + 4), flops=3 * T * V)
    passes = 2 if case["grad"] else 1
    return dict(bytes=passes * T * V * b + T * (8 * min(case["K"], V) + 8), flops=(3 + 3 * (passes - 1)) * T * V)


def _exact_sample(s):
    """One row at a time would be slow: a block of rows, each sorted by value, its kept prefix put back into id order."""
    T, V = s["T"], s["V"]
    logp, logq = [], []
    dev = s["logits"].device
    tau, k, p, floor = (torch.as_tensor(s[n], dtype=torch.float64, device=dev).expand(T) for n in ("temperature", "top_k", "top_p", "min_p"))
    for a in range(0, T, 64):
        x = s["logits"][a:a + 64].to(torch.float64)
        n = x.shape[0]
        t = tau[a:a + n].clone()
        cold = t < 2.0 ** -20
        t[cold] = 1.0
        x = x / t[:, None]
        lse = torch.logsumexp(x, 1)
        prob = torch.exp(x - lse[:, None])
        by = torch.argsort(-x, dim=1, stable=True)
        sorted_prob = prob.gather(1, by)
        count = k[a:a + n].clone()
        count[(count <= 0) | (count > V)] = V
        place = torch.arange(V, device=dev, dtype=torch.float64)[None].expand(n, V)
        inside = torch.where(place < count[:, None], sorted_prob, torch.zeros_like(sorted_prob))
        before = inside.cumsum(1) - inside
        nucleus = (before < p[a:a + n, None] * inside.sum(1, keepdim=True)) | (p[a:a + n, None] >= 1.0)
        likely = sorted_prob >= floor[a:a + n, None] * sorted_prob[:, :1]
        kept = torch.where(nucleus & likely, inside, torch.zeros_like(inside))
        in_order = torch.zeros_like(kept).scatter_(1, by, kept)
        steps = in_order.cumsum(1)
        hit = torch.searchsorted(steps, (s["u"][a:a + n].double() * steps[:, -1])[:, None], right=True)[:, 0].clamp(max=V - 1)
        hit = torch.where(cold, x.argmax(1), hit)
        lp = x.gather(1, hit[:, None])[:, 0] - lse
        logp.append(lp)
        logq.append(torch.where(cold, torch.zeros_like(lp), lp - torch.log(steps[:, -1])))
    return [None, torch.cat(logp), torch.cat(logq)]


def _exact_topk(s):
    vals, lse = [], []
    for a in range(0, s["T"], 64):
        x = s["logits"][a:a + 64].to(torch.float64)
        vals.append(torch.topk(x, s["K"], dim=1).values)
        lse.append(torch.logsumexp(x / s["temperature"], 1))
    return [None, torch.cat(vals), torch.cat(lse)]


def _exact_distill(s):
    T, V, tau = s["T"], s["V"], s["temperature"]
    kl = torch.zeros(T, dtype=torch.float64, device=s["logits"].device)
    grad = torch.zeros((T, V), dtype=torch.float64, device=kl.device) if s["grad"] else None
    for a in range(0, T, 256):
        x = s["logits"][a:a + 256].to(torch.float64) / tau
        i = s["ids"][a:a + 256].long()
        y = s["values"][a:a + 256].to(torch.float64) / tau
        norm = s["teacher_lse"][a:a + 256].to(torch.float64) if s["teacher_lse"] is not None else torch.logsumexp(y, 1)
        teacher = torch.exp(y - norm[:, None])
        logprob = x - torch.logsumexp(x, 1, keepdim=True)
        row = (teacher * ((y - norm[:, None]) - logprob.gather(1, i))).sum(1)
        slope = torch.exp(logprob)
        held = torch.zeros_like(x, dtype=torch.bool).scatter_(1, i, True)
        mass = teacher.sum(1, keepdim=True)
        if s["rest"]:
            left = torch.clamp(1.0 - mass, min=0.0)
            away = torch.logsumexp(torch.where(held, torch.full_like(logprob, -math.inf), logprob), 1, keepdim=True)
            row = row + torch.where(left > 0, left * (torch.log(left) - away), torch.zeros_like(left))[:, 0]
            pull = torch.where(held, torch.zeros_like(x), left * torch.exp(logprob - away))
            slope = slope * (mass + left) - pull
        else:
            slope = slope * mass
        slope.scatter_add_(1, i, -teacher)
        w = s["row_weight"][a:a + 256]
        kl[a:a + 256] = torch.where(w != 0, row, torch.zeros_like(row))
        if grad is not None:
            grad[a:a + 256] = slope * (w / tau)[:, None]
    out = dict(loss=(kl * s["row_weight"]).sum().reshape(1), kl=kl)
    if grad is not None:
        out["dlogits"] = grad
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "topk": _exact_topk, "distill": _exact_distill}[case["op"]](s)
