"""Token log-probabilities in fp64 by elementary operations, for batches of more rows than the numpy oracle takes in a test's time, and
the comparison with pods_logp_chunk.  Not collected by pytest.

Tolerances: those derived in test_gpu_logp.py, the same for each row of a batch.  Each of its terms is one row's, and a thread of the
kernels for many rows adds at most 64 blocks' sums of a row (131072 vectors over 512 threads of four vectors a block)."""
import torch

REL = 2.0 ** -19


def rows64(z, tok, tau):
    """z [T,V], tok [T] -> (logp, lse, entropy, spread) fp64 [T]; spread: the largest distance from the row's maximum, over tau."""
    T, V = z.shape
    out = [torch.empty(T, dtype=torch.float64, device=z.device) for _ in range(4)]
    step = max(1, (1 << 24) // V)
    for a in range(0, T, step):
        x = z[a:a + step].double()
        top = x.amax(1, keepdim=True)                  # NaN where one of the row is
        d = (x - top) / tau
        e = d.exp()
        e[e < 1e-300] = 0.0
        s = e.sum(1).log()
        at = d.gather(1, tok[a:a + step, None].long())[:, 0]
        u = torch.where(e > 0, e * d, torch.zeros_like(d)).sum(1) / e.sum(1)
        lse, bad = top[:, 0] / tau + s, ~(top[:, 0].abs() < torch.inf)
        nan = torch.full_like(s, torch.nan)
        out[0][a:a + step] = torch.where(bad, nan, at - s)
        out[1][a:a + step] = torch.where(bad, torch.where(top[:, 0] == -torch.inf, top[:, 0], nan), lse)
        out[2][a:a + step] = torch.where(bad, nan, s - u)
        out[3][a:a + step] = torch.where(torch.isfinite(x), d.abs(), torch.zeros_like(d)).amax(1).nan_to_num(0.0)
    return out


def compare(got, want, rows=None):
    """got: pods_logp_chunk's (logp, lse or None, entropy or None); rows: which of them (bool), all where None."""
    lp, ls, H, spread = want
    tol = REL + 2.0 ** -23 * spread.clamp(max=100.0)
    bounds = (tol + 2.0 ** -23 * lp.abs(), tol + 2.0 ** -24 * ls.abs(), 4 * tol * H.clamp(min=1.0) + 2.0 ** -23 * H)
    for name, x, w, bound in zip(("logp", "lse", "entropy"), got, (lp, ls, H), bounds):
        if x is None:
            continue
        x = x.double()
        fine = (x == w) | (x.isnan() & w.isnan()) | ((x - w).abs() <= bound)
        if rows is not None:
            fine |= ~rows
        bad = (~fine).nonzero()[:, 0]
        assert bad.numel() == 0, (name, bad.numel(), bad[:6].tolist(), x[bad[:6]].tolist(), w[bad[:6]].tolist())
