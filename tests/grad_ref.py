"""Plain 64-bit forms of the training step's operators, with bounds on what a right implementation may be off.

Bounds count roundings: U is half a step of the type relative to the value (torch.finfo(t).eps / 2).  A sum
of k products held in float32 is off by at most a random walk of k steps, taken 8 standard deviations wide,
and the scores, exponents and statistics before it by a few dozen float32 roundings: F32(k) relative to the
sum of the terms' magnitudes.  What is rounded to bfloat16 on the way (probabilities, score gradients, the
stored output) enters with U times its magnitude."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f32_steps(k):
    return (8.0 * math.sqrt(k) + 64.0) * 2.0 ** -24


def seen_mask(n_q, n_kv, length, causal, device):
    key = torch.arange(n_kv, device=device)
    m = (key < length).expand(n_q, n_kv).clone()
    if causal:
        row = torch.arange(n_q, device=device).view(-1, 1)
        m &= key <= row + length - n_q
    return m


def attention(Q, K, V, lens=None, causal=False, scale=None, dO=None, out=None):
    """{"out", "lse", and with dO "dQ", "dK", "dV"}: (value, bound) in float64, sample and head at a time.
    out: the stored output that D is taken from, whose rounding is in the bounds (float64 otherwise)."""
    B, h, n_q, d = Q.shape
    hk, n_kv = K.shape[1], K.shape[2]
    dt, dev = Q.dtype, Q.device
    u = U[dt]
    up = u if dt == torch.bfloat16 else 0.0   # float32 operands are not rounded on the way
    c = f32_steps(d + n_kv + n_q * (h // hk))
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)  # noqa: E731
    names = ["out"] + (["dQ", "dK", "dV"] if dO is not None else [])
    shapes = {"out": (B, h, n_q, d), "dQ": (B, h, n_q, d), "dK": (B, hk, n_kv, d), "dV": (B, hk, n_kv, d)}
    r = {k: [z(*shapes[k]), z(*shapes[k])] for k in names}
    r["lse"] = [torch.full((B, h, n_q), -math.inf, dtype=torch.float64, device=dev), z(B, h, n_q)]
    for b in range(B):
        n = n_kv if lens is None else min(max(int(lens[b]), 0), n_kv)
        if n == 0 or n_q == 0:
            continue
        m = seen_mask(n_q, n, n, causal, dev)
        for i in range(h):
            q, k, v = Q[b, i].double(), K[b, i * hk // h, :n].double(), V[b, i * hk // h, :n].double()
            s = (q @ k.T.contiguous()) * scale
            smag = float(abs(scale) * (q.abs() @ k.abs().T.contiguous()).max())
            cp = c + 4.0 * smag * 2.0 ** -24      # a score's own rounding becomes a relative error of P
            s = s.masked_fill(~m, -math.inf)
            lse = torch.logsumexp(s, -1)
            some = lse > -math.inf
            p = torch.where(m, torch.exp(s - torch.where(some, lse, 0.0).unsqueeze(-1)), 0.0)
            r["lse"][0][b, i] = lse
            r["lse"][1][b, i] = cp + 2.0 ** -24 * torch.where(some, lse.abs(), 0.0)
            o, omag = p @ v, p @ v.abs()
            r["out"][0][b, i], r["out"][1][b, i] = o, (up + 2 * cp) * omag + u * o.abs()
            if dO is None:
                continue
            g = dO[b, i].double()
            dp, dpmag = g @ v.T.contiguous(), g.abs() @ v.abs().T.contiguous()
            D = (g * o).sum(-1, keepdim=True)
            Dmag = (g.abs() * (o.abs() if out is None else out[b, i].double().abs())).sum(-1, keepdim=True)
            ds = p * (dp - D)
            e = up * ds.abs() + p * (up * Dmag + 2 * cp * (dpmag + Dmag))
            pT, dsT, eT = p.T.contiguous(), ds.T.contiguous(), e.T.contiguous()
            j, a = i * hk // h, abs(scale)
            r["dQ"][0][b, i], r["dQ"][1][b, i] = scale * (ds @ k), a * (e @ k.abs() + c * (ds.abs() @ k.abs()))
            r["dK"][0][b, j, :n] += scale * (dsT @ q)
            r["dK"][1][b, j, :n] += a * (eT @ q.abs() + c * (dsT.abs() @ q.abs()))
            r["dV"][0][b, j, :n] += pT @ g
            r["dV"][1][b, j, :n] += (up + 2 * cp) * (pT @ g.abs())
    for k in names[1:]:
        r[k][1] += u * r[k][0].abs()
    return r


def norm(x, m, a, layer, eps, rps, dy=None, add=None):
    """m, a: [samples, H] multipliers and offsets (float64).  {"y", and with dy "dx", "dm", "da"}: (value, bound)."""
    R, H = x.shape
    u, c = U[x.dtype], f32_steps(H)
    x = x.double()
    b = torch.arange(R, device=x.device) // rps
    mr, ar = m[b], a[b]
    mean = x.mean(-1, keepdim=True) if layer else torch.zeros(R, 1, dtype=torch.float64, device=x.device)
    var = ((x - mean) ** 2).mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = (x - mean) * rstd
    # the mean's rounding moves every difference by up to c times the row's mean magnitude
    xe = c * (xh.abs() + rstd * (x.abs().mean(-1, keepdim=True) + x.abs() * 2.0 ** -20))
    y = xh * mr + ar
    r = {"y": (y, xe * mr.abs() + u * y.abs() + c * ar.abs())}
    if dy is None:
        return r
    g0 = dy.double()
    g = g0 * mr
    c1 = g.mean(-1, keepdim=True) if layer else 0.0
    c2 = (g * xh).mean(-1, keepdim=True)
    dx = rstd * (g - c1 - xh * c2)
    e = rstd * (2 * c * (g.abs() + g.abs().mean(-1, keepdim=True) + xh.abs() * (g * xh).abs().mean(-1, keepdim=True))
                + xe * c2.abs() + xh.abs() * (g.abs() * xe).mean(-1, keepdim=True))
    if add is not None:
        dx = dx + add.double()
        e = e + 2.0 ** -24 * add.double().abs()
    S = m.shape[0]
    z = lambda: torch.zeros(S, H, dtype=torch.float64, device=x.device)  # noqa: E731
    k = f32_steps(min(R, rps))
    dm, da = z().index_add_(0, b, g0 * xh), z().index_add_(0, b, g0)
    dme = k * z().index_add_(0, b, (g0 * xh).abs()) + z().index_add_(0, b, g0.abs() * xe)
    dae = k * z().index_add_(0, b, g0.abs())
    r.update(dx=(dx, e + u * dx.abs()), dm=(dm, dme + 2.0 ** -24 * dm.abs()), da=(da, dae + 2.0 ** -24 * da.abs()))
    return r


def within(got, ref, what):
    val, bound = ref
    got = got.detach().double()
    assert got.shape == val.shape, (what, got.shape, val.shape)
    if val.numel() == 0:
        return
    inf = torch.isinf(val)
    assert torch.equal(torch.isinf(got) & (got == val), inf), (what, "infinities")
    d = torch.where(inf, 0.0, (got - torch.where(inf, 0.0, val)).abs())
    d = torch.where(inf, torch.zeros_like(d), d)
    assert bool(torch.isfinite(d).all()), (what, "not finite")
    worst = float((d / bound.clamp_min(1e-300)).max())
    print(f"PARITY {what} worst/bound={worst:.3f} maxabs={float(d.max()):.3e}", flush=True)
    assert worst <= 1.0, (what, worst)
