"""Bounds of bfloat16 attention on long axes, where those of grad_ref (which add every rounding's magnitude) would let a
whole split or block of keys go missing.

The probabilities, and the score gradients, are rounded to bfloat16 one by one as operands of the products over keys or
queries: independent errors of at most U relative each (half a step), so that their sum over an axis is off by 8 U sqrt(sum
of the squared terms): above 13 standard deviations, for a rounding's is at most U / sqrt(3).  The result's own rounding
adds U of it, and what is held in float32 the terms of grad_ref.  D is taken from the stored output, as its definition says,
and carries no rounding of that."""
import math

import torch

import grad_ref as R


def operands(seed, B, h, hk, n_q, n_kv, d, device):
    """Q, K, V, dO in bfloat16, token-major in memory."""
    g = torch.Generator(device=device).manual_seed(seed)
    one = lambda heads, n: torch.randn(B, n, heads, d, generator=g, device=device).to(torch.bfloat16).transpose(1, 2)  # noqa: E731
    return one(h, n_q), one(hk, n_kv), one(hk, n_kv), one(h, n_q)


def attention(Q, K, V, lens=None, causal=False, dO=None, out=None, without=None):
    """{"out", "lse"}, or with dO and out {"dQ", "dK", "dV"}: (value, bound).  without: (keys or None, queries or None),
    slices whose terms are left out of the sums over them (the planted mistake of a lost block)."""
    B, h, n_q, d = Q.shape
    hk, n_kv = K.shape[1], K.shape[2]
    u, dev = R.U[torch.bfloat16], Q.device
    c = R.f32_steps(d + n_kv + n_q * (h // hk))
    scale = 1.0 / math.sqrt(d)
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)  # noqa: E731
    names = ("out",) if dO is None else ("dQ", "dK", "dV")
    val = {k: z(*(K if k in ("dK", "dV") else Q).shape) for k in names}
    square, flat = ({k: torch.zeros_like(t) for k, t in val.items()} for _ in range(2))   # of the terms' squares; of what is float32's
    lse_all, lse_bound = torch.full((B, h, n_q), -math.inf, dtype=torch.float64, device=dev), z(B, h, n_q)
    keys, queries = without or (None, None)

    def lost(x):   # [n_q, n] without what the planted mistake leaves out
        x = x.clone()
        if keys is not None:
            x[:, keys] = 0.0
        if queries is not None:
            x[queries] = 0.0
        return x

    for b in range(B):
        n = n_kv if lens is None else lens[b]
        m = R.seen_mask(n_q, n, n, causal, dev)
        for i in range(h):
            j = i * hk // h
            q, k, v = Q[b, i].double(), K[b, j, :n].double(), V[b, j, :n].double()
            s = (q @ k.T.contiguous()) * scale
            cp = c + 4.0 * float(s.abs().max()) * 2.0 ** -24 + 4.0 * 2.0 ** -24 * float((q.norm(dim=1).max() * k.norm(dim=1).max()) * scale)
            s = s.masked_fill(~m, -math.inf)
            lse = torch.logsumexp(s, -1)
            some = lse > -math.inf
            p = torch.where(m, torch.exp(s - torch.where(some, lse, 0.0).unsqueeze(-1)), 0.0)
            lse_all[b, i], lse_bound[b, i] = lse, cp + 2.0 ** -24 * torch.where(some, lse.abs(), 0.0)
            if dO is None:
                val["out"][b, i] = lost(p) @ v
                square["out"][b, i] = p.square() @ v.square()
                flat["out"][b, i] = 2 * cp * (p @ v.abs())
                continue
            g = dO[b, i].double()
            D = (g * out[b, i].double()).sum(-1, keepdim=True)
            Dmag = (g * out[b, i].double()).abs().sum(-1, keepdim=True)
            ds = p * (g @ v.T.contiguous() - D)
            e = p * 2 * cp * (g.abs() @ v.abs().T.contiguous() + Dmag) + c * ds.abs()
            L, LP = lost(ds), lost(p)
            val["dQ"][b, i] = scale * (L @ k)
            square["dQ"][b, i] = scale ** 2 * (ds.square() @ k.square())
            flat["dQ"][b, i] = scale * (e @ k.abs())
            T = lambda x: x.T.contiguous()  # noqa: E731
            val["dK"][b, j, :n] += scale * (T(L) @ q)
            square["dK"][b, j, :n] += scale ** 2 * (T(ds.square()) @ q.square())
            flat["dK"][b, j, :n] += scale * (T(e) @ q.abs())
            val["dV"][b, j, :n] += T(LP) @ g
            square["dV"][b, j, :n] += T(p.square()) @ g.square()
            flat["dV"][b, j, :n] += 2 * cp * (T(p) @ g.abs())
    r = {k: (val[k], 8 * u * square[k].sqrt() + flat[k] + u * val[k].abs()) for k in names}
    if dO is None:
        r["lse"] = (lse_all, lse_bound)
    return r


def worst(got, ref):
    """Largest error in units of its bound."""
    val, bound = ref
    return float(((got.double() - val).abs() / bound.clamp_min(1e-300)).max())
