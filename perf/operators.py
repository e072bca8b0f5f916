"""The operators of a training step, as cases that can be timed and checked.

A case is a dict of plain values.  `listed()` gives the named cases, `draw(rng)` one more of the same
ranges, `prepare(case, seed)` what a program holds before the call, `run(state)` one pass through an
operator, `work(case)` the bytes and operations the pass cannot do without, and `exact(case, seed)` the
same outputs in 64 bits.

Kinds:
  attention_forward       softmax(scale Q K^T) V with the rows' log-sum-exp: grouped heads, key lengths,
                          causal order
  attention_backward      its gradients dQ, dK, dV from the stored output and log-sum-exp
  norm_affine             layer or RMS norm with weight and bias
  norm_affine_backward    its gradients dx, dw, dbias; with "add" the residual's gradient is added to dx
  norm_modulate_backward  the gradients dx, dshift, dscale of the modulated norm

With `own` false, `run` computes the operators from elementary torch operations in 32 bits, rounded
once at the end; with `own` true it calls the library.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
# operations of the largest listed case, which no drawn one exceeds
MOST_FLOPS = 10.0 * 8 * 24 * 4352 * 4352 * 128
MOST_ELEMENTS = 8 * 4096 * 3072


# ------------------------------------------------------------------ the cases

def _attn(kind, B, heads, kv_heads, n_q, n_kv, d, dtype="bf16", causal=False, ragged=False, layout="head", name=None):
    """ragged: sample b has the first n_kv - b n_kv // (2 B) keys (a padded batch).  layout "head": operands
    [B, heads, n, d] in memory; "token": [B, n, heads, d]; "packed": slices of one projection [B, n, (q|k|v) heads, d]."""
    c = {"kind": kind, "B": B, "heads": heads, "kv_heads": kv_heads, "n_q": n_q, "n_kv": n_kv, "d": d, "dtype": dtype,
         "causal": causal, "ragged": ragged, "layout": layout}
    if name:
        c["name"] = name
    return c


def _norm(kind, samples, rows, H, dtype="bf16", layer=True, add=False, name=None):
    """rows: of a sample; affine norms have one sample.  layer: layer norm, else RMS norm."""
    c = {"kind": kind, "samples": samples, "rows": rows, "H": H, "dtype": dtype, "layer": layer, "add": add}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token of each of 16 sequences against up to 4096 kept ones, eight key heads for 32: serving, latency
        _attn("attention_forward", 16, 32, 8, 1, 4096, 128, ragged=True, layout="token", name="forward_single_tokens"),
        # joint attention of a training batch of 512-pixel images with their text: 16 samples of 1024 + 512 tokens
        _attn("attention_forward", 16, 24, 24, 1536, 1536, 128, name="forward_joint_512px"),
        # the float32 model of the tests and of smoke(): launches and latency
        _attn("attention_backward", 8, 4, 4, 24, 24, 16, dtype="f32", name="backward_tiny_f32"),
        # joint attention of a training batch of 1024-pixel images: 8 samples of 4096 + 256 tokens
        _attn("attention_backward", 8, 24, 24, 4352, 4352, 128, name="backward_joint_1024px"),
        # a video's cross-attention to its text, two prompts, one of them shorter: many queries, few keys
        _attn("attention_backward", 2, 12, 12, 32760, 512, 128, ragged=True, name="backward_cross_video"),
        # causal order, shared key heads, a packed projection and a padded batch of odd length
        _attn("attention_backward", 4, 16, 4, 2047, 2047, 64, causal=True, ragged=True, layout="packed",
              name="backward_causal_grouped_packed"),
        # the affine norm before a video block's cross-attention
        _norm("norm_affine", 1, 32760, 1536, name="norm_video"),
        # an odd width in float32: nothing is aligned
        _norm("norm_affine", 1, 4099, 1001, dtype="f32", name="norm_odd_f32"),
        # the same norm's gradients, with the residual stream's gradient
        _norm("norm_affine_backward", 1, 32760, 1536, add=True, name="norm_backward_video"),
        # the float32 model's width and row count: latency
        _norm("norm_affine_backward", 1, 192, 64, dtype="f32", name="norm_backward_tiny_f32"),
        # the modulated norm of a training batch of 1024-pixel images: 8 samples of 4096 rows
        _norm("norm_modulate_backward", 8, 4096, 3072, layer=False, name="modulate_backward_1024px"),
        # a few short samples of uneven length, layer norm
        _norm("norm_modulate_backward", 5, 333, 2560, layer=True, add=True, name="modulate_backward_short"),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["attention_forward", "attention_backward", "attention_backward", "norm_affine", "norm_affine_backward",
                       "norm_modulate_backward"])
    if kind.startswith("attention"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        d = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([16, 32, 64, 128])
        share = rng.choice([1, 1, 2, 4, 8])
        while True:
            kv_heads = rng.randint(1, 24)
            B = _spread(rng, 1, 32)
            n_kv = _spread(rng, 16, 16384)
            same = rng.random() < 0.5
            n_q = n_kv if same else 1 if kind == "attention_forward" and rng.random() < 0.3 else _spread(rng, 1, 32768)
            c = _attn(kind, B, kv_heads * share, kv_heads, n_q, n_kv, d, dtype, causal=rng.random() < 0.4 and n_q <= n_kv,
                      ragged=rng.random() < 0.5, layout=rng.choice(["head", "token", "packed" if same else "token"]))
            pairs = B * kv_heads * share * n_q * n_kv
            # the 32-bit products of the plain form and its matrices of scores bound what is drawn
            if pairs * d * 10 <= MOST_FLOPS / (4 if dtype == "bf16" else 16):
                return c
    while True:
        samples = _spread(rng, 1, 32) if kind == "norm_modulate_backward" else 1
        H = rng.choice([_spread(rng, 32, 8192), 64 * rng.randint(1, 96)])
        rows = _spread(rng, 1, 32768)
        if samples * rows * H <= MOST_ELEMENTS:
            return _norm(kind, samples, rows, H, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5,
                         kind != "norm_affine" and rng.random() < 0.5)


def _lengths(case):
    B, n = case["B"], case["n_kv"]
    return [n - b * n // (2 * B) if case["ragged"] else n for b in range(B)]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("attention"):
        B, h, hk, n_q, n_kv, d = (case[k] for k in ("B", "heads", "kv_heads", "n_q", "n_kv", "d"))
        pairs, keys = 0, 0
        for n in _lengths(case):
            keys += n
            if not case["causal"]:
                pairs += n_q * n
            else:   # row i sees i + 1 + n - n_q keys
                rows = min(n_q, n)
                pairs += rows * n - rows * (rows - 1) // 2
        q, k = B * h * n_q * d * e, keys * hk * d * e
        if case["kind"] == "attention_forward":
            return {"bytes": 2 * q + 2 * k + 4 * B * h * n_q, "flops": 4.0 * h * pairs * d}
        return {"bytes": 4 * q + 2 * k + 2 * B * n_kv * hk * d * e + 4 * B * h * n_q, "flops": 10.0 * h * pairs * d}
    R, H, S = case["samples"] * case["rows"], case["H"], case["samples"]
    x = R * H * e
    if case["kind"] == "norm_affine":
        return {"bytes": 2 * x + 2 * H * e, "flops": 7.0 * R * H}
    small = (H * e + 8 * H) if case["kind"] == "norm_affine_backward" else 12 * S * H
    return {"bytes": (4 if case["add"] else 3) * x + small, "flops": 14.0 * R * H}


# ------------------------------------------------------------------ what a program holds before the call

def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _unit_rows(x):
    """Per-head RMS norm, as the queries and keys of the blocks have."""
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _operands(case, gen, dt):
    B, h, hk, n_q, n_kv, d = (case[k] for k in ("B", "heads", "kv_heads", "n_q", "n_kv", "d"))
    if case["layout"] == "packed":
        x = _randn(gen, B, n_q, h + 2 * hk, d)
        x[:, :, :h + hk] = _unit_rows(x[:, :, :h + hk])
        x = x.to(dt).transpose(1, 2)
        return x[:, :h], x[:, h:h + hk], x[:, h + hk:]

    def one(heads, n, norm):
        x = _randn(gen, B, n, heads, d) if case["layout"] == "token" else _randn(gen, B, heads, n, d)
        x = (_unit_rows(x) if norm else x).to(dt)
        return x.transpose(1, 2) if case["layout"] == "token" else x

    return one(h, n_q, True), one(hk, n_kv, True), one(hk, n_kv, False)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = dict(case)
    if case["kind"].startswith("attention"):
        s["Q"], s["K"], s["V"] = _operands(case, gen, dt)
        s["kv_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
        if case["kind"] == "attention_backward":
            B, h, n_q, d = s["Q"].shape
            # the forward pass's output, token-major as the output projection takes it, and log-sum-exp
            out, s["lse"] = _plain_attention(s)
            s["out"] = out.transpose(1, 2).contiguous().transpose(1, 2)
            s["dO"] = _randn(gen, B, n_q, h, d).to(dt).transpose(1, 2)
        return s
    R, H, S = case["samples"] * case["rows"], case["H"], case["samples"]
    # a residual stream: channels of uneven size and offset
    s["x"] = (_randn(gen, R, H) * (1.0 + _randn(gen, H).abs()) + 0.5 * _randn(gen, H)).to(dt)
    if case["kind"] == "norm_modulate_backward":
        s["scale"] = 0.3 * _randn(gen, S, H)
    else:
        s["w"] = (1.0 + 0.1 * _randn(gen, H)).to(dt)
        s["bias"] = (0.1 * _randn(gen, H)).to(dt)
    if case["kind"] != "norm_affine":
        s["dy"] = _randn(gen, R, H).to(dt)
        s["add"] = _randn(gen, R, H).to(dt) if case["add"] else None
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _library(s)
    if s["kind"] == "attention_forward":
        return _plain_attention(s)
    if s["kind"] == "attention_backward":
        return _plain_attention_backward(s)
    if s["kind"] == "norm_affine":
        return _plain_norm(s)
    return _plain_norm_backward(s)


def _library(s):
    from paper_2602_12529_amd import api
    from paper_2602_12529_amd import configs as C
    if s["kind"] == "attention_forward":
        return api.attention_forward(s["Q"], s["K"], s["V"], kv_len=s["kv_len"], causal=s["causal"])
    if s["kind"] == "attention_backward":
        return api.attention_backward(s["dO"], s["Q"], s["K"], s["V"], s["out"], s["lse"], kv_len=s["kv_len"],
                                      causal=s["causal"])
    kind = C.NORM_LN if s["layer"] else C.NORM_RMS
    if s["kind"] == "norm_affine":
        return api.norm_affine(s["x"], s["w"], s["bias"], norm_kind=kind, eps=EPS)
    if s["kind"] == "norm_affine_backward":
        return api.norm_affine_backward(s["dy"], s["x"], s["w"], norm_kind=kind, eps=EPS, add=s["add"])
    return api.norm_modulate_backward(s["dy"], s["x"], scale=s["scale"], mod_ld=s["H"], rows_per_sample=s["rows"],
                                      norm_kind=kind, eps=EPS, add=s["add"])


# ------------------------------------------------------------------ plain forms

def _heads(x, heads):
    """float32 [B, heads, n, d] of a tensor with fewer, shared heads."""
    return x.float().repeat_interleave(heads // x.shape[1], 1).contiguous()


def _seen(s):
    """[B, 1, n_q, n_kv]: whether the row may see the key; None where every one may."""
    if s["kv_len"] is None and not s["causal"]:
        return None
    key = torch.arange(s["n_kv"], device=DEV)
    n = s["kv_len"].view(-1, 1, 1, 1) if s["kv_len"] is not None else torch.full((s["B"], 1, 1, 1), s["n_kv"], device=DEV)
    if not s["causal"]:
        return (key < n).expand(-1, 1, s["n_q"], -1)
    row = torch.arange(s["n_q"], device=DEV).view(-1, 1)
    return (key < n) & (key <= row + (n - s["n_q"]))


def _scores(s, q, k):
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(s["d"]))
    seen = _seen(s)
    return x if seen is None else x.masked_fill_(~seen, -math.inf)


def _plain_attention(s):
    q, k, v = s["Q"].float().contiguous(), _heads(s["K"], s["heads"]), _heads(s["V"], s["heads"])
    x = _scores(s, q, k)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out.to(s["Q"].dtype), (top + total.log()).squeeze(-1)


def _plain_attention_backward(s):
    q, k, v = s["Q"].float().contiguous(), _heads(s["K"], s["heads"]), _heads(s["V"], s["heads"])
    do, out = s["dO"].float().contiguous(), s["out"].float()
    lse = s["lse"].unsqueeze(-1)
    # a row that sees no key has exp(-inf - 0) = 0 everywhere
    p = _scores(s, q, k).sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_()
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
    ds.mul_(1.0 / math.sqrt(s["d"]))
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    shape = (s["B"], s["kv_heads"], s["heads"] // s["kv_heads"], s["n_kv"], s["d"])
    dt = s["Q"].dtype
    return dq.to(dt), dk.view(shape).sum(2).to(dt), dv.view(shape).sum(2).to(dt)


def _normed(s):
    x = s["x"].float()
    if s["layer"]:
        x = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * rstd, rstd


def _plain_norm(s):
    return (_normed(s)[0] * s["w"].float() + s["bias"].float()).to(s["x"].dtype)


def _plain_norm_backward(s):
    xh, rstd = _normed(s)
    dy = s["dy"].float()
    if s["kind"] == "norm_affine_backward":
        g = dy * s["w"].float()
    else:
        g = (dy.view(s["samples"], s["rows"], -1) * (1.0 + s["scale"]).unsqueeze(1)).view_as(dy)
    c = g - xh * (g * xh).mean(-1, keepdim=True)
    if s["layer"]:
        c = c - g.mean(-1, keepdim=True)
    dx = c * rstd
    if s["add"] is not None:
        dx = dx + s["add"].float()
    dx = dx.to(s["x"].dtype)
    if s["kind"] == "norm_affine_backward":
        return dx, (dy * xh).sum(0), dy.sum(0)
    rows = (s["samples"], s["rows"], -1)
    return dx, dy.view(rows).sum(1), (dy * xh).view(rows).sum(1)


# ------------------------------------------------------------------ in 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("attention"):
        return _exact_attention(s)
    x = s["x"].double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    if case["layer"]:
        n = (x - mean) / (var + EPS).sqrt()
        r = 1.0 / (var + EPS).sqrt()
    else:
        r = 1.0 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        n = x * r
    if case["kind"] == "norm_affine":
        return n * s["w"].double() + s["bias"].double()
    dy = s["dy"].double().view(case["samples"], case["rows"], -1)
    n = n.view_as(dy)
    m = s["w"].double() if case["kind"] == "norm_affine_backward" else 1.0 + s["scale"].double().unsqueeze(1)
    g = dy * m
    dx = g - n * (g * n).mean(-1, keepdim=True)
    if case["layer"]:
        dx = dx - g.mean(-1, keepdim=True)
    dx = (dx * r.view(case["samples"], case["rows"], 1)).view_as(x)
    if s["add"] is not None:
        dx = dx + s["add"].double()
    dm, da = (dy * n).sum(1), dy.sum(1)
    return (dx, dm[0], da[0]) if case["kind"] == "norm_affine_backward" else (dx, da, dm)


def _exact_attention(s):
    """Sample by sample and head group by head group, over the keys that the sample has."""
    B, h, n_q, d = s["Q"].shape
    hk, g = s["kv_heads"], s["heads"] // s["kv_heads"]
    back = s["kind"] == "attention_backward"
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, lse = f64(B, h, n_q, d), f64(B, h, n_q)
    dq, dk, dv = f64(B, h, n_q, d), f64(B, hk, s["n_kv"], d), f64(B, hk, s["n_kv"], d)
    for b, n in enumerate(_lengths(s)):
        hidden = None
        if s["causal"]:
            hidden = torch.ones(n_q, n, dtype=torch.bool, device=DEV).triu(n - n_q + 1)
        for i in range(hk):
            q, k, v = s["Q"][b, i * g:(i + 1) * g].double(), s["K"][b, i, :n].double(), s["V"][b, i, :n].double()
            z = (q.reshape(g * n_q, d) @ k.T.contiguous()).view(g, n_q, n) / math.sqrt(d)
            if hidden is not None:
                z.masked_fill_(hidden, -math.inf)
            l = torch.logsumexp(z, -1)
            p = torch.nan_to_num(torch.exp(z - l.unsqueeze(-1)), nan=0.0)
            del z
            if not back:
                out[b, i * g:(i + 1) * g] = (p.view(g * n_q, n) @ v).view(g, n_q, d)
                lse[b, i * g:(i + 1) * g] = l
                continue
            do = s["dO"][b, i * g:(i + 1) * g].double().reshape(g * n_q, d)
            p = p.view(g * n_q, n)
            dp = do @ v.T.contiguous()
            dv[b, i, :n] = p.T.contiguous() @ do
            dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p).div_(math.sqrt(d))
            dq[b, i * g:(i + 1) * g] = (dp @ k).view(g, n_q, d)
            dk[b, i, :n] = dp.T.contiguous() @ q.reshape(g * n_q, d)
    return (dq, dk, dv) if back else (out, lse)
