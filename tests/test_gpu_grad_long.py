"""bfloat16 attention of a training step on long axes, split and unsplit, against 64 bits with the bounds of grad_bounds,
which notice a lost split or block; and NaN and infinities in what is seen."""
import math

import pytest
import torch

import grad_bounds as G
import grad_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def check(api, seed, size, causal=False, lens=None):
    print("attention", size, "causal" if causal else "", lens, flush=True)
    Q, K, V, dO = G.operands(seed, *size, "cuda")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = api.attention_forward(Q, K, V, kv_len=kv_len, causal=causal)
    grads = api.attention_backward(dO, Q, K, V, out, lse, kv_len=kv_len, causal=causal)
    torch.cuda.synchronize()
    ref = G.attention(Q, K, V, lens, causal)
    R.within(out, ref["out"], "out")
    R.within(lse, ref["lse"], "lse")
    ref = G.attention(Q, K, V, lens, causal, dO=dO, out=out)
    for name, g in zip(("dQ", "dK", "dV"), grads):
        R.within(g, ref[name], name)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_kv", [17000, 16128, 5001, 1088])
def test_one_token(gpu_lib, n_kv, d):
    check(gpu_lib, 920, (1, 1, 1, 1, n_kv, d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size,causal,lens", [
    ((1, 8, 2, 1, 5000), False, None),             # a narrow tile of four heads' tokens
    ((2, 3, 3, 30, 4000), True, (4000, 2500)),     # narrow, causal, ragged
    ((2, 24, 24, 300, 520), False, (520, 390)),
    ((1, 2, 1, 3000, 40), False, None),            # few keys: dK, dV split over the queries
    ((1, 4, 4, 700, 700), True, None),
    ((2, 4, 2, 2047, 2047), True, (2047, 1500)),   # the key side in several splits
    ((1, 3, 3, 2500, 2600), False, None),
], ids=["shared", "rows", "heads", "queries", "causal", "causal_shared", "square"])
def test_long(gpu_lib, size, causal, lens, d):
    check(gpu_lib, 930, (*size, d), causal, lens)


@pytest.mark.parametrize("dt,d", [(BF, 128), (BF, 64), (BF, 40), (F, 32)])
@pytest.mark.parametrize("n_kv", [100, 1500])
@pytest.mark.parametrize("what", ["Q", "K", "V", "dO"])
def test_nan_in_what_is_seen(gpu_lib, what, n_kv, dt, d):
    """A NaN in one row spoils what the formulas say it enters (the others' values here are 64-bit plain sums), and a
    spoiled sample or head leaves the others' bits as they were."""
    B, h, n_q = 2, 2, 70
    t = {k: torch.randn(B, h, n, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(940 + i)).to(dt)
         for i, (k, n) in enumerate((("Q", n_q), ("K", n_kv), ("V", n_kv), ("dO", n_q)))}

    def run():
        out, lse = gpu_lib.attention_forward(t["Q"], t["K"], t["V"])
        return [x.clone() for x in (out, lse, *gpu_lib.attention_backward(t["dO"], t["Q"], t["K"], t["V"], out, lse))]

    clean = run()
    t[what][0, 1, 33, 5] = math.nan
    out, lse, dQ, dK, dV = got = run()
    torch.cuda.synchronize()
    for a, b in zip(got, clean):
        assert torch.equal(a[1], b[1]) and torch.equal(a[0, 0], b[0, 0])   # other samples and heads
    o, l, dq, dk, dv = (torch.isnan(x[0, 1]) for x in got)
    one = torch.zeros(n_q, dtype=torch.bool, device="cuda")
    one[33] = True
    if what == "Q":        # row 33 of the queries, and every key's gradients through its P
        assert torch.equal(o.all(-1), one) and torch.equal(o.any(-1), one) and torch.equal(l, one)
        assert torch.equal(dq.all(-1), one) and torch.equal(dq.any(-1), one) and bool(dk.all()) and bool(dv.all())
    elif what == "K":      # every score row has one NaN
        assert bool(o.all()) and bool(l.all()) and bool(dq.all()) and bool(dk.all()) and bool(dv.all())
    elif what == "V":      # one column of the output, and D with it
        assert bool(o[:, 5].all()) and int(o.sum()) == n_q and not bool(l.any())
        assert bool(dq.all()) and bool(dk.all()) and not bool(dv.any())
    else:                  # dO: its row of dS, and column 5 of dV
        assert not bool(o.any()) and not bool(l.any())
        assert torch.equal(dq.all(-1), one) and torch.equal(dq.any(-1), one)
        assert bool(dk.all()) and bool(dv[:, 5].all()) and int(dv.sum()) == n_kv


@pytest.mark.parametrize("H", [64, 1536, 2560, 5000, 13001])
@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
def test_nan_and_infinity_in_a_norms_row(gpu_lib, H, dt, value, layer):
    """One element of x that is not finite: its row of y and dx holds NaN where a 32-bit plain form does, every other row
    keeps its bits, and dw and dbias are spoiled in the columns where the row's terms are NaN."""
    from paper_2602_12529_amd import configs as C
    rows, kind = 37, C.NORM_LN if layer else C.NORM_RMS
    g = torch.Generator(device="cuda").manual_seed(950)
    x, dy = (torch.randn(rows, H, device="cuda", generator=g).to(dt) for _ in range(2))
    w = torch.randn(H, device="cuda", generator=g).to(dt)

    def run():
        return gpu_lib.norm_affine(x, w, norm_kind=kind), *gpu_lib.norm_affine_backward(dy, x, w, norm_kind=kind)

    clean = [t.clone() for t in run()]
    x[20, 3] = value
    y, dx, dw, db = run()
    torch.cuda.synchronize()
    rest = torch.arange(rows, device="cuda") != 20
    assert torch.equal(y[rest], clean[0][rest]) and torch.equal(dx[rest], clean[1][rest]) and torch.equal(db, clean[3])
    X = x[20].float()
    c = X - X.mean() if layer else X
    rstd = torch.rsqrt((c * c).mean() + 1e-6)
    n = torch.isnan(c * rstd)                      # RMS norm of infinity: rstd 0, NaN in its own column alone
    assert torch.equal(torch.isnan(y[20]), n) and torch.equal(torch.isnan(dw), n)
    # dx = rstd (g - mean g - xh mean(g xh)): the last mean is NaN
    assert bool(torch.isnan(dx[20]).all())
