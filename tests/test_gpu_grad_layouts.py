"""Attention of a training step with outputs and inputs in orders other than head-major, token-major and packed."""
import math

import pytest
import torch

import grad_ref as R

pytestmark = pytest.mark.gpu

# where (B, heads, n) lie in memory, outermost first; the head dimension is innermost
ORDERS = {"samples_innermost": (2, 1, 0), "heads_outermost": (1, 0, 2), "tokens_outermost": (2, 0, 1)}


def ordered(shape, order, dt, pad, fill=None):
    """[B, heads, n, d] whose axes lie in memory in `order`, each row with `pad` elements behind it."""
    dims = [shape[i] for i in order]
    t = torch.empty(*dims, shape[3] + pad, dtype=dt, device="cuda")
    t.fill_(3.0) if fill is None else t.normal_(generator=torch.Generator(device="cuda").manual_seed(fill))
    back = [order.index(i) for i in range(3)]
    return t, t.permute(*back, 3)[..., :shape[3]]


@pytest.mark.parametrize("dt,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.bfloat16, 24), (torch.float32, 36)])
@pytest.mark.parametrize("order", list(ORDERS))
@pytest.mark.parametrize("B,h,hk,n_q,n_kv,causal", [(3, 4, 2, 70, 90, True), (2, 6, 2, 1, 1200, False), (2, 2, 2, 1500, 33, False)],
                         ids=["square", "token", "queries"])
def test_any_order(gpu_lib, B, h, hk, n_q, n_kv, causal, order, dt, d):
    """Given outputs of any order are written at their elements and nowhere else, split or not, with a given lse."""
    pad, o = 8, ORDERS[order]
    Q, K, V, dO = (ordered(s, o, dt, pad, 980 + i)[1] for i, s in enumerate(((B, h, n_q, d), (B, hk, n_kv, d), (B, hk, n_kv, d), (B, h, n_q, d))))
    outs = [ordered(s, o, dt, pad) for s in ((B, h, n_q, d), (B, h, n_q, d), (B, hk, n_kv, d), (B, hk, n_kv, d))]
    lse = torch.full((B, h, n_q), math.nan, device="cuda")
    lens = [n_kv - 5 * b for b in range(B)]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, got = gpu_lib.attention_forward(Q, K, V, kv_len=kv_len, causal=causal, scale=0.2, out=outs[0][1], lse=lse)
    assert out is outs[0][1] and got is lse
    gpu_lib.attention_backward(dO, Q, K, V, out, lse, kv_len=kv_len, causal=causal, scale=0.2, dQ=outs[1][1], dK=outs[2][1], dV=outs[3][1])
    torch.cuda.synchronize()
    ref = R.attention(Q, K, V, lens, causal, 0.2, dO=dO, out=out)
    for name, t in (("out", out), ("lse", lse), ("dQ", outs[1][1]), ("dK", outs[2][1]), ("dV", outs[3][1])):
        R.within(t, ref[name], name)
    for whole, _ in outs:
        assert bool((whole[..., d:] == 3.0).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H", [40, 1536, 2560, 13001])
def test_norm_with_bias_alone(gpu_lib, H, dt):
    from paper_2602_12529_amd import configs as C
    g = torch.Generator(device="cuda").manual_seed(990)
    x, bias = torch.randn(50, H, device="cuda", generator=g).to(dt), torch.randn(H, device="cuda", generator=g).to(dt)
    one = torch.ones(1, H, dtype=torch.float64, device="cuda")
    for kind in (C.NORM_LN, C.NORM_RMS):
        y = gpu_lib.norm_affine(x, None, bias, norm_kind=kind)
        R.within(y, R.norm(x, one, bias.double()[None], kind == C.NORM_LN, 1e-6, 50)["y"], "y")
