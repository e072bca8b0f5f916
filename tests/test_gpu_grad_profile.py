"""What ff_profile_read reports of the training step's attention."""
import pytest
import torch

import grad_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,d", [(torch.bfloat16, 64), (torch.float32, 32)])
@pytest.mark.parametrize("n_q,n_kv", [(130, 130), (70, 200), (200, 70), (1, 50)])
@pytest.mark.parametrize("causal", [False, True])
def test_operations_of_the_pairs_that_are_seen(gpu_lib, n_q, n_kv, causal, dt, d):
    """Two products forward, three in the dQ kernel and four in the dK, dV kernel, 2 d operations to a pair each."""
    B, h = 2, 4
    Q, dO = (torch.randn(B, h, n_q, d, device="cuda").to(dt) for _ in range(2))
    K = torch.randn(B, 2, n_kv, d, device="cuda").to(dt)
    pairs = B * h * int(R.seen_mask(n_q, n_kv, n_kv, causal, "cpu").sum())
    try:
        gpu_lib.profile_reset()
        gpu_lib.profile_enable(True)
        out, lse = gpu_lib.attention_forward(Q, K, K, causal=causal)
        gpu_lib.attention_backward(dO, Q, K, K, out, lse, causal=causal)
        torch.cuda.synchronize()
        gpu_lib.profile_enable(False)
        prof = gpu_lib.profile_read()
    finally:
        gpu_lib.profile_enable(False)
        gpu_lib.profile_reset()
    for name, products in (("attn_forward", 2), ("attn_backward_dq", 3), ("attn_backward_dkv", 4)):
        assert prof[name]["launches"] == 1 and prof[name]["flops"] == products * 2.0 * d * pairs, (name, prof[name], pairs)
