"""The norms and their gradients with row offsets past 2^32 elements."""
import pytest
import torch

import grad_ref as R
from paper_2602_12529_amd import configs as C

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [40, 2200, 2201, 13001])
@pytest.mark.parametrize("rows,stride", [(2100, 1 << 21), (1030, 1 << 22)], ids=["many", "few"])
def test_norm_rows_past_32_bits(gpu_lib, rows, stride, H):
    """The widest row strides; x, dy, y and dx are columns of one buffer."""
    print("norm", rows, stride, H, flush=True)
    buf = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)
    x, dy, y, dx = (buf[:, 16384 * i:16384 * i + H] for i in range(4))
    g = torch.Generator(device="cuda").manual_seed(960)
    for t in (x, dy):
        t.copy_(torch.randn(rows, H, device="cuda", generator=g))
    w, bias = (torch.randn(H, device="cuda", generator=g).bfloat16() for _ in range(2))
    gpu_lib.norm_affine(x, w, bias, y=y)
    _, dw, db = gpu_lib.norm_affine_backward(dy, x, w, dx=dx)
    _, dshift, dscale = gpu_lib.norm_modulate_backward(dy, x, rows_per_sample=rows, norm_kind=C.NORM_LN)
    torch.cuda.synchronize()
    ref = R.norm(x, w.double()[None], bias.double()[None], True, 1e-6, rows, dy)
    for name, t in (("y", y), ("dx", dx), ("dm", dw[None]), ("da", db[None])):
        R.within(t, ref[name], name)
    assert torch.equal(dscale[0], dw) and torch.equal(dshift[0], db)
