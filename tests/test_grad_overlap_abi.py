"""The training step's operators refuse an output at the address of another operand that it may not be: their workgroups
write while others still read (include/ff_grad.h).  From the host, before any device call."""
import ctypes
from ctypes import byref

import pytest

from paper_2602_12529_amd import _lib
from paper_2602_12529_amd import configs as C

STEP = 1 << 24
NAMES = ("dO", "Q", "K", "V", "out", "lse", "dQ", "dK", "dV")


def call(at, backward, n_q=10, n_kv=12, dtype=C.BF16):
    """at: address of every operand by name."""
    B, h, d = 2, 4, 64
    sh = _lib.AttnShape(B, h, h, n_q, n_kv, d, dtype, 0, 0.0, None)
    op = {k: (ctypes.c_int64 * 4)(at[k], h * n * d, n * d, d)
          for k, n in (("dO", n_q), ("Q", n_q), ("K", n_kv), ("V", n_kv), ("out", n_q), ("dQ", n_q), ("dK", n_kv), ("dV", n_kv))}
    lib, ws = _lib.load(), 100 * STEP
    if not backward:
        return lib.ff_attention_forward(byref(sh), *(byref(op[k]) for k in ("Q", "K", "V", "out")), at["lse"], ws, 1 << 40, None)
    return lib.ff_attention_backward(byref(sh), *(byref(op[k]) for k in ("dO", "Q", "K", "V", "out")), at["lse"],
                                     *(byref(op[k]) for k in ("dQ", "dK", "dV")), ws, 1 << 40, None)


@pytest.mark.parametrize("dtype", [C.BF16, C.F32])
@pytest.mark.parametrize("backward,output,other", [(False, o, i) for o, i in [("out", "Q"), ("out", "K"), ("out", "V"), ("out", "lse"),
                                                                             ("lse", "Q"), ("lse", "K"), ("lse", "V")]]
                         + [(True, o, i) for o in ("dQ", "dK", "dV") for i in ("dO", "Q", "K", "V", "out", "lse")]
                         + [(True, "dQ", "dK"), (True, "dQ", "dV"), (True, "dK", "dV")])
def test_an_output_over_another_operand_is_refused(backward, output, other, dtype):
    at = {k: (i + 1) * STEP for i, k in enumerate(NAMES)}
    at[output] = at[other]
    assert call(at, backward, dtype=dtype) == _lib.FF_EINVAL
    message = _lib.load().ff_last_error().decode()
    assert output in message and other in message, message


@pytest.mark.parametrize("rows", [3, 5000])
@pytest.mark.parametrize("same", [("dw", "dbias")] + [(o, i) for o in ("dw", "dbias") for i in ("dy", "x", "add", "dx", "w")] + [("dx", "w")])
def test_norm_gradients_over_another_operand_are_refused(same, rows):
    at = {k: (i + 1) * STEP for i, k in enumerate(("dy", "x", "w", "add", "dx", "dw", "dbias"))}
    at[same[0]] = at[same[1]]
    lib, H, ws = _lib.load(), 64, 100 * STEP
    assert lib.ff_norm_affine_backward(at["dy"], H, at["x"], H, at["w"], at["add"], H, at["dx"], H, at["dw"], at["dbias"], rows, H,
                                       C.NORM_LN, 1e-6, C.BF16, ws, 1 << 40, None) == _lib.FF_EINVAL
    assert b"column sum" in lib.ff_last_error() or b"multiplier" in lib.ff_last_error()
    # the modulated norm: dscale, dshift and scale in their places
    assert lib.ff_norm_modulate_backward(at["dy"], H, at["x"], H, at["w"], H, 1000, at["add"], H, at["dx"], H, at["dbias"], at["dw"], H,
                                         rows, H, C.NORM_RMS, 1e-6, C.BF16, ws, 1 << 40, None) == _lib.FF_EINVAL
    assert b"column sum" in lib.ff_last_error() or b"multiplier" in lib.ff_last_error()


@pytest.mark.parametrize("over", ["w", "bias"])
def test_a_norm_over_its_weight_is_refused(over):
    at = {"w": 2 * STEP, "bias": 3 * STEP}
    lib = _lib.load()
    assert lib.ff_norm_affine(STEP, 64, at["w"], at["bias"], at[over], 64, 10, 64, C.NORM_LN, 1e-6, C.BF16, None) == _lib.FF_EINVAL
    assert b"y is w or bias" in lib.ff_last_error()
