"""Attention of a training step refuses an output at the address of another operand: its workgroups write while others
still read (include/ff_grad.h).  From the host, before any device call."""
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
