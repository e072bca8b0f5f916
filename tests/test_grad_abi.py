"""Refusals of the training step's operators (include/ff_grad.h): they come from the host, before any device call."""
import ctypes
from ctypes import byref, c_size_t, c_void_p

import pytest
import torch

from paper_2602_12529_amd import _lib, api
from paper_2602_12529_amd import configs as C

FAKE = 1 << 20


def shape(**kw):
    s = dict(B=2, heads=4, kv_heads=2, n_q=10, n_kv=12, head_dim=64, dtype=C.BF16, causal=0, scale=0.0, kv_len=None)
    s.update(kw)
    return _lib.AttnShape(*(s[k] for k in ("B", "heads", "kv_heads", "n_q", "n_kv", "head_dim", "dtype", "causal", "scale", "kv_len")))


def heads(n, h, d=64, data=FAKE, batch=None, head=None, token=None):
    return ((ctypes.c_int64 * 4))(data or 0, n * h * d if batch is None else batch, n * d if head is None else head, d if token is None else token)


def forward(sh, q=None, k=None, out=None, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    q = q or heads(sh.n_q, sh.heads, sh.head_dim)
    k = k or heads(sh.n_kv, sh.kv_heads, sh.head_dim)
    out = out or heads(sh.n_q, sh.heads, sh.head_dim)
    return _lib.load().ff_attention_forward(byref(sh), byref(q), byref(k), byref(k), byref(out), lse, ws, ws_bytes, None)


def backward(sh, dk=None, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
    q, k = heads(sh.n_q, sh.heads, sh.head_dim), heads(sh.n_kv, sh.kv_heads, sh.head_dim)
    return _lib.load().ff_attention_backward(byref(sh), byref(q), byref(q), byref(k), byref(k), byref(q), lse, byref(q),
                                             byref(dk or k), byref(k), ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), _lib.FF_EINVAL), (dict(heads=0), _lib.FF_EINVAL), (dict(heads=5), _lib.FF_EINVAL), (dict(n_q=-1), _lib.FF_EINVAL),
    (dict(causal=2), _lib.FF_EINVAL), (dict(scale=float("nan")), _lib.FF_EINVAL), (dict(scale=float("inf")), _lib.FF_EINVAL),
    (dict(kv_len=FAKE + 2), _lib.FF_EINVAL), (dict(head_dim=136), _lib.FF_EUNSUPPORTED), (dict(head_dim=36), _lib.FF_EUNSUPPORTED),
    (dict(head_dim=6, dtype=C.F32), _lib.FF_EUNSUPPORTED), (dict(n_q=(1 << 27) + 1), _lib.FF_EUNSUPPORTED),
    (dict(n_kv=1 << 28), _lib.FF_EUNSUPPORTED), (dict(heads=1 << 17, kv_heads=1), _lib.FF_EUNSUPPORTED),
    (dict(B=1 << 20, n_q=1 << 12), _lib.FF_EUNSUPPORTED),
])
def test_attention_shapes_refused(kw, code):
    sh = shape(**kw)
    n = c_size_t()
    assert forward(sh) == code and _lib.load().ff_last_error()
    assert backward(sh) == code
    assert _lib.load().ff_attention_forward_workspace_size(byref(sh), byref(n)) == code
    assert _lib.load().ff_attention_backward_workspace_size(byref(sh), byref(n)) == code


def test_attention_operands_refused():
    lib, sh = _lib.load(), shape()
    E, W, U = _lib.FF_EINVAL, _lib.FF_EWORKSPACE, _lib.FF_EUNSUPPORTED
    assert forward(sh, q=heads(10, 4, data=None)) == E
    assert forward(sh, q=heads(10, 4, data=FAKE + 8)) == E
    assert forward(sh, q=heads(10, 4, token=68)) == E             # strides in 16-byte steps
    assert forward(sh, q=heads(10, 4, token=-64)) == E
    assert forward(sh, q=heads(10, 4, batch=1 << 41)) == U
    assert forward(sh, q=heads(10, 4, token=(1 << 24) + 8)) == U
    assert forward(sh, out=heads(10, 4, token=0)) == E             # rows of an output overlap
    assert forward(sh, out=heads(10, 4, head=64, token=64)) == E
    assert forward(sh, out=heads(10, 4, token=56)) == E
    assert forward(sh, lse=None) == E and forward(sh, lse=FAKE + 2) == E
    assert backward(sh, dk=heads(12, 2, head=64, token=64)) == E
    assert backward(sh, lse=None) == E
    assert backward(sh, ws=None) == W and backward(sh, ws_bytes=8) == W and backward(sh, ws=FAKE + 8) == E
    split = shape(B=1, n_q=1, n_kv=4096)
    n = c_size_t()
    assert lib.ff_attention_forward_workspace_size(byref(split), byref(n)) == 0 and n.value > 0
    assert forward(split, ws=None) == W and forward(split, ws_bytes=n.value - 1) == W
    assert lib.ff_attention_forward(None, None, None, None, None, None, None, 0, None) == E
    q = heads(10, 4)
    assert lib.ff_attention_forward(byref(sh), byref(q), None, byref(q), byref(q), FAKE, None, 0, None) == E
    assert lib.ff_attention_forward_workspace_size(byref(sh), None) == E
    # nothing to do
    assert forward(shape(B=0), q=(ctypes.c_int64 * 4)(), k=(ctypes.c_int64 * 4)(), out=(ctypes.c_int64 * 4)(), lse=None) == 0
    assert forward(shape(n_q=0), q=(ctypes.c_int64 * 4)(), out=(ctypes.c_int64 * 4)(), lse=None) == 0


def test_norm_refused():
    lib = _lib.load()
    E, U, W = _lib.FF_EINVAL, _lib.FF_EUNSUPPORTED, _lib.FF_EWORKSPACE
    p, big = c_void_p(FAKE), 1 << 40

    def fwd(x=p, ldx=64, y=p, ldy=64, w=p, rows=4, H=64, kind=1, eps=1e-6, dt=1):
        return lib.ff_norm_affine(x, ldx, w, None, y, ldy, rows, H, kind, eps, dt, None)

    assert fwd(dt=3) == E and fwd(kind=2) == E and fwd(eps=0.0) == E and fwd(eps=float("nan")) == E and fwd(rows=-1) == E
    assert fwd(H=0) == E and fwd(x=None) == E and fwd(y=None) == E and fwd(ldx=63) == E and fwd(w=c_void_p(FAKE + 1)) == E
    assert fwd(ldy=72) == E                                                              # y over x with another stride
    assert fwd(rows=(1 << 27) + 1) == U and fwd(ldx=(1 << 22) + 1) == U and fwd(H=(1 << 22) + 1, ldx=1 << 23, ldy=1 << 23) == U
    assert fwd(rows=0, x=None, y=None) == 0

    def bwd(dy=p, x=p, add=None, ldadd=64, dx=p, lddx=64, dw=p, rows=4000, ws=p, nb=big):
        return lib.ff_norm_affine_backward(dy, 64, x, 64, p, add, ldadd, dx, lddx, dw, p, rows, 64, 1, 1e-6, 1, ws, nb, None)

    assert bwd(dy=None) == E and bwd(x=None) == E and bwd(dw=c_void_p(FAKE + 2)) == E and bwd(add=p, ldadd=32) == E
    assert bwd(lddx=128) == E and bwd(ws=None) == W and bwd(nb=16) == W and bwd(ws=c_void_p(FAKE + 4)) == E

    def mod(rps=2000, mod_ld=64, dmod_ld=64, scale=p, rows=8000):
        return lib.ff_norm_modulate_backward(p, 64, p, 64, scale, mod_ld, rps, None, 0, c_void_p(2 * FAKE), 64, p, p, dmod_ld, rows, 64, 0,
                                             1e-6, 1, p, 16, None)

    assert mod(rps=0) == E and mod(mod_ld=32) == E and mod(dmod_ld=32) == E and mod(scale=c_void_p(FAKE + 2)) == E
    assert mod(rps=1, rows=65536) == U and mod() == W and mod(rows=0) == 0
    n = c_size_t()
    assert lib.ff_norm_backward_workspace_size(4, 64, 0, byref(n)) == E and lib.ff_norm_backward_workspace_size(4, 64, 2, None) == E
    assert lib.ff_norm_backward_workspace_size(65536, 64, 1, byref(n)) == U
    assert lib.ff_norm_backward_workspace_size(0, 64, 0, byref(n)) == 0 and n.value == 0


def test_binding_refuses():
    """Tensors of the host, of another type or shape, and layouts that the structures cannot hold."""
    q = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.attention_forward(q, q, q)
    with pytest.raises(ValueError):
        api.attention_forward(q[0], q[0], q[0])
    with pytest.raises(ValueError):
        api.attention_forward(q.half(), q.half(), q.half())
    for kw in (dict(kv_len=torch.zeros(1)), dict(kv_len=torch.zeros(2, dtype=torch.int32)), dict(scale=0.0), dict(scale=float("inf"))):
        with pytest.raises(ValueError):
            api.attention_forward(q, q, q, **kw)
    with pytest.raises(ValueError):
        api._heads(q.transpose(2, 3), q.transpose(2, 3).shape, q.dtype, q.device, "Q")
    with pytest.raises(ValueError):
        api._heads(q, torch.Size((1, 2, 9, 64)), q.dtype, q.device, "Q")
    with pytest.raises(ValueError):
        api._heads(q, q.shape, q.dtype, torch.device("cuda", 0), "Q")
    with pytest.raises(ValueError):
        api._device(q)
    with pytest.raises(ValueError):
        api._lse_ok(torch.zeros(1, 2, 9), q)
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        api.norm_affine(x)
    with pytest.raises(ValueError):
        api._matrix(x[:, ::2], x[:, :32], "x")
    with pytest.raises(ValueError):
        api._vector(torch.zeros(63), 64, torch.float32, "w")


@pytest.mark.parametrize("scale", [1e-50, -1e-50, 2.0 ** -65, 2.0 ** 65, float("nan")])
def test_binding_refuses_scales_that_float32_would_lose(scale):
    """1e-50 is 0 in float32, which the library takes as the default scale."""
    q = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scale"):
        api.attention_forward(q, q, q, scale=scale)
    with pytest.raises(ValueError, match="scale"):
        api.attention_backward(q, q, q, q, q, torch.zeros(1, 2, 8), scale=scale)


def test_binding_refuses_a_broadcast_scale():
    """One row of scales for every sample has a row stride of 0, which mod_ld = 0 does not stand for."""
    x, scale = torch.zeros(6, 64), torch.zeros(1, 64)
    for mod_ld in (0, 64):
        with pytest.raises(ValueError, match="scale"):
            api.norm_modulate_backward(x, x, scale=scale.expand(3, 64), mod_ld=mod_ld, rows_per_sample=2)
    with pytest.raises(ValueError, match="scale"):
        api.norm_modulate_backward(x, x, scale=torch.zeros(3, 128)[:, :64], rows_per_sample=2)
    with pytest.raises(ValueError, match="current device"):   # dense rows are taken
        api.norm_modulate_backward(x, x, scale=torch.zeros(3, 64), rows_per_sample=2)


def test_structures_match_the_header():
    assert ctypes.sizeof(_lib.AttnShape) == 72
