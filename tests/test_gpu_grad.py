"""The training step's operators (include/ff_grad.h) against 64-bit plain forms, at the sizes, layouts and
masks where they can go wrong."""
import math

import pytest
import torch

import grad_ref as R
from paper_2602_12529_amd import configs as C

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def say(*a):
    print(*a, flush=True)


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def operands(seed, B, h, hk, n_q, n_kv, d, dt, layout):
    def one(i, heads, n):
        if layout == "token":
            return randn(seed + i, B, n, heads, d).to(dt).transpose(1, 2)
        return randn(seed + i, B, heads, n, d).to(dt)
    if layout == "packed":
        x = randn(seed, B, n_q, h + 2 * hk, d).to(dt).transpose(1, 2)
        return x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    return one(0, h, n_q), one(1, hk, n_kv), one(2, hk, n_kv)


def check_attention(api, seed, B, h, hk, n_q, n_kv, d, dt, causal=False, lens=None, layout="head", scale=None, poison=True):
    say("attention", B, h, hk, n_q, n_kv, d, dt, "causal" if causal else "", lens, layout)
    Q, K, V = operands(seed, B, h, hk, n_q, n_kv, d, dt, layout)
    dO = randn(seed + 7, B, n_q, h, d).to(dt).transpose(1, 2)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    ref = R.attention(Q, K, V, lens, causal, scale)
    if lens is not None and poison:   # what lies past a sample's keys is never read
        K, V = K.clone(), V.clone()
        for b, n in enumerate(lens):
            K[b, :, max(0, min(n, n_kv)):] = math.nan
            V[b, :, max(0, min(n, n_kv)):] = math.inf
    out, lse = api.attention_forward(Q, K, V, kv_len=kv_len, causal=causal, scale=scale)
    torch.cuda.synchronize()
    R.within(out, ref["out"], "out")
    R.within(lse, ref["lse"], "lse")
    grads = [torch.full_like(t, math.nan) for t in (Q, K, V)]
    api.attention_backward(dO, Q, K, V, out, lse, kv_len=kv_len, causal=causal, scale=scale, dQ=grads[0], dK=grads[1], dV=grads[2])
    torch.cuda.synchronize()
    K0, V0 = (torch.nan_to_num(t, nan=0.0, posinf=0.0) for t in (K, V))
    ref = R.attention(Q, K0, V0, lens, causal, scale, dO=dO, out=out)
    for name, g in zip(("dQ", "dK", "dV"), grads):
        R.within(g, ref[name], name)


SIZES = [   # B, heads, kv_heads, n_q, n_kv
    (1, 1, 1, 1, 1), (2, 4, 4, 24, 24), (1, 2, 1, 33, 65), (2, 6, 2, 127, 130), (1, 3, 3, 257, 31), (3, 8, 1, 1, 300), (1, 4, 2, 300, 8),
]


@pytest.mark.parametrize("d", [64, 128, 8, 96])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_attention_bf16(gpu_lib, size, d):
    check_attention(gpu_lib, 100, *size, d, BF)


@pytest.mark.parametrize("d", [4, 16, 64, 100, 128])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_attention_f32(gpu_lib, size, d):
    check_attention(gpu_lib, 200, *size, d, F)


@pytest.mark.parametrize("dt,d", [(BF, 128), (BF, 64), (BF, 40), (F, 16), (F, 128)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("size,lens", [((5, 4, 2, 70, 100), (0, 1, 32, 99, 1000)), ((3, 2, 2, 200, 161), (161, 64, 65)),
                                       ((2, 4, 4, 1, 520), (-3, 513))], ids=["short", "more_queries", "token"])
def test_attention_masks(gpu_lib, size, lens, layout, causal, dt, d):
    """Samples without keys, queries that see none (causal with fewer keys than queries), lengths outside
    [0, n_kv], and values past a sample's keys that would spoil any product they entered."""
    check_attention(gpu_lib, 300, *size, d, dt, causal, lens, layout)


@pytest.mark.parametrize("dt,d", [(BF, 128), (BF, 64), (F, 64)])
@pytest.mark.parametrize("size", [(1, 8, 2, 1, 5000), (2, 3, 3, 5, 1500), (1, 2, 1, 3000, 40), (1, 4, 4, 700, 700), (2, 24, 24, 300, 520)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True])
def test_attention_long(gpu_lib, size, d, dt, causal):
    """Few rows against a long axis (split and joined), both ways round, and several tiles of both."""
    check_attention(gpu_lib, 400, *size, d, dt, causal, layout="token")


@pytest.mark.parametrize("dt,d", [(BF, 128), (BF, 64), (F, 40), (F, 128)])
@pytest.mark.parametrize("n_kv", [16128, 17000, 1088])
def test_attention_most_splits(gpu_lib, n_kv, d, dt):
    """One token against keys in 63, 64 (the most) and 4 splits: the join's lanes hold the weights of all of them."""
    check_attention(gpu_lib, 450, 1, 1, 1, 1, n_kv, d, dt)


@pytest.mark.parametrize("dt", [BF, F])
def test_attention_packed_and_scale(gpu_lib, dt):
    check_attention(gpu_lib, 500, 2, 6, 2, 90, 90, 64, dt, True, (90, 41), "packed", scale=0.3)
    check_attention(gpu_lib, 510, 1, 2, 2, 40, 70, 128, dt, scale=-0.05)


def test_attention_packed_gradient_and_broadcast_inputs(gpu_lib):
    """Slices of one packed gradient are written in place and nothing else is; an expanded dO and shared K, V are read."""
    B, h, n, d = 2, 3, 50, 64
    Q, K, V = operands(520, B, h, h, n, n, d, BF, "packed")
    dO = randn(521, 1, 1, 1, d).to(BF).expand(B, h, n, d)
    Ks = K[:1].expand(B, h, n, d)
    buf = torch.full((B, n, 3 * h + 1, d), 7.0, dtype=BF, device="cuda")
    g = buf.transpose(1, 2)
    out, lse = gpu_lib.attention_forward(Q, Ks, V)
    gpu_lib.attention_backward(dO, Q, Ks, V, out, lse, dQ=g[:, :h], dK=g[:, h:2 * h], dV=g[:, 2 * h:3 * h])
    torch.cuda.synchronize()
    ref = R.attention(Q, Ks, V, dO=dO, out=out)
    for i, name in enumerate(("dQ", "dK", "dV")):
        R.within(g[:, i * h:(i + 1) * h], ref[name], name)
    assert bool((buf[:, :, 3 * h] == 7.0).all())


@pytest.mark.parametrize("dt,d", [(BF, 128), (F, 16)])
def test_attention_peaked(gpu_lib, dt, d):
    """Scores far apart: the running maximum moves by more than an exponent's range within a row."""
    B, h, n = 1, 2, 200
    Q, K, V = operands(530, B, h, h, n, n, d, dt, "head")
    K = (K.float() * torch.linspace(0.05, 12.0, n, device="cuda").view(1, 1, n, 1)).to(dt)
    dO = randn(531, B, h, n, d).to(dt)
    out, lse = gpu_lib.attention_forward(Q, K, V)
    dQ, dK, dV = gpu_lib.attention_backward(dO, Q, K, V, out, lse)
    torch.cuda.synchronize()
    ref = R.attention(Q, K, V, dO=dO, out=out)
    for name, t in (("out", out), ("lse", lse), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        R.within(t, ref[name], name)


def test_attention_matches_differences(gpu_lib):
    """The gradients against central differences of the 64-bit forward pass along random directions: the error of a
    difference with step t is t^2 / 6 times the third derivative, and of the kernel's float32 sums far less."""
    B, h, hk, n_q, n_kv, d = 1, 4, 2, 20, 27, 16
    Q, K, V = operands(540, B, h, hk, n_q, n_kv, d, F, "head")
    dO = randn(541, B, h, n_q, d)
    out, lse = gpu_lib.attention_forward(Q, K, V, causal=True)
    grads = gpu_lib.attention_backward(dO, Q, K, V, out, lse, causal=True)
    loss = lambda *t: float((R.attention(*(x.double() for x in t), causal=True)["out"][0] * dO.double()).sum())  # noqa: E731
    R.U[torch.float64] = 2.0 ** -53
    for i in range(3):
        e = randn(542 + i, *(Q, K, V)[i].shape).double()
        t = 1e-4
        up, down = ([x.double() + (s * t * e if j == i else 0.0) for j, x in enumerate((Q, K, V))] for s in (1, -1))
        want = (loss(*up) - loss(*down)) / (2 * t)
        got = float((grads[i].double() * e).sum())
        size = float(torch.linalg.norm(grads[i].double()) * torch.linalg.norm(e))
        say("difference", i, got, want)
        assert abs(got - want) <= 1e-5 * size


@pytest.mark.parametrize("dt,d", [(BF, 128), (F, 32)])
@pytest.mark.parametrize("size", [(2, 4, 2, 96, 96), (1, 4, 1, 1, 3000), (1, 1, 1, 2500, 30)], ids=["square", "token", "long"])
def test_attention_repeats_streams_and_graphs(gpu_lib, size, dt, d):
    """The same bits on every run, on another stream and in a replayed graph, on a workspace that holds anything."""
    Q, K, V = operands(550, *size, d, dt, "token")
    dO = randn(551, *Q.shape).to(dt)
    kv_len = torch.tensor([size[4] - 3 * b for b in range(size[0])], dtype=torch.int32, device="cuda")
    nb = max(gpu_lib.attention_backward_workspace_size(Q, K), gpu_lib.attention_forward_workspace_size(Q, K), 16)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")

    def step():
        out, lse = gpu_lib.attention_forward(Q, K, V, kv_len=kv_len, ws=ws)
        return [out, lse, *gpu_lib.attention_backward(dO, Q, K, V, out, lse, kv_len=kv_len, ws=ws)]

    first = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = step()
    for _ in range(3):
        for t in third:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, third))
        step()
        torch.cuda.synchronize()


def test_two_calls_at_once(gpu_lib):
    """Two streams' steps at the same time, each on workspaces of its own, and two captured graphs replayed at the same time."""
    def make(seed, n):
        Q, K, V = operands(seed, 2, 4, 2, n, n, 128, BF, "token")
        dO, x = randn(seed + 3, *Q.shape).to(BF), randn(seed + 4, 3 * n, 1536).to(BF)

        def step():
            out, lse = gpu_lib.attention_forward(Q, K, V)
            return [out, lse, *gpu_lib.attention_backward(dO, Q, K, V, out, lse), *gpu_lib.norm_affine_backward(x, x)]
        return step

    steps = [make(580, 700), make(590, 900)]
    alone = [s() for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                got.append(s())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, alone) for a, b in zip(x, y))
    graphs, outs = [], []
    for s in steps:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(s())
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(outs, alone) for a, b in zip(x, y))
        steps[0]()
        torch.cuda.synchronize()


def test_attention_no_keys_and_no_queries(gpu_lib):
    Q, K = randn(560, 2, 3, 5, 64).to(BF), torch.empty(2, 3, 0, 64, dtype=BF, device="cuda")
    out, lse = gpu_lib.attention_forward(Q, K, K)
    dQ, dK, dV = gpu_lib.attention_backward(Q, Q, K, K, out, lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all()) and bool((dQ == 0).all()) and dK.numel() == 0
    Q0 = torch.empty(2, 3, 0, 64, dtype=BF, device="cuda")
    K = randn(561, 2, 3, 40, 64).to(BF)
    out, lse = gpu_lib.attention_forward(Q0, K, K)
    dQ, dK, dV = gpu_lib.attention_backward(Q0, Q0, K, K, out, lse)
    assert out.numel() == 0 and bool((dK == 0).all()) and bool((dV == 0).all())


@pytest.mark.parametrize("dt,d", [(BF, 40), (F, 16), (F, 128)])
def test_float32_arithmetic_no_keys_and_no_queries(gpu_lib, dt, d):
    Q, K = randn(562, 2, 3, 5, d).to(dt), torch.empty(2, 3, 0, d, dtype=dt, device="cuda")
    out, lse = gpu_lib.attention_forward(Q, K, K)
    dQ, dK, _ = gpu_lib.attention_backward(Q, Q, K, K, out, lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all()) and bool((dQ == 0).all()) and dK.numel() == 0
    Q0, K = torch.empty(2, 3, 0, d, dtype=dt, device="cuda"), randn(563, 2, 3, 40, d).to(dt)
    out, lse = gpu_lib.attention_forward(Q0, K, K)
    _, dK, dV = gpu_lib.attention_backward(Q0, Q0, K, K, out, lse)
    assert bool((dK == 0).all()) and bool((dV == 0).all())


@pytest.mark.parametrize("d", [4, 12, 16, 20])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_f32_narrow_heads(gpu_lib, d, causal):
    """Head dimensions that leave a product over rows partly empty, split and joined, with a negative scale as well."""
    check_attention(gpu_lib, 565, 2, 6, 3, 200, 230, d, F, causal, (230, 57), "token")
    check_attention(gpu_lib, 566, 1, 2, 2, 40, 1500, d, F, causal, scale=-0.4)


@pytest.mark.parametrize("dt,d", [(BF, 64), (F, 64)])
def test_attention_far_offsets(gpu_lib, dt, d):
    """The widest token stride, which takes the last keys and queries past 2^32 bytes."""
    B, h, n, stride = 1, 2, 150, 1 << 24
    buf = torch.zeros(stride * n, dtype=dt, device="cuda").view(n, stride)
    for i in range(3):
        buf[:, 256 * i:256 * i + h * d] = randn(570 + i, n, h * d).to(dt)
    Q, K, V = (buf[:, 256 * i:256 * i + h * d].view(1, n, h, d).transpose(1, 2) for i in range(3))
    dO = randn(574, B, h, n, d).to(dt)
    out, lse = gpu_lib.attention_forward(Q, K, V)
    g = [torch.empty(B, h, n, d, dtype=dt, device="cuda") for _ in range(3)]
    gpu_lib.attention_backward(dO, Q, K, V, out, lse, dQ=g[0], dK=g[1], dV=g[2])
    torch.cuda.synchronize()
    Q, K, V = (t.contiguous() for t in (Q, K, V))
    del buf
    ref = R.attention(Q, K, V, dO=dO, out=out)
    for name, t in (("out", out), ("lse", lse), ("dQ", g[0]), ("dK", g[1]), ("dV", g[2])):
        R.within(t, ref[name], name)


# ------------------------------------------------------------------ norms
def rows_of(seed, R_, H, dt, ld, off=0):
    """[R, H] inside a wider buffer: row stride ld, `off` elements from an aligned start."""
    buf = torch.full((R_ * ld + off,), 3.0, dtype=dt, device="cuda")
    t = buf[off:].view(R_, ld)[:, :H] if R_ else buf[off:].view(0, ld)[:, :H]
    t.copy_((randn(seed, R_, H) * 1.5 + 0.7).to(dt))
    return t


WIDTHS = [1, 7, 64, 96, 200, 512, 513, 1024, 1536, 2560, 3072, 5000, 8192, 8200, 12288, 12296, 20000]


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
def test_norm_affine(gpu_lib, H, dt, layer):
    for n, rows, pad, off in ((0, 37, 0, 0), (1, 1, 0, 0), (2, 70, 8, 8), (3, 9, 3, 1)):
        say("norm_affine", H, dt, layer, rows, pad, off)
        x = rows_of(600 + n, rows, H, dt, H + pad, off)
        w, bias = (randn(610, H) * 0.5 + 1.0).to(dt), randn(611, H).to(dt)
        dy, add = rows_of(612, rows, H, dt, H + pad, off), rows_of(613, rows, H, dt, H + 2 * pad, off)
        use = n != 1
        kind = C.NORM_LN if layer else C.NORM_RMS
        y = gpu_lib.norm_affine(x, w if use else None, bias if use else None, norm_kind=kind, eps=1e-5)
        dx = rows_of(614, rows, H, dt, H + pad, off)
        dx, dw, db = gpu_lib.norm_affine_backward(dy, x, w if use else None, norm_kind=kind, eps=1e-5, add=add if use else None, dx=dx)
        torch.cuda.synchronize()
        one, zero = torch.ones(1, H, dtype=torch.float64, device="cuda"), torch.zeros(1, H, dtype=torch.float64, device="cuda")
        ref = R.norm(x, w.double()[None] if use else one, bias.double()[None] if use else zero, layer, 1e-5, rows, dy, add if use else None)
        R.within(y, ref["y"], "y")
        R.within(dx, ref["dx"], "dx")
        R.within(dw[None], ref["dm"], "dw")
        R.within(db[None], ref["da"], "dbias")


@pytest.mark.parametrize("H", [600, 1501, 1536, 2048, 2560, 3500, 4096, 5000, 7000, 9000, 10001])
@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("layer,with_add", [(True, True), (False, False)], ids=["layer_add", "rms"])
def test_norm_many_rows(gpu_lib, H, dt, layer, with_add):
    """More rows than one to a workgroup, which is cut otherwise than few rows are; the buffers end with the last row and
    what lies around them stays as it was."""
    rows = 2131
    say("many rows", H, dt, layer)
    x, dy, add = (rows_of(650 + i, rows, H, dt, H) for i in range(3))
    w, bias = (randn(653, H) * 0.5 + 1.0).to(dt), randn(654, H).to(dt)
    around = torch.full(((rows + 2) * H,), 3.0, dtype=dt, device="cuda")
    dx = around[H:-H].view(rows, H)
    kind = C.NORM_LN if layer else C.NORM_RMS
    y = gpu_lib.norm_affine(x, w, bias, norm_kind=kind)
    gpu_lib.norm_affine(x, w, bias, norm_kind=kind, y=dx)
    torch.cuda.synchronize()
    assert torch.equal(dx, y) and bool((around[:H] == 3.0).all()) and bool((around[-H:] == 3.0).all())
    _, dw, db = gpu_lib.norm_affine_backward(dy, x, w, norm_kind=kind, add=add if with_add else None, dx=dx)
    torch.cuda.synchronize()
    assert bool((around[:H] == 3.0).all()) and bool((around[-H:] == 3.0).all())
    ref = R.norm(x, w.double()[None], bias.double()[None], layer, 1e-6, rows, dy, add if with_add else None)
    for name, got, want in (("y", y, "y"), ("dx", dx, "dx"), ("dw", dw[None], "dm"), ("dbias", db[None], "da")):
        R.within(got, ref[want], name)


@pytest.mark.parametrize("H", [64, 200, 1536, 3072, 13001])
@pytest.mark.parametrize("dt", [BF, F])
@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("samples,rps,rows", [(1, 100, 100), (3, 41, 123), (4, 33, 110), (50, 1, 50)],
                         ids=["one", "even", "last_short", "single_rows"])
def test_norm_modulate_backward(gpu_lib, H, dt, layer, samples, rps, rows):
    """dshift and dscale as columns of a wider gradient, which keeps its other columns; the norm as ff_norm_modulate computes it."""
    x, dy, add = (rows_of(700 + i, rows, H, dt, H) for i in range(3))
    mod = randn(703, samples, 3 * H + 1)
    scale, shift = mod[:, 1:H + 1], mod[:, H + 1:2 * H + 1]
    dmod = torch.full((samples, 3 * H), 5.0, device="cuda")
    kind = C.NORM_LN if layer else C.NORM_RMS
    y = torch.empty_like(x)
    gpu_lib.norm_modulate(x.contiguous(), y, shift=shift, scale=scale, mod_ld=3 * H + 1, rows_per_sample=rps, norm_kind=kind, eps=1e-6)
    dx, dshift, dscale = gpu_lib.norm_modulate_backward(dy, x, scale=scale, mod_ld=3 * H + 1, rows_per_sample=rps, norm_kind=kind,
                                                        eps=1e-6, add=add, dshift=dmod[:, :H], dscale=dmod[:, 2 * H:])
    torch.cuda.synchronize()
    ref = R.norm(x, 1.0 + scale.double(), shift.double(), layer, 1e-6, rps, dy, add)
    R.within(y, ref["y"], "y")
    R.within(dx, ref["dx"], "dx")
    R.within(dshift, ref["da"], "dshift")
    R.within(dscale, ref["dm"], "dscale")
    assert bool((dmod[:, H:2 * H] == 5.0).all())


@pytest.mark.parametrize("H", [96, 1536, 13001])
def test_norm_in_place_and_missing_outputs(gpu_lib, H):
    """dx over dy, x or add, y over x; single outputs; no rows."""
    x, dy, add = (rows_of(720 + i, 60, H, BF, H) for i in range(3))
    w = randn(724, H).to(BF)
    want = gpu_lib.norm_affine_backward(dy, x, w, add=add)
    for over in range(3):
        t = [dy.clone(), x.clone(), add.clone()]
        got = gpu_lib.norm_affine_backward(t[0], t[1], w, add=t[2], dx=t[over])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), over
    y, z = gpu_lib.norm_affine(x, w), x.clone()
    assert torch.equal(gpu_lib.norm_affine(z, w, y=z), y)
    dw, db = gpu_lib.norm_affine_backward(dy[:0], x[:0], w)[1:]
    assert bool((dw == 0).all()) and bool((db == 0).all())
    lib = gpu_lib.load()
    ws = torch.empty(gpu_lib.norm_backward_workspace_size(60, H, 60), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for keep in range(3):
        outs = [torch.zeros_like(t) for t in want]
        ptr = [t.data_ptr() if i == keep else None for i, t in enumerate(outs)]
        rc = lib.ff_norm_affine_backward(dy.data_ptr(), H, x.data_ptr(), H, w.data_ptr(), add.data_ptr(), H, ptr[0], H, ptr[1], ptr[2],
                                         60, H, C.NORM_LN, 1e-6, C.BF16, ws.data_ptr(), ws.numel(), stream)
        assert rc == 0
        torch.cuda.synchronize()
        assert torch.equal(outs[keep], want[keep])


@pytest.mark.parametrize("H", [7, 50, 513, 1501, 2050])
@pytest.mark.parametrize("dt", [BF, F])
def test_norm_leaves_the_columns_between_rows(gpu_lib, H, dt):
    """Outputs as columns of wider matrices: what lies past column H keeps its value."""
    rows, ld = 77, H + 5
    x, dy = rows_of(660, rows, H, dt, H), rows_of(661, rows, H, dt, H)
    y, dx = (torch.full((rows, ld), 5.0, dtype=dt, device="cuda") for _ in range(2))
    gpu_lib.norm_affine(x, y=y[:, :H])
    gpu_lib.norm_affine_backward(dy, x, dx=dx[:, :H])
    torch.cuda.synchronize()
    assert bool((y[:, H:] == 5.0).all()) and bool((dx[:, H:] == 5.0).all())
    assert torch.equal(y[:, :H], gpu_lib.norm_affine(x)) and torch.equal(dx[:, :H], gpu_lib.norm_affine_backward(dy, x)[0])


def test_norm_far_mean_and_constant_rows(gpu_lib):
    """A mean a thousand times the spread, and rows without any spread: the variance comes from differences."""
    H, rows = 1536, 20
    x = randn(730, rows, H) + 1000.0
    x[3] = 2.5
    dy, w = randn(731, rows, H), randn(732, H)
    y = gpu_lib.norm_affine(x, w)
    dx, dw, db = gpu_lib.norm_affine_backward(dy, x, w)
    zero = torch.zeros(1, H, dtype=torch.float64, device="cuda")
    ref = R.norm(x, w.double()[None], zero, True, 1e-6, rows, dy)
    for n, t in (("y", y), ("dx", dx), ("dm", dw[None]), ("da", db[None])):
        R.within(t, ref[n], n)


def test_norm_matches_differences(gpu_lib):
    """The gradients against central differences of the 64-bit forward pass along random directions."""
    H, rows = 48, 6
    x, w, b, dy = randn(740, rows, H), randn(741, H), randn(742, H), randn(743, rows, H)
    grads = gpu_lib.norm_affine_backward(dy, x, w)

    def loss(x, w, b):
        c = x - x.mean(-1, keepdim=True)
        return float(((c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6) * w + b) * dy.double()).sum())

    t = 1e-4
    for i in range(3):
        e = randn(744 + i, *(x, w, b)[i].shape).double()
        up, down = ([v.double() + (s * t * e if j == i else 0.0) for j, v in enumerate((x, w, b))] for s in (1, -1))
        want, got = (loss(*up) - loss(*down)) / (2 * t), float((grads[i].double() * e).sum())
        size = float(torch.linalg.norm(grads[i].double()) * torch.linalg.norm(e))
        assert abs(got - want) <= 1e-5 * size, (i, got, want)


@pytest.mark.parametrize("rows,H", [(300, 1536), (5, 64), (40, 13001)])
def test_norm_repeats_streams_and_graphs(gpu_lib, rows, H):
    x, dy = rows_of(750, rows, H, BF, H), rows_of(751, rows, H, BF, H)
    w = randn(752, H).to(BF)
    ws = torch.full((gpu_lib.norm_backward_workspace_size(rows, H, rows),), 255, dtype=torch.uint8, device="cuda")
    step = lambda: [gpu_lib.norm_affine(x, w), *gpu_lib.norm_affine_backward(dy, x, w, ws=ws)]  # noqa: E731
    first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = step()
    for _ in range(3):
        for t in third:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, third))
        step()
        torch.cuda.synchronize()


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dt", [F, BF])
def test_block_half_backward(gpu_lib, dt):
    """x + attention(norm(x) W_qkv) as a block runs it, and its gradient through the library's operators and
    plain projections, against 64 bits by torch's own differentiation.

    float32: every step is off by F32(k) of its magnitudes, a chain of eight products, taken as 8 F32(k) of
    the gradient's norm times 4 for its growth through the norm.  bf16: nine tensors on the way are rounded
    (norm, Q K V, P, out, gradients of out, Q K V and the norm's), each by U / sqrt(3) of its norm at
    random: 9 U / sqrt(3) is three times their root sum of squares."""
    B, n, h, d = 2, 45, 4, 64
    H = h * d
    x = randn(800, B * n, H).to(dt)
    w, bias = (1.0 + 0.1 * randn(801, H)).to(dt), (0.1 * randn(802, H)).to(dt)
    W = (randn(803, 3 * H, H) / math.sqrt(H)).to(dt)
    dres = randn(804, B * n, H).to(dt)
    kv_len = torch.tensor([n, 30], dtype=torch.int32, device="cuda")
    mm = lambda a, b: (a.float() @ b.float()).to(dt)  # noqa: E731
    # forward
    xn = gpu_lib.norm_affine(x, w, bias)
    qkv = mm(xn, W.t()).view(B, n, 3, h, d)
    Q, K, V = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    out, lse = gpu_lib.attention_forward(Q, K, V, kv_len=kv_len)
    # backward of y = x + out for dy = dres
    dqkv = torch.empty_like(qkv)
    gpu_lib.attention_backward(dres.view(B, n, h, d).transpose(1, 2), Q, K, V, out, lse, kv_len=kv_len,
                               **{k: dqkv[:, :, i].transpose(1, 2) for i, k in enumerate(("dQ", "dK", "dV"))})
    g = mm(dqkv.view(B * n, 3 * H), W)
    dx, dw, db = gpu_lib.norm_affine_backward(g, x, w, add=dres)
    # 64 bits
    X, Wn, Bn = (t.double().requires_grad_() for t in (x, w, bias))
    c = X - X.mean(-1, keepdim=True)
    q3 = ((c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-6) * Wn + Bn) @ W.double().t()).view(B, n, 3, h, d)
    loss = (X * dres.double()).sum()
    for b, m in enumerate((n, 30)):
        for i in range(h):
            s = q3[b, :, 0, i] @ q3[b, :m, 1, i].t() / math.sqrt(d)
            o = torch.softmax(s, -1) @ q3[b, :m, 2, i]
            loss = loss + (o * dres.view(B, n, h, d)[b, :, i].double()).sum()
    loss.backward()
    tol = 32 * R.f32_steps(H) if dt == F else 9 * R.U[BF] / math.sqrt(3.0)
    for name, got, want in (("dx", dx, X.grad), ("dw", dw, Wn.grad), ("dbias", db, Bn.grad)):
        rel = float(torch.linalg.norm(got.double() - want) / torch.linalg.norm(want))
        say("block", name, rel, tol)
        assert rel <= tol
