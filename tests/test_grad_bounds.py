"""The bounds of grad_bounds notice a lost split or block on long axes (needs no GPU)."""
import pytest
import torch

import grad_bounds as G


def keep(t):
    return t.to(torch.bfloat16)


@pytest.mark.parametrize("n_kv,d,splits", [(17000, 64, 64), (16128, 128, 63), (1088, 128, 4)])
def test_a_split_missing_from_a_token_is_noticed(n_kv, d, splits):
    Q, K, V, _ = G.operands(900, 1, 1, 1, 1, n_kv, d, "cpu")
    ref = G.attention(Q, K, V)["out"]
    assert G.worst(keep(ref[0]), ref) <= 0.5          # the stored output's rounding alone
    per = -(-(-(-n_kv // 64)) // splits) * 64
    for s in range(-(-n_kv // per)):
        got = G.attention(Q, K, V, without=(slice(s * per, (s + 1) * per), None))["out"][0]
        assert G.worst(keep(got), ref) > 1.0, s


@pytest.mark.parametrize("size,keys", [((1, 8, 2, 1, 5000, 128), True), ((1, 2, 1, 3000, 40, 128), False), ((1, 1, 1, 700, 700, 64), True),
                                       ((1, 1, 1, 700, 700, 64), False)], ids=["token", "queries", "square_keys", "square_queries"])
def test_a_block_missing_from_a_gradient_is_noticed(size, keys):
    """32 keys missing from dQ, or 32 queries from dK and dV."""
    Q, K, V, dO = G.operands(910, *size, "cpu")
    out = keep(G.attention(Q, K, V)["out"][0])
    ref = G.attention(Q, K, V, dO=dO, out=out)
    for name in ("dQ", "dK", "dV"):
        assert G.worst(keep(ref[name][0]), ref[name]) <= 1.0, name
    for at in range(0, size[4] if keys else size[3], 32 * 7):
        block = slice(at, at + 32)
        got = G.attention(Q, K, V, dO=dO, out=out, without=(block, None) if keys else (None, block))
        for name in ("dQ",) if keys else ("dK", "dV"):
            assert G.worst(keep(got[name][0]), ref[name]) > 1.0, (name, at)
