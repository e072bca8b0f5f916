"""Keys at or past a sample's kv_len are never read: a workgroup of the bfloat16 dK, dV kernels whose keys no query sees
stores its zeros without a load of K or V rows, on the instructions of the built library (needs no GPU; a value that was
read and dropped shows in no result)."""
import pytest

import test_lds_ring_order as ring
from test_lds_ring_order import kernels  # noqa: F401  (the fixture)

DKV = "dkv_kernelILi"


@pytest.fixture(scope="module", autouse=True)
def named():
    before = ring.KERNELS
    ring.KERNELS = (DKV,)
    yield
    ring.KERNELS = before


def stores_without_row_loads(ins):
    """Whether a path leads from the entry to a store and meets no load of 16 bytes a lane (how rows of K and V are read,
    into registers or LDS)."""
    index = {a: i for i, (a, *_) in enumerate(ins)}
    seen, work = set(), [0]
    while work:
        i = work.pop()
        while i < len(ins) and i not in seen:
            seen.add(i)
            _, op, _, target = ins[i]
            if op.split("_")[0] in ("global", "flat", "buffer"):
                if "store" in op:
                    return True
                if "load" in op and "x4" in op:
                    break
            if target is not None:
                work.append(index[target])
                if op == "s_branch":
                    break
            if op == "s_endpgm":
                break
            i += 1
    return False


def test_the_walk_tells_the_two_apart():
    listing = """0000000000000100 <k>:
\ts_cbranch_scc1 2                              // 000000000100: 00 <k+0xc>
\tglobal_load_dwordx4 v[0:3], v4, s[0:1]        // 000000000104: 00
\ts_nop 0                                       // 000000000108: 00
\tglobal_store_dwordx4 v4, v[0:3], s[0:1]       // 00000000010C: 00
\ts_endpgm                                      // 000000000114: 00
"""
    assert stores_without_row_loads(ring.instructions(listing))
    assert not stores_without_row_loads(ring.instructions(listing.replace("s_cbranch_scc1 2 ", "s_nop 0 ")))


def test_keys_that_no_query_sees_are_not_read(named, kernels):  # noqa: F811
    assert len(kernels) == 2, sorted(kernels)
    for name, text in kernels.items():
        assert stores_without_row_loads(ring.instructions(text)), name
