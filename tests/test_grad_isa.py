"""The bfloat16 attention kernels of a training step on the instructions of the built library (needs no GPU): what
they may leave outstanding at a barrier, and that nothing of theirs is spilled to memory."""
import pytest

import test_lds_ring_order as ring
from test_lds_ring_order import kernels  # noqa: F401  (the fixture)

# LDS reads that may be outstanding at a barrier: those of the operands read ahead from tiles that are not refilled
# behind it (two instructions an operand for columns).
READ_AHEAD = {"fwd_kernelILi": 8, "dq_kernelILi": 3, "dkv_kernelILi": 0}


@pytest.fixture(scope="module", autouse=True)
def named():
    before = ring.KERNELS
    ring.KERNELS = tuple(READ_AHEAD)
    yield
    ring.KERNELS = before


@pytest.mark.parametrize("kernel", READ_AHEAD)
def test_reads_of_a_buffer_return_before_the_barrier_that_frees_it(named, kernels, kernel):  # noqa: F811
    ours = {n: t for n, t in kernels.items() if kernel in n}
    assert len(ours) == (2 if kernel.startswith("dkv") else 4), sorted(ours)
    for name, text in ours.items():
        at = ring.reads_outstanding_at_barriers(ring.instructions(text))
        assert at, name
        assert max(at.values()) <= READ_AHEAD[kernel], (name, at)


@pytest.mark.parametrize("kernel", READ_AHEAD)
def test_no_register_is_spilled(named, kernels, kernel):  # noqa: F811
    """A spilled register's reload waits for every memory access before it, the tile loads in flight among them."""
    for name, text in kernels.items():
        if kernel in name:
            assert "scratch_" not in text, name
