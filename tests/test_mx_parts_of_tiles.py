"""The largest tile's work-groups go on from tile to tile only where tiles are whole: parts of K have a work-group each, whatever the number of
CUs (256 of them always hold all parts that are chosen; a partition of 32 does not)."""
import pytest

from paper_2607_07862_amd import binding as B
from tests._mx_launches import products, program

pytestmark = pytest.mark.skipif(program() is None, reason="hipcc not available")


def cdiv(a, b):
    return -(-a // b)


@pytest.mark.parametrize("cus", [256, 32])
def test_parts_have_a_work_group_each(cus):
    shapes = [(M, N, K, act, B.DTYPE_BF16) for M in (130, 257, 500, 1000, 2000, 4096) for N in (257, 520, 1100, 2111, 4100) for K in (1300, 8300, 20000, 70000)
              for act in (B.ACT_IDENTITY, B.ACT_SWIGLU)]
    crowded = whole = 0
    for (M, N, K, act, _), p in zip(shapes, products(*shapes, cus=cus)):
        if p.choice != 256:
            continue
        tiles = cdiv(M, 256) * cdiv(N, 128 if act == B.ACT_SWIGLU else 256)
        if p.parts == 1:
            assert p.groups == min(tiles, cus)
            whole += tiles > cus
            continue
        stages = cdiv(cdiv(K, 128) * 128, 256)
        parts = cdiv(stages, cdiv(stages, p.parts))
        assert p.groups == tiles * parts, (M, N, K, act, p)
        crowded += p.groups > cus
    assert whole and (crowded if cus == 32 else not crowded)
