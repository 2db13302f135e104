"""The block pool's host side: what it refuses before any GPU work.  Pools on the CPU: no GPU here."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def blocks():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import blocks
    return blocks


def make(blocks, slots=3, pages=12, heads=2, dim=64, width=5, fmt="int8"):
    return blocks.BlockPool(pages, heads, dim, slots, width, fmt, device="cpu")


def state(pool):
    return list(pool.free), [list(p) for p in pool.page_of], list(pool.tokens), pool.table.tolist()


@pytest.mark.parametrize("other", [dict(heads=1), dict(heads=4), dict(dim=128), dict(fmt="e4m3"),
                                   dict(heads=1, dim=128)])
def test_move_between_unlike_pools(blocks, other):
    """Pages of another shape or format are neither written nor taken."""
    src, dst = make(blocks), make(blocks, **other)
    src.reserve([40, 0, 0])
    src.tokens[0] = 40
    before = state(dst)
    with pytest.raises(ValueError):
        blocks.move(src, 0, dst, 1)
    assert state(dst) == before
