"""What the block pool's chunks of new tokens refuse, and how they leave the pool then.  Pools on the CPU:
no GPU here."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_blocks_host import make, rows  # noqa: E402
from tests.test_pool_chunk_host import blocks, everything, rotary  # noqa: E402,F401


@pytest.mark.parametrize("scale", [1e-46, 1e-300, 2.36e38, 3.4e38, 1e39])
def test_scales_that_the_attention_refuses(blocks, rotary, scale):  # noqa: F811
    """A scale that is 0 or infinite in 32 bits, or infinite times log2(e), is refused before tokens are
    stored: no tokens twice after another try."""
    pool = make(blocks)
    before = everything(pool)
    with pytest.raises(ValueError):
        pool.extend(rows(48, 4), rows(48), rows(48), [16, 16, 16], rotary, scale=scale)
    assert everything(pool) == before
    with pytest.raises(ValueError):
        pool.attend_chunk(rows(0, 4), [0, 0, 0], scale=scale)
