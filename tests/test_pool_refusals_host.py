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


def test_nothing_is_asked_for_after_tokens_are_stored(blocks, rotary, monkeypatch):  # noqa: F811
    """Outputs, rotated queries and the workspace are there before the append: where they do not fit, the
    pool is as it was."""
    pool, empty, empty_like, log = make(blocks), torch.empty, torch.empty_like, []
    monkeypatch.setattr(blocks.netkv, "netkv_kv_append", lambda *a, **k: log.append("append"))
    monkeypatch.setattr(blocks.netkv, "netkv_attn_chunk", lambda *a, **k: log.append("attend"))
    monkeypatch.setattr(torch, "empty", lambda *a, **k: log.append("empty") or empty(*a, **k))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: log.append("empty") or empty_like(*a, **k))
    pool.extend(rows(48, 4), rows(48), rows(48), [16, 16, 16], rotary)
    assert log.count("append") == log.count("attend") == 1 and log.count("empty") >= 4
    assert log[-2:] == ["append", "attend"]


def test_an_attention_that_fails(blocks, rotary, monkeypatch):  # noqa: F811
    """Whatever stops the attention, the tokens that were stored for it are not counted."""
    pool = make(blocks)
    pool.reserve([20, 0, 1])
    before = everything(pool)

    def fail(*a, **k):
        raise blocks.netkv.NetKVError("netkv_attn_chunk", blocks.netkv.NETKV_ECUDA)

    monkeypatch.setattr(blocks.netkv, "netkv_kv_append", lambda *a, **k: None)
    monkeypatch.setattr(blocks.netkv, "netkv_attn_chunk", fail)
    with pytest.raises(blocks.netkv.NetKVError):
        pool.extend(rows(48, 4), rows(48), rows(48), [16, 16, 16], rotary)
    now = everything(pool)
    assert now[0][1:3] == before[0][1:3] and now[1:] == before[1:] and sorted(now[0][0]) == sorted(before[0][0])
