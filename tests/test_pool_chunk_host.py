"""The block pool's chunks of new tokens: what is refused, and that nothing changes then.  Pools on the
CPU: no GPU here."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_blocks_host import make, rows, state  # noqa: E402


@pytest.fixture(scope="module")
def blocks():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import blocks
    return blocks


@pytest.fixture(scope="module")
def rotary(blocks):
    return blocks.netkv.Rotary(32)


def everything(pool):
    return state(pool), list(pool.seen), pool.length.tolist()


@pytest.mark.parametrize("change", [
    dict(counts=[16]), dict(counts=[-1, 16, 16]), dict(counts=[16, 16, 17]), dict(counts=[1.5, 0, 0]),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(q=rows(48, 3)),
    dict(q=rows(40, 4)), dict(k=rows(40)), dict(axes=True), dict(counts=[48, 0, 0], width=2)])
def test_refused_chunks_change_nothing(blocks, rotary, change):
    pool = make(blocks, width=change.pop("width", 5))
    before = everything(pool)
    rot = blocks.netkv.Rotary(32, sections=[16, 16]) if change.pop("axes", False) else rotary
    args = {**dict(q=rows(48, 4), k=rows(48), v=rows(48), counts=[16, 16, 16]), **change}
    with pytest.raises(ValueError):
        pool.extend(rotary=rot, **args)
    assert everything(pool) == before


def test_a_chunk_that_the_binding_refuses(blocks, rotary):
    """Tensors of the host: the pages that were taken go back."""
    pool = make(blocks)
    pool.reserve([20, 0, 1])
    before = everything(pool)
    for counts in ([30, 5, 0], [0, 0, 40]):
        n = sum(counts)
        with pytest.raises(TypeError):
            pool.extend(rows(n, 4), rows(n), rows(n), counts, rotary)
        now = everything(pool)
        assert now[0][:3] == before[0][:3] and now[1:] == before[1:]
        assert sorted(now[0][0] + sum(now[0][1], [])) == list(range(12))
    with pytest.raises(MemoryError):
        make(blocks, pages=2).extend(rows(48, 4), rows(48), rows(48), [16, 16, 16], rotary)


def test_positions_go_on_behind_what_has_gone(blocks, rotary, monkeypatch):
    """Blocks that were evicted keep their positions: the next token's number counts them."""
    pool, calls = make(blocks), []
    monkeypatch.setattr(blocks.netkv, "netkv_kv_append", lambda *a, **k: calls.append(k["pos"]))
    monkeypatch.setattr(blocks.netkv, "netkv_attn_chunk", lambda *a, **k: None)
    pool.extend(rows(40, 4), rows(40), rows(40), [20, 20, 0], rotary)
    pool.extend(rows(2, 4), rows(2), rows(2), [1, 1, 0], rotary)
    assert calls == [None, None] and pool.seen == [21, 21, 0] and pool.tokens == [21, 21, 0]
    pool.tokens[1] -= 16  # a block given up
    pool.extend(rows(2, 4), rows(2), rows(2), [2, 0, 0], rotary)
    assert calls[2] is None
    pool.extend(rows(5, 4), rows(5), rows(5), [1, 2, 1], rotary)
    assert calls[3].tolist() == [23, 21, 22, 0, 0] and calls[3].dtype == torch.int32
    assert pool.seen == [24, 23, 1]
    pool.release(1)
    assert pool.seen == [24, 0, 1]


def test_seen_moves_along(blocks, monkeypatch):
    src, dst = make(blocks), make(blocks)
    monkeypatch.setattr(blocks.netkv, "netkv_copy_group_async", lambda *a, **k: None)
    src.reserve([20, 0, 0])
    src.tokens[0], src.seen[0] = 20, 36
    blocks.move(src, 0, dst, 2)
    assert dst.seen == [0, 0, 36] and dst.tokens == [0, 0, 20]
