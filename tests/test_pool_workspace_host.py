"""Workspaces of the block pool's calls: calls on other streams may overlap, or come before the last one
has ended, so each has its own, from the stream that it runs on.  Pools on the CPU: no GPU here."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_blocks_host import make, rows  # noqa: E402


@pytest.fixture(scope="module")
def blocks():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import blocks
    return blocks


def test_chunks_of_two_streams_share_no_workspace(blocks, monkeypatch):
    """attend_chunk() changes nothing in the pool, so two of them may run at a time; and a call that needs
    more takes nothing from one that may still run."""
    pool, kept = make(blocks), []
    monkeypatch.setattr(blocks.netkv, "netkv_attn_chunk", lambda *a, **k: kept.append(k["workspace"]))
    pool.reserve([20, 20, 20])
    pool.tokens = [20, 20, 20]
    for counts in ([1, 1, 1], [1, 1, 1], [20, 20, 20], [1, 0, 0]):
        pool.attend_chunk(rows(sum(counts), 4), counts)
    assert len({w.data_ptr() for w in kept}) == 4
    for w, n in zip(kept, (3, 3, 60, 1)):
        assert w.nbytes >= blocks.netkv.netkv_attn_chunk_workspace_size(pool.pages, n, 3, 4)
    assert not any(x is w for x in vars(pool).values() for w in kept)


def test_a_call_with_other_heads_frees_no_workspace_in_use(blocks, monkeypatch):
    """A decode call on another stream than the last one's, and with other heads, while that runs."""
    pool, kept = make(blocks), []
    monkeypatch.setattr(blocks.netkv, "netkv_attn_decode", lambda *a, **k: kept.append(k["workspace"]))
    for heads in (4, 8, 4, 4):
        pool.attend(rows(3, heads))
    assert len({w.data_ptr() for w in kept}) == 4
    for w, heads in zip(kept, (4, 8, 4, 4)):
        assert w.nbytes >= blocks.netkv.netkv_attn_decode_workspace_size(pool.pages, 3, heads, 5, True)
    assert not any(x is w for x in vars(pool).values() for w in kept)
