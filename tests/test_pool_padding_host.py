"""Rows of a padded batch in the block pool's outputs.  Pools on the CPU: no GPU here."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_blocks_host import make, rows  # noqa: E402
from tests.test_pool_chunk_host import blocks, rotary  # noqa: E402,F401


def test_rows_of_no_slot_hold_nothing(blocks, rotary, monkeypatch):  # noqa: F811
    """The attention writes the slots' rows only; the outputs are the pool's, so what stands in the others
    is its to say: 0 and -inf, as of rows that see nothing, and not what the memory held."""
    pool, like = make(blocks), torch.empty_like
    monkeypatch.setattr(torch, "empty_like", lambda x, **k: like(x, **k).fill_(math.nan))

    def attend(pages, q, off, length, table, out, lse, **k):
        out[:int(off[-1])], lse[:int(off[-1])] = 7.0, 7.0

    monkeypatch.setattr(blocks.netkv, "netkv_kv_append", lambda *a, **k: None)
    monkeypatch.setattr(blocks.netkv, "netkv_attn_chunk", attend)
    for out, lse in (pool.extend(rows(40, 4), rows(40), rows(40), [20, 0, 3], rotary),
                     pool.attend_chunk(rows(40, 4), [20, 0, 3])):
        assert (out[:23] == 7).all() and (out[23:] == 0).all()
        assert (lse[:23] == 7).all() and (lse[23:] == -math.inf).all()
    out, lse = pool.extend(rows(5, 4), rows(5), rows(5), [1, 4, 0], rotary)
    assert (out == 7).all() and (lse == 7).all()
    out, lse = pool.attend_chunk(rows(2, 4), [0, 0, 0])
    assert (out == 0).all() and (lse == -math.inf).all()
