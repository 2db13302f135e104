"""The block pool and the example that runs scorer, prompts, blocks, decode and eviction together."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def make(fmt="int8", slots=3, pages=40, heads=2, dim=64, width=20):
    from paper_2606_03910_gb300.blocks import BlockPool
    return BlockPool(pages, heads, dim, slots, width, fmt)


def rows(n, heads=2, dim=64, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, heads, dim), generator=g).half().cuda()


def check_attend(pool, q, before):
    """attend() against the blocks' values in 64 bits."""
    out, lse = pool.attend(q)
    torch.cuda.synchronize()
    k, v, ks, vs = [x.cpu().float().double() for x in pool.pages.tensors]
    heads, group = k.shape[1], q.shape[1] // k.shape[1]
    for s in range(pool.slots):
        n, pages = pool.tokens[s], pool.page_of[s]
        assert pool.table[s, :len(pages)].tolist() == pages and int(pool.length[s]) == n
        drawn = torch.zeros(len(pages) * 16, dtype=torch.float64)
        for h in range(heads):
            kk = (k[pages, h] * ks[pages, h][:, None, None]).flatten(0, 1)
            vv = (v[pages, h] * vs[pages, h][:, None, None]).flatten(0, 1)
            see = (torch.arange(len(kk)) < n).expand(group, -1)
            at = slice(h * group, (h + 1) * group)
            o, z, p, weight, size = plain.attention(q[s, at].cpu().double(), kk, vv,
                                                    q.shape[2] ** -0.5, see)
            plain.close_out(out[s, at].cpu(), o, weight, size, q.shape[2], q.dtype, 2.0 ** -11,
                            n * 2.0 ** -25 * 8)
            plain.close_lse(lse[s, at].cpu(), z, size, q.shape[2])
            drawn += p.sum(0)
        want = before[s, :len(pages)].cpu().double() + drawn.view(-1, 16).sum(1)
        assert torch.allclose(pool.mass[s, :len(pages)].cpu().double(), want, rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_pool_appends_attends_evicts_and_moves(fmt):
    from paper_2606_03910_gb300.blocks import move
    pool = make(fmt)
    pool.append(rows(170), rows(170, seed=1), [100, 0, 70])
    pool.append(rows(3, seed=2), rows(3, seed=3), [1, 1, 1])
    check_attend(pool, rows(3, heads=6, seed=4), pool.mass.clone())
    assert len(pool.free) == 40 - 7 - 1 - 5
    before = [list(p) for p in pool.page_of]
    gone = pool.evict([5, 5, 3], sink=1, recent=1)
    assert [len(x) for x in gone] == [2, 0, 2] and pool.tokens == [101 - 32, 1, 71 - 32]
    for s in range(3):
        assert set(gone[s]) | set(pool.page_of[s]) == set(before[s])
        assert before[s][0] == pool.page_of[s][0] and before[s][-1] == pool.page_of[s][-1]
    check_attend(pool, rows(3, heads=6, seed=5), pool.mass.clone())
    other = make(fmt, slots=2)
    moved = move(pool, 0, other, 1)
    assert moved == 5 * 2 * 2 * (16 * 64 + 4)
    check_attend(other, rows(2, heads=2, seed=6), other.mass.clone())
    a, b = torch.zeros((69, 2, 64), dtype=torch.float16, device="cuda"), rows(69)
    c, d = torch.zeros_like(a), rows(69)
    pool.read(a, b, [69, 0, 0])
    other.read(c, d, [0, 69])
    assert torch.equal(a, c) and torch.equal(b, d)
    pool.release(0)
    assert len(pool.free) == 40 - 1 - 3 and pool.tokens[0] == 0
    assert int(pool.status) == 0 and int(other.status) == 0


def test_pool_refusals():
    from paper_2606_03910_gb300.blocks import move
    pool = make(pages=6, width=5)
    with pytest.raises(MemoryError):
        pool.append(rows(112), rows(112), [48, 32, 32])
    with pytest.raises(ValueError):
        pool.append(rows(81), rows(81), [81, 0, 0])
    assert len(pool.free) == 6 and pool.tokens == [0, 0, 0]
    pool.append(rows(80), rows(80), [80, 0, 0])
    with pytest.raises(ValueError):
        pool.read(rows(81), rows(81), [81, 0, 0])
    with pytest.raises(ValueError):
        move(pool, 1, pool, 0)


def test_bytes_per_token():
    from paper_2606_03910_gb300.blocks import bytes_per_token
    assert bytes_per_token(80, 2, 128) == 41_040  # half of Eq. 1's 81,920, and the scales


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_example_serves_decisions(fmt):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import serve_decisions
    finally:
        sys.path.pop(0)
    lines = []
    results, pools = serve_decisions.serve(steps=10, fmt=fmt, report=lines.append)
    assert len(lines) == 1 + len(pools) and len(pools) > 1
    for d, (out, lse) in results.items():
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        used = [p for s in pools[d].page_of for p in s]
        assert len(set(used)) == len(used) and not set(used) & set(pools[d].free)
        for s, pages in enumerate(pools[d].page_of):
            assert pools[d].table[s, :len(pages)].tolist() == pages
            assert int(pools[d].length[s]) == pools[d].tokens[s]
