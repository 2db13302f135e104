"""The block pool on a GPU: what it keeps in step with the blocks."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_blocks import check_attend, make, rows  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def test_appends_after_refused_ones():
    """Another type of values, fewer rows than counts, a strided row: refused, and what follows is as
    if it had not been asked."""
    pool = make(pages=12)
    pool.append(rows(20), rows(20, seed=1), [10, 0, 10])
    free, held = list(pool.free), [list(p) for p in pool.page_of]
    for k, v, counts, error in ((rows(60), rows(60).bfloat16(), [20, 20, 20], TypeError),
                                (rows(59), rows(59), [20, 20, 20], ValueError),
                                (rows(60, dim=32), rows(60, dim=32), [20, 20, 20], ValueError),
                                (rows(60).transpose(0, 1).contiguous().transpose(0, 1), rows(60),
                                 [20, 20, 20], ValueError)):
        with pytest.raises(error):
            pool.append(k, v, counts)
        assert pool.free == free and pool.page_of == held and pool.tokens == [10, 0, 10]
    pool.append(rows(64, seed=2), rows(64, seed=3), [20, 30, 14])
    check_attend(pool, rows(3, heads=6, seed=4), pool.mass.clone())
    assert int(pool.status) == 0


def test_a_moved_sequence_keeps_its_weights():
    """The weight that each block has drawn goes with it: eviction after a move takes the blocks that
    it would have taken before."""
    from paper_2606_03910_gb300.blocks import move
    pool = make(slots=1, width=20)
    pool.append(rows(200), rows(200, seed=1), [200])
    pool.attend(rows(1, heads=6, seed=2) * 4)
    torch.cuda.synchronize()
    drawn = pool.mass[0, :13].clone()
    assert float(drawn.max()) > 2 * float(drawn.min()) > 0
    there = make(slots=2, width=16)
    there.append(rows(30), rows(30), [30, 0])
    move(pool, 0, there, 1)
    assert torch.equal(there.mass[1, :13], drawn) and (there.mass[1, 13:] == 0).all()
    held, order = list(pool.page_of[0]), list(there.page_of[1])
    gone = pool.evict([6], sink=1, recent=1)[0]
    assert [held.index(p) for p in gone] == \
        [order.index(p) for p in there.evict([2, 6], sink=1, recent=1)[1]]
    assert gone != held[1:8]  # not the oldest, as equal weights would have it


def test_a_move_of_a_slot_with_pages_in_advance():
    """Pages that either slot holds beyond its tokens are neither copied nor in the way."""
    from paper_2606_03910_gb300.blocks import move
    pool, there = make(slots=2), make(slots=2)
    pool.append(rows(20), rows(20, seed=1), [20, 0])
    pool.reserve([100, 0])
    there.reserve([0, 60])
    moved = move(pool, 0, there, 1)
    assert moved == 2 * 2 * 2 * (16 * 64 + 4) and there.tokens == [0, 20]
    check_same_tokens(pool, 0, there, 1)


def test_pages_in_advance_outlive_an_eviction():
    """A slot that holds pages for tokens to come still has them in its table after blocks before
    them have gone."""
    pool = make(pages=40, width=16)
    pool.append(rows(170), rows(170, seed=1), [100, 0, 70])
    pool.reserve([60, 40, 0])
    held = [list(p) for p in pool.page_of]
    gone = pool.evict([3, 3, 3], sink=1, recent=1)
    assert [len(x) for x in gone] == [4, 0, 2]
    for s in range(3):
        assert pool.page_of[s] == [p for p in held[s] if p not in gone[s]]
        assert pool.table[s, :len(pool.page_of[s])].tolist() == pool.page_of[s]
    pool.append(rows(110, seed=2), rows(110, seed=3), [60, 40, 10])
    check_attend(pool, rows(3, heads=6, seed=4), pool.mass.clone())
    assert int(pool.status) == 0


def check_same_tokens(a, i, b, j):
    """Two slots' tokens, value for value."""
    n = a.tokens[i]
    assert b.tokens[j] == n and int(b.length[j]) == n
    got = [torch.zeros((n, 2, 64), dtype=torch.float16, device="cuda") for _ in range(4)]
    a.read(got[0], got[1], [n if s == i else 0 for s in range(a.slots)])
    b.read(got[2], got[3], [n if s == j else 0 for s in range(b.slots)])
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3]) and got[0].any()


def test_only_eviction_waits_for_the_device():
    """Every call but evict() only enqueues work: what the host sends is staged, and nothing asks the
    device for an answer."""
    from paper_2606_03910_gb300.blocks import move
    pool, there = make(), make()
    k, v, q = rows(90), rows(90, seed=1), rows(3, heads=6, seed=2)
    pool.append(k[:3], v[:3], [1, 1, 1])
    torch.cuda.synchronize()
    torch.cuda.set_sync_debug_mode("error")
    try:
        pool.append(k, v, [40, 50, 0])
        pool.append(k[:3], v[:3], [1, 1, 1])
        pool.attend(q)
        pool.read(k, v, [40, 50, 0])
        move(pool, 1, there, 2)
        pool.release(1)
        pool.reserve([0, 100, 0])
    finally:
        torch.cuda.set_sync_debug_mode("default")
    torch.cuda.synchronize()
    check_attend(pool, q, pool.mass.clone())
    check_attend(there, q, there.mass.clone())
