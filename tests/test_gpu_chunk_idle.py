"""Attention of new tokens where most sequences have none: a pool passes all of its slots, and in a step
few may be at work."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_attn_chunk import call  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets, pool  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture
def netkv():
    from paper_2606_03910_gb300 import netkv
    return netkv


def check(netkv, n, active, idle_tokens=40, heads=8, kv_heads=2, dim=64):
    """active: (sequence, new tokens, tokens before them); the others hold idle_tokens.  The call splits
    and sums as one of the active sequences alone does, so its outputs are the same to the bit."""
    width = max(-(-max(a + b for _, a, b in active) // 16), -(-idle_tokens // 16))
    pages = netkv.KvPages(*pool(len(active) * width, kv_heads, dim, "int8"))
    own = torch.arange(len(active) * width, dtype=torch.int32, device="cuda").view(-1, width)
    at = ints([i for i, _, _ in active], torch.int64)
    counts = torch.zeros(n, dtype=torch.int64, device="cuda")
    counts[at] = ints([a for _, a, _ in active], torch.int64)
    off = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    length = torch.full((n,), idle_tokens, dtype=torch.int32, device="cuda")
    length[at] = ints([a + b for _, a, b in active])
    table = torch.zeros((n, width), dtype=torch.int32, device="cuda")
    table[at] = own
    rows = sum(a for _, a, _ in active)
    q = torch.randn((rows, heads, dim), device="cuda").half()
    got, want = torch.full_like(q, 5), torch.full_like(q, 6)
    assert call(netkv, pages, q, off, length, table, got) == 0
    assert call(netkv, pages, q, offsets([a for _, a, _ in active]), ints([a + b for _, a, b in active]), own,
                want) == 0
    assert torch.equal(got, want)


@pytest.mark.parametrize("at", [[0], [4095], [31, 32], [0, 4095], [0, 33, 64, 4000], [31, 63, 95, 4095],
                                [1, 2, 40, 41, 42, 2047, 2048, 4094]])
@pytest.mark.parametrize("tokens", [(1, 0), (4, 500), (300, 1000)])
def test_few_of_many(netkv, at, tokens):
    check(netkv, 4096, [(i, *tokens) for i in at])


def test_gaps_of_every_size(netkv):
    """Around the 32 sequences that are looked at together."""
    at = [0]
    for gap in (1, 2, 30, 31, 32, 33, 63, 64, 65, 96, 97, 500):
        at.append(at[-1] + gap)
    check(netkv, at[-1] + 70, [(i, 1 + i % 5, 17 * (i % 7)) for i in at])


def test_as_many_sequences_as_a_call_takes(netkv):
    """Rows in the first, a middle and the last of 2^24 - 1 sequences: no wait runs out on the way."""
    n = (1 << 24) - 1
    check(netkv, n, [(0, 3, 9), (n // 3, 1, 13), (n - 1, 2, 6)], idle_tokens=3)
