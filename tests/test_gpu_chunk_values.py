"""Attention of new tokens over values of any size."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_attn_chunk import call  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets, pool, tables  # noqa: E402


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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("new,held", [([4], [500]), ([1, 5], [30000, 9]), ([300, 2], [2000, 70]),
                                      ([700], [20000]), ([20, 300], [-7, -200])])
def test_values_times_a_power_of_two(netkv, fmt, heads, kv_heads, dim, new, held):
    """Value scales times a power of two give outputs times that power, to the bit, as far as bf16 has
    them, whole row blocks and those in parts alike: in between are sums of up to 2^15 times the tokens,
    which are the range of values nearer to fp32's end than the values."""
    total = [a + b for a, b in zip(new, held)]
    blocks = [-(-x // 16) for x in total]
    k, v, ks, vs = pool(sum(blocks), kv_heads, dim, fmt)
    table = tables(blocks, max(blocks), sum(blocks))
    q = torch.randn((sum(new), heads, dim), device="cuda").bfloat16()
    outs = []
    for power in (0, 60, 110, 123, -60, -90):
        out, lse = torch.full_like(q, 5), torch.empty(q.shape[:2], device="cuda")
        # values are up to 1.25, which 2^123 leaves below bf16's end, and the sums of their weights do not
        assert call(netkv, netkv.KvPages(k, v, ks, vs * 2.0 ** power), q, offsets(new), ints(total), table, out,
                    lse=lse) == 0
        outs.append((power, out, lse))
    want, want_lse = outs[0][1:]
    assert torch.isfinite(want.float()).all()
    for power, out, lse in outs[1:]:
        assert torch.equal(lse, want_lse)
        back = out.double() * 2.0 ** -power
        # below bf16's smallest normal number, 2^-126, its steps are 2^-133
        fine = out.abs() >= 2.0 ** -120
        assert torch.equal(back[fine], want.double()[fine])
        assert ((back - want.double()).abs()[~fine] <= 2.0 ** (-133 - power)).all()
