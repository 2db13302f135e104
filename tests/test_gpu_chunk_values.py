"""Attention of new tokens over values of any size."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_attn_chunk import WEIGHT_UNIT, call  # noqa: E402
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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("new,held", [(100, 0), (300, 0), (300, 50), (90, 3000)])
@pytest.mark.parametrize("power", [12, 24, 40, 100])
def test_values_of_tokens_that_a_row_does_not_see(netkv, fmt, heads, kv_heads, dim, new, held, power):
    """A chunk whose values grow by a power of two from one of its blocks on: rows before that block are as
    exact as without it, and are the same to the bit whatever stands there."""
    total = new + held
    blocks = -(-total // 16)
    k, v, ks, vs = pool(blocks, kv_heads, dim, fmt)
    table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    q = torch.randn((new, heads, dim), device="cuda").bfloat16()
    large = (held + new // 2) // 16   # the first block of large values
    row = large * 16 - held           # the first row that sees it
    outs = []
    for p in (0, power):
        more = vs.clone()
        more[large:] *= 2.0 ** p
        out, lse = torch.full_like(q, 5), torch.empty((new, heads), device="cuda")
        assert call(netkv, netkv.KvPages(k, v, ks, more), q, offsets([new]), ints([total]), table, out,
                    lse=lse) == 0
        outs.append((out, lse, more))
    assert torch.equal(outs[0][0][:row], outs[1][0][:row]) and torch.equal(outs[0][1], outs[1][1])
    out, _, more = outs[1]
    see = torch.arange(total, device="cuda")[None] <= torch.arange(new, device="cuda")[:, None] + held
    for h in (0, heads - 1):
        hk = h // (heads // kv_heads)
        kh, vh = ((x[:, hk].double() * s[:, hk].double()[:, None, None]).flatten(0, 1)[:total]
                  for x, s in ((k, ks), (v, more)))
        o, _, _, weight, size = plain.attention(q[:, h].double(), kh, vh, dim ** -0.5, see)
        # weights below fp16's smallest step: half of it, times the largest value that the row sees
        for lo, hi in ((0, row), (row, new)):
            top = float(more[:large if lo == 0 else blocks, hk].max()) * plain.TOP[fmt]
            plain.close_out(out[lo:hi, h], o[lo:hi], weight[lo:hi], size, dim, torch.bfloat16, WEIGHT_UNIT,
                            total * 2.0 ** -25 * top)


def test_scales_at_both_ends_of_fp32(netkv):
    """The quotient of a hidden block's scale by a visible one's is past fp32's range."""
    k, v, ks, vs = pool(4, 1, 64, "int8")
    vs[:2], vs[2:] = 1e-30, 1e36
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    q = torch.randn((64, 4, 64), device="cuda").bfloat16()
    out = torch.full_like(q, 5)
    assert call(netkv, netkv.KvPages(k, v, ks, vs), q, offsets([64]), ints([64]), table, out) == 0
    assert torch.isfinite(out.float()).all()
    # values of up to 127 * 1e-30 in the rows before, of up to 127 * 1e36 behind
    assert 0 < out[:32].abs().max() < 1.3e-28 and out[32:].abs().amax((1, 2)).min() > 1e30
