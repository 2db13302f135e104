"""The range of attention's 16-bit values: what a key far below the largest score adds, and what a
small channel of a query adds, against the definitions in 64 bits.

An attention sink is the usual case: one key takes nearly all of a row's weight, its value is
small, and the output is what the many other keys add.  A weight that goes into the second product
in fp16 is rounded to 2^-11 of itself, or by 2^-25 of fp16's unit where it is subnormal.  The
largest weight of a row may stand at 2^7 at least (weights are at most 2^8 above it, and fp16 ends
at 2^16), so that is 2^-32 of the largest weight, or of the row's sum, for each key (decode: times up
to 2 for the unit of the value scales).
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets  # noqa: E402

FLOOR = 2.0 ** -32


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


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [10, 22, 24, 26])
@pytest.mark.parametrize("rows,heads,kv_heads,dim,sink", [(2, 2, 1, 64, 0), (2, 2, 1, 128, 8000),
                                                          (2000, 64, 8, 64, 3), (2000, 63, 9, 128, 0)])
def test_prompt_sinks(netkv, dtype, gap, rows, heads, kv_heads, dim, sink):
    """A sink 2^gap above the other keys, with values of 0."""
    n = 8192
    g = torch.Generator().manual_seed(gap)
    q = 0.05 * torch.randn((rows, heads, dim), generator=g)
    k = torch.randn((n, kv_heads, dim), generator=g)
    v = 0.5 + torch.rand((n, kv_heads, dim), generator=g)
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[sink], v[sink] = 0.0, 0.0
    k[sink, :, 0] = gap * math.log(2)
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    out, lse = torch.empty_like(q), torch.empty((rows, heads), device="cuda")
    netkv.netkv_attn_prompt(q, k, v, offsets([rows]), offsets([n]), out, lse=lse, scale=1.0)
    torch.cuda.synchronize()
    at = torch.tensor(sorted({0, rows // 2, rows - 1}), device="cuda")
    see = torch.arange(n, device="cuda")[None] <= at[:, None] + n - rows
    for h in {0, heads - 1}:
        hk = h // (heads // kv_heads)
        o, z, _, weight, size = plain.attention(q[at, h].double(), k[:, hk].double(),
                                                v[:, hk].double(), 1.0, see)
        slack = n * FLOOR * 1.5 if dtype == torch.float16 else 0.0
        plain.close_out(out[at, h], o, weight, size, dim, dtype, plain.U[dtype], slack)
        plain.close_lse(lse[at, h], z, size, dim)


@pytest.mark.parametrize("n,dim,heads,kv_heads", [(40000, 64, 2, 1), (20000, 128, 16, 2)])
def test_long_prompts_to_a_narrow_bound(netkv, n, dim, heads, kv_heads):
    """Near-uniform scores over many keys, where outputs are small themselves."""
    g = torch.Generator().manual_seed(n)
    q, k, v = (torch.randn((n, h, dim), generator=g).half().cuda() for h in (heads, kv_heads, kv_heads))
    out, off = torch.empty_like(q), offsets([n])
    netkv.netkv_attn_prompt(q, k, v, off, off, out)
    torch.cuda.synchronize()
    at = torch.tensor([0, 100, n // 2, n - 1], device="cuda")
    see = torch.arange(n, device="cuda")[None] <= at[:, None]
    for h in {0, heads - 1}:
        hk = h // (heads // kv_heads)
        o, _, _, weight, size = plain.attention(q[at, h].double(), k[:, hk].double(),
                                                v[:, hk].double(), dim ** -0.5, see)
        plain.close_out(out[at, h], o, weight, size, dim, q.dtype, plain.U[q.dtype], n * FLOOR * 6.0)


def paged(k, v, fmt):
    """Rows k, v [n, heads, dim] float32 as blocks: codes, scales, the values that they stand for
    (float64, on the CPU) and the table of one sequence."""
    n, heads, dim = k.shape
    blocks = -(-n // 16)
    got, values = [], []
    for x in (k, v):
        x = torch.cat([x, torch.zeros((blocks * 16 - n, heads, dim))])
        x = x.view(blocks, 16, heads, dim).transpose(1, 2).contiguous()
        scale = x.abs().amax((2, 3)).clamp_min(2.0 ** -100) / plain.TOP[fmt]
        codes = (x / scale[..., None, None]).clamp(-plain.TOP[fmt], plain.TOP[fmt])
        codes = codes.round().to(torch.int8) if fmt == "int8" else codes.to(torch.float8_e4m3fn)
        got += [codes.cuda(), scale.cuda()]
        values.append((codes.float().double() * scale.double()[..., None, None]).transpose(1, 2)
                      .reshape(blocks * 16, heads, dim)[:n])
    return (got[0], got[2], got[1], got[3]), values, ints(range(blocks)).view(1, blocks)


def decode(netkv, q, tensors, table, n, scale, mass=True):
    """One sequence's output, lse and block weights."""
    heads = q.shape[1]
    pages = netkv.KvPages(*tensors)
    size = netkv.netkv_attn_decode_workspace_size(pages, 1, heads, table.shape[1], mass)
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, heads), device="cuda")
    m = torch.zeros(table.shape, device="cuda") if mass else None
    netkv.netkv_attn_decode(pages, q, ints([n]), table, out, lse=lse, mass_out=m, scale=scale,
                            workspace=ws)
    torch.cuda.synchronize()
    return out[0].cpu(), lse[0].cpu(), None if m is None else m[0].cpu().double()


def check_decode(netkv, q, k, v, fmt, scale=1.0):
    """q [heads, dim] of its type, one KV head."""
    n, dim = len(k), q.shape[1]
    tensors, (kk, vv), table = paged(k, v, fmt)
    out, lse, mass = decode(netkv, q[None].cuda(), tensors, table, n, scale)
    see = torch.ones((len(q), n), dtype=torch.bool)
    o, z, p, weight, size = plain.attention(q.double(), kk[:, 0], vv[:, 0], scale, see)
    # a weight's unit goes by the largest value that a block of the call can hold, and is a power
    # of two up to twice above
    slack = n * 2 * FLOOR * float(tensors[3].max()) * plain.TOP[fmt]
    plain.close_out(out, o, weight, size, dim, q.dtype, 2.0 ** -11, slack)
    plain.close_lse(lse, z, size, dim)
    drawn = torch.cat([p.sum(0), torch.zeros(-n % 16, dtype=torch.float64)]).view(-1, 16).sum(1)
    tol = (2 * plain.score_error(size, dim) + 2.0 ** -18) * drawn + 1e-30
    assert ((mass - drawn).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("gap,sink", [(10, 0), (22, 5), (24, 0), (26, 0), (24, 130000)])
@pytest.mark.parametrize("n,heads,dim", [(500, 8, 64), (131072, 8, 128), (131072, 12, 64)])
def test_decode_sinks(netkv, dtype, fmt, gap, sink, n, heads, dim):
    """A sink 2^gap above the other keys, with values of 0, in a block whose other values are as
    everywhere."""
    sink = min(sink, n - 1)
    g = torch.Generator().manual_seed(gap)
    q = (0.05 * torch.randn((heads, dim), generator=g))
    k = torch.randn((n, 1, dim), generator=g)
    v = 0.5 + torch.rand((n, 1, dim), generator=g)
    q[:, 0], k[..., 0] = 1.0, 0.0
    k[sink], v[sink] = 0.0, 0.0
    k[sink, :, 0] = gap * math.log(2)
    check_decode(netkv, q.to(dtype), k, v, fmt)


@pytest.mark.parametrize("n", [40000, 70000])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_long_decodes_to_a_narrow_bound(netkv, fmt, n):
    """Near-uniform scores over many keys, where outputs are small themselves."""
    g = torch.Generator().manual_seed(n)
    q = torch.randn((8, 128), generator=g).half()
    k, v = torch.randn((n, 1, 128), generator=g), torch.randn((n, 1, 128), generator=g)
    check_decode(netkv, q, k, v, fmt, scale=128 ** -0.5)


@pytest.mark.parametrize("spread", [4, 12])
def test_decode_value_scales_far_apart(netkv, spread):
    """Blocks whose values are 2^spread below another's: that one's scale sets the unit."""
    g = torch.Generator().manual_seed(spread)
    n, dim = 4000, 64
    q = torch.randn((8, dim), generator=g).bfloat16()
    k, v = torch.randn((n, 1, dim), generator=g), torch.rand((n, 1, dim), generator=g)
    v[16:] *= 2.0 ** -spread
    k[:16, :, :] = 0.0
    q[:, 0], k[:, :, 0] = 1.0, 0.0
    k[:16, :, 0] = -20 * math.log(2)  # and the large values have little weight
    check_decode(netkv, q, k, v, "int8")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("heads", [8, 16])
@pytest.mark.parametrize("dtype,large,small", [(torch.float16, 300.0, 0.003),
                                               (torch.float16, 60000.0, 0.01),
                                               (torch.bfloat16, 300.0, 0.003),
                                               (torch.bfloat16, 1.0, 2.0 ** -20),
                                               (torch.bfloat16, 1000.0, 2.0 ** -12)])
def test_decode_channels_of_a_query_far_apart(netkv, dtype, large, small, heads, fmt):
    """One channel dominates the query and is 0 in the keys, as outlier channels are: the others
    make the scores, to all bits that they have."""
    g = torch.Generator().manual_seed(heads)
    n, dim = 700, 64
    q = small * torch.randn((heads, dim), generator=g)
    k, v = torch.randn((n, 1, dim), generator=g) / small, torch.randn((n, 1, dim), generator=g)
    q[:, 5], k[..., 5] = large, 0.0
    check_decode(netkv, q.to(dtype), k, v, fmt, scale=0.5)


@pytest.mark.parametrize("power", [127, 126, 100, -100, -118, -126])
def test_decode_queries_at_the_ends_of_bf16(netkv, power):
    """Queries as large and as small as bf16 holds, with keys that bring the scores back."""
    g = torch.Generator().manual_seed(1)
    n, dim = 100, 64
    q = (1 + torch.rand((8, dim), generator=g)).mul(0.99).double() * torch.randn((8, dim), generator=g).sign()
    q = torch.ldexp(q, torch.tensor(power)).to(torch.bfloat16)
    assert torch.isfinite(q.float()).all() and (q != 0).all()
    k = torch.ldexp(torch.randn((n, 1, dim), generator=g).double(), torch.tensor(-max(-90, min(90, power)))).float()
    v = torch.randn((n, 1, dim), generator=g)
    check_decode(netkv, q, k, v, "int8", scale=2.0 ** (max(-90, min(90, power)) - power) / 8)
