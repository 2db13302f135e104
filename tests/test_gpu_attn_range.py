"""The range of attention's 16-bit values: what a key far below the largest score adds, and what a
small channel of a query adds, against the definitions in 64 bits.

An attention sink is the usual case: one key takes nearly all of a row's weight, its value is
small, and the output is what the many other keys add.  A weight that goes into the second product
in fp16 is rounded to 2^-11 of itself, or by 2^-25 of fp16's unit where it is subnormal.  The
largest weight of a row may stand at 2^7 at least (weights are at most 2^8 above it, and fp16 ends
at 2^16), so that is 2^-32 of the largest weight, or of the row's sum, for each key.
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
