"""The block pool's chunks of new tokens, step by step: turned queries and stored keys as they are held, so
that outputs are bound by their own rounding and that of the weights alone."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_pool_chunk import blocks, held, rows  # noqa: E402,F401
from tests.test_gpu_rotary import ANGLE, exact  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


def check_outputs(pool, turned, counts, out, lse, dtype):
    """Rows of turned [rows, heads, dim] (as 16-bit values) over what the pool's blocks hold."""
    heads, dim = turned.shape[1:]
    kv_heads, row = pool.pages.heads_dim[0], 0
    for s, c in enumerate(counts):
        if c == 0:
            continue
        kk, vv = held(pool, s)
        see = torch.arange(len(kk))[None] <= torch.arange(c)[:, None] + len(kk) - c
        for h in range(heads):
            hk = h // (heads // kv_heads)
            o, z, _, weight, size = plain.attention(turned[row:row + c, h].cpu().double(), kk[:, hk], vv[:, hk],
                                                    dim ** -0.5, see)
            # a weight below fp16's smallest step is off by half of it at most, against a sum of at least 1
            slack = len(kk) * 2.0 ** -25 * float(vv[:, hk].abs().max())
            plain.close_out(out[row:row + c, h].cpu(), o, weight, size, dim, dtype, 2.0 ** -11, slack)
            plain.close_lse(lse[row:row + c, h].cpu(), z, size, dim)
        row += c
    # an output of zeros, or of another row's queries, is not within these bounds
    assert float(out[:row].float().abs().max()) > 0.01


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (6, 6, 64)])
def test_a_run(blocks, fmt, dtype, heads, kv_heads, dim):  # noqa: F811
    slots = 4
    pool = blocks.BlockPool(200, kv_heads, dim, slots, 60, fmt)
    rotary = blocks.netkv.Rotary(dim // 2)
    for i, counts in enumerate([[200, 0, 17, 300], [100, 40, 0, 301], [5, 4, 3, 2], [1, 1, 1, 1], None,
                                [1, 0, 2, 33]]):
        if counts is None:
            pool.attend(rows(slots, heads, dim, dtype, 99))
            assert sum(map(len, pool.evict([10, 8, 8, 20], 2, 2))) > 0
            continue
        n = sum(counts)
        q, k, v = (rows(n, h, dim, dtype, 10 * i + j) for j, h in enumerate((heads, kv_heads, kv_heads)))
        at = [s + t for s, c in zip(pool.seen, counts) for t in range(c)]
        turned = torch.empty_like(q)
        blocks.netkv.netkv_rotate(rotary, q, torch.tensor([at], dtype=torch.int32, device="cuda"), turned)
        out, lse = pool.extend(q, k, v, counts, rotary)
        torch.cuda.synchronize()
        assert int(pool.status) == 0
        check_outputs(pool, turned, counts, out, lse, dtype)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_three_axes(blocks, fmt, dtype):  # noqa: F811
    """Positions of every axis as given: keys to half a step of their codes, and the outputs over them."""
    heads, kv_heads, dim, counts = 4, 2, 64, [40, 25]
    n, sections = sum(counts), [8, 12, 12]
    pool = blocks.BlockPool(20, kv_heads, dim, 2, 8, fmt)
    rotary = blocks.netkv.Rotary(dim // 2, sections=sections)
    q, k, v = (rows(n, h, dim, dtype, h + j) for j, h in enumerate((heads, kv_heads, kv_heads)))
    pos = torch.randint(0, 1000, (3, n), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    out, lse = pool.extend(q, k, v, counts, rotary, positions=pos.cuda())
    turned = torch.empty_like(q)
    blocks.netkv.netkv_rotate(rotary, q, pos.cuda(), turned)
    torch.cuda.synchronize()
    assert int(pool.status) == 0
    want, size = exact(k, pos, [10000.0 ** (-p / 32) for p in range(32)], sections, False)
    row = 0
    for s, c in enumerate(counts):
        got = held(pool, s)[0]
        # a block's scale is its largest value over the format's; int8: half a code of it; e4m3: 2^-4 of the
        # value, and half of the smallest step, 2^-10, of the scale.  Each scale and quotient is rounded to
        # 2^-24 of itself, of up to 448 codes
        scale = pool.pages.tensors[2][pool.table[s, :-(-c // 16)].long()].cpu().double()
        scale = scale.repeat_interleave(16, 0)[:c, :, None]
        x = want[row:row + c]
        step = 0.5 * scale if fmt == "int8" else 2.0 ** -4 * x.abs() + 2.0 ** -10 * scale
        tol = step + ANGLE * size[row:row + c] + 448 * 2.0 ** -23 * scale
        assert ((got - x).abs() <= tol).all()
        row += c
    check_outputs(pool, turned, counts, out, lse, dtype)


def test_chunks_on_two_streams(blocks):  # noqa: F811
    """attend_chunk() changes nothing in the pool: calls on two streams at once, small ones and ones that
    need more in turn, give what they give one after another."""
    heads, kv_heads, dim = 8, 2, 128
    pool = blocks.BlockPool(700, kv_heads, dim, 2, 400)
    k, v = (rows(8000, kv_heads, dim, torch.bfloat16, j) for j in range(2))
    pool.append(k, v, [5000, 3000])
    calls = [(rows(sum(c), heads, dim, torch.bfloat16, i), c)
             for i, c in enumerate([[4, 0], [600, 1], [1, 3], [90, 700], [2, 2], [1000, 1000]])]
    want = [pool.attend_chunk(q, c) for q, c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for turn in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                for j in range(len(calls)):
                    at = (j + turn + 3 * i) % len(calls)
                    got.append((at, pool.attend_chunk(*calls[at])))
    torch.cuda.synchronize()
    assert int(pool.status) == 0
    for at, (out, lse) in got:
        assert torch.equal(out, want[at][0]) and torch.equal(lse, want[at][1])
