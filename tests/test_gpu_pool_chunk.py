"""New tokens of a block pool's sequences, turned, stored and attended together, against the definition
in 64 bits and against the same tokens in other portions."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_rotary import exact  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture
def blocks():
    from paper_2606_03910_gb300 import blocks
    return blocks


def rows(n, heads, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, heads, dim), generator=g).to(dtype).cuda()


def held(pool, slot):
    """A slot's keys and values, as its codes and scales stand for, [tokens, kv heads, dim] float64."""
    n = pool.tokens[slot]
    k, v, ks, vs = pool.pages.tensors
    pages = pool.table[slot, :-(-n // 16)].long()
    out = []
    for c, s in ((k, ks), (v, vs)):
        x = plain.codes_value(c[pages]) * s[pages].cpu().double()[..., None, None]
        out.append(x.permute(0, 2, 1, 3).flatten(0, 1)[:n])
    return out


@pytest.mark.parametrize("fmt,dtype", [("int8", torch.bfloat16), ("e4m3", torch.float16)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (6, 6, 64)])
def test_a_run(blocks, fmt, dtype, heads, kv_heads, dim):
    """Prompts in two parts, drafted tokens, single ones, an eviction and more tokens: after each step the
    output is that of the turned queries over what the blocks hold."""
    slots, frequencies = 4, [10000.0 ** (-p / (dim // 2)) for p in range(dim // 2)]
    pool = blocks.BlockPool(200, kv_heads, dim, slots, 60, fmt)
    rotary = blocks.netkv.Rotary(dim // 2)
    steps = [[200, 0, 17, 300], [100, 40, 0, 301], [5, 4, 3, 2], [1, 1, 1, 1], None, [1, 0, 2, 33]]
    for i, counts in enumerate(steps):
        if counts is None:
            pool.attend(rows(slots, heads, dim, dtype, 99))
            assert sum(map(len, pool.evict([10, 8, 8, 20], 2, 2))) > 0
            continue
        n = sum(counts)
        q, k, v = (rows(n, h, dim, dtype, 10 * i + j) for j, h in enumerate((heads, kv_heads, kv_heads)))
        at = [s + t for s, c in zip(pool.seen, counts) for t in range(c)]
        out, lse = pool.extend(q, k, v, counts, rotary)
        torch.cuda.synchronize()
        assert int(pool.status) == 0
        want, size = exact(q, torch.tensor([at]), frequencies, [dim // 2], False)
        row = 0
        for s, c in enumerate(counts):
            kk, vv = held(pool, s)
            see = torch.arange(len(kk))[None] <= torch.arange(c)[:, None] + len(kk) - c
            for h in range(heads):
                hk = h // (heads // kv_heads)
                turned = want[row:row + c, h]
                o, z, p, weight, top = plain.attention(turned, kk[:, hk], vv[:, hk], dim ** -0.5, see)
                if c == 0:
                    continue
                # queries are rounded once on the way, by the unit of their type: a score by that of
                # the sum of its products' sizes, a weight and the sum it is divided by by that twice
                off = float(((turned.abs() + 2.0 ** -20 * size[row:row + c, h]) @ kk[:, hk].abs().T).max()) * \
                    dim ** -0.5 * plain.U[dtype]
                spread = math.expm1(2 * off)
                slack = spread * float(vv[:, hk].abs().max()) + len(kk) * 2.0 ** -25 * float(vv[:, hk].abs().max())
                plain.close_out(out[row:row + c, h].cpu(), o, weight, top, dim, dtype, 2.0 ** -11, slack)
                assert ((lse[row:row + c, h].cpu().double() - z).abs() <= off + plain.score_error(top, dim) + 1e-5).all()
            row += c


@pytest.mark.parametrize("cuts", [[64], [16, 48, 160], [240]])
def test_parts_of_a_prompt_are_the_prompt(blocks, cuts):
    """Cut between blocks, a prompt's parts leave the same codes as the whole one, and the same outputs
    up to the order of their sums: weights to 2^-11 and the output to 2^-8 of values below 5, each way."""
    n, heads, kv_heads, dim = 300, 8, 2, 128
    q, k, v = (rows(n, h, dim, torch.bfloat16, j) for j, h in enumerate((heads, kv_heads, kv_heads)))
    rotary = blocks.netkv.Rotary(64, base=500000.0)
    pools = [blocks.BlockPool(20, kv_heads, dim, 1, 20) for _ in range(2)]
    whole, lse = pools[0].extend(q, k, v, [n], rotary)
    parts, at = [], 0
    for to in cuts + [n]:
        parts.append(pools[1].extend(q[at:to], k[at:to], v[at:to], [to - at], rotary))
        at = to
    got, got_lse = (torch.cat([p[i] for p in parts]) for i in (0, 1))
    torch.cuda.synchronize()
    for slot in range(19):
        a, b = int(pools[0].table[0, slot]), int(pools[1].table[0, slot])
        for x, y in zip(pools[0].pages.tensors, pools[1].pages.tensors):
            assert torch.equal(x[a].view(torch.uint8), y[b].view(torch.uint8))
    assert ((got.float() - whole.float()).abs() <= 5 * 2 * (2.0 ** -8 + 2.0 ** -11)).all()
    assert ((got_lse - lse).abs() <= 1e-5 * (1 + lse.abs())).all()


def test_three_axes_and_given_positions(blocks):
    """Positions of every axis as given, other rows than counts say left alone."""
    pool = blocks.BlockPool(10, 2, 64, 2, 5)
    other = blocks.BlockPool(10, 2, 64, 2, 5)
    rotary = blocks.netkv.Rotary(32, sections=[8, 12, 12])
    q, k, v = (rows(22, h, 64, torch.float16, h) for h in (4, 2, 2))
    pos = torch.randint(0, 1000, (3, 22), dtype=torch.int32, device="cuda")
    out, _ = pool.extend(q, k, v, [12, 8], rotary, positions=pos)
    turned = torch.empty_like(q)
    blocks.netkv.netkv_rotate(rotary, q, pos, turned)
    tk = torch.empty_like(k)
    blocks.netkv.netkv_rotate(rotary, k, pos, tk)
    other.append(tk, v, [12, 8])
    want, _ = other.attend_chunk(turned, [12, 8])
    torch.cuda.synchronize()
    # keys differ by one rounding to fp16 before their codes, and so codes by one step at most: 2^-7 of the
    # largest key of a block in a channel, scores by that times |q|_1 / 8 at most, which is below 6
    assert ((out[:20].float() - want[:20].float()).abs() <= 5 * math.expm1(2 * 6 * 5 * 2.0 ** -7)).all()
    assert torch.equal(pool.pages.tensors[1], other.pages.tensors[1])


def test_a_captured_step(blocks):
    """Append and attention of one step captured in a graph and replayed on new rows and lengths."""
    netkv = blocks.netkv
    pool = blocks.BlockPool(40, 2, 128, 3, 12)
    rotary = netkv.Rotary(64)
    q, k, v = (rows(60, h, 128, torch.bfloat16, h) for h in (8, 2, 2))
    pool.extend(q, k, v, [30, 20, 10], rotary)
    pool.reserve([8, 8, 8])
    off = torch.tensor([0, 3, 4, 6], dtype=torch.int64, device="cuda")
    start, length = pool.length.clone(), pool.length.clone()
    turned, out = torch.empty_like(q[:6]), torch.empty_like(q[:6])
    a, b, c = q[:6].clone(), k[:6].clone(), v[:6].clone()
    ws = torch.empty(netkv.netkv_attn_chunk_workspace_size(pool.pages, 6, 3, 8), dtype=torch.uint8, device="cuda")
    length += torch.tensor([3, 1, 2], dtype=torch.int32, device="cuda")

    def step():
        netkv.netkv_kv_append(pool.pages, b, c, off, start, pool.table, rotary, q=a, q_out=turned)
        netkv.netkv_attn_chunk(pool.pages, turned, off, length, pool.table, out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    a.copy_(q[10:16])
    b.copy_(k[10:16])
    c.copy_(v[10:16])
    off.copy_(torch.tensor([0, 1, 5, 6]))
    length.copy_(start + torch.tensor([1, 4, 1], dtype=torch.int32, device="cuda"))
    before = [x.clone() for x in pool.pages.tensors]
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (*pool.pages.tensors, turned, out)]
    for x, y in zip(pool.pages.tensors, before):
        x.copy_(y)
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, (*pool.pages.tensors, turned, out)))


def test_pages_past_four_gigabytes(blocks):
    """The same blocks at the end of a pool whose codes are past 32 bits, and in a small one."""
    netkv = blocks.netkv
    n, heads, kv_heads, dim, new = 1_200_000, 8, 2, 128, [70, 1]
    big = [torch.empty((n, kv_heads, 16, dim), dtype=torch.int8, device="cuda") for _ in "kv"] + \
        [torch.empty((n, kv_heads), device="cuda") for _ in "kv"]
    small = [x[-20:].clone().zero_() for x in big]
    for x in big:
        x[-20:] = 0
    q, k, v = (rows(71, h, dim, torch.bfloat16, h) for h in (heads, kv_heads, kv_heads))
    off = torch.tensor([0, 70, 71], dtype=torch.int64, device="cuda")
    length = torch.tensor(new, dtype=torch.int32, device="cuda")
    outs = []
    for codes, first in ((big, n - 20), (small, 0)):
        pages = netkv.KvPages(*codes)
        table = (torch.arange(20, dtype=torch.int32, device="cuda").flip(0) + first).view(2, 10).contiguous()
        turned, out = torch.empty_like(q), torch.empty_like(q)
        ws = torch.empty(netkv.netkv_attn_chunk_workspace_size(pages, 71, 2, heads), dtype=torch.uint8, device="cuda")
        netkv.netkv_kv_append(pages, k, v, off, None, table, netkv.Rotary(64), q=q, q_out=turned)
        netkv.netkv_attn_chunk(pages, turned, off, length, table, out, workspace=ws)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    for x, y in zip(big, small):
        assert torch.equal(x[-20:], y)
