"""Attention of new tokens over their sequences' 8-bit blocks, against its definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets, pool, tables  # noqa: E402

WEIGHT_UNIT = 2.0 ** -11   # softmax weights are fp16 in the second product


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


def call(netkv, pages, q, off, length, table, out, stream=None, **kw):
    size = netkv.netkv_attn_chunk_workspace_size(pages, q.shape[0], off.numel() - 1, q.shape[1])
    assert size > 0
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")  # no initial value
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    netkv.netkv_attn_chunk(pages, q, off, length, table, out, workspace=ws, status=status,
                           stream=stream, **kw)
    torch.cuda.synchronize()
    return int(status.item())


def check(netkv, new, held, heads, kv_heads, dim, dtype, fmt, seed=0, scale=None, pad=0, sharp=1.0,
          spread=False, garbage=True, lead=0, rows=None, only_heads=None, stream=None, spare=2):
    """held: tokens before the new ones (negative: fewer tokens than new rows).  lead: rows before the
    first sequence and after the last, which stay as they are."""
    n, group = len(new), heads // kv_heads
    total = [a + b for a, b in zip(new, held)]
    blocks = [-(-x // 16) for x in total]
    width = max(max(blocks), 1) + spare
    n_pages = sum(blocks) + 3
    k, v, ks, vs = pool(n_pages, kv_heads, dim, fmt, seed)
    g = torch.Generator().manual_seed(seed + 9)
    if spread:  # scales over many orders, some of them zero
        for s in (ks, vs):
            s *= torch.exp2(torch.randint(-24, 8, s.shape, generator=g).float()).cuda()
        vs[0], ks[min(1, n_pages - 1)] = 0, 0
    table = tables(blocks, width, n_pages, seed)
    if garbage:  # codes past the last token: the NaN of e4m3, the unused code of int8
        bad = 0x7F if fmt == "e4m3" else 0x80
        for i, x in enumerate(total):
            if x % 16:
                for c in (k, v):
                    c.view(torch.uint8)[int(table[i, x // 16]), :, x % 16:] = bad
    rows_all = sum(new) + 2 * lead
    wide = (torch.randn((rows_all, heads * dim + pad), generator=g) * sharp).to(dtype).cuda()
    q = wide[:, :heads * dim].unflatten(1, (heads, dim))
    if lead:
        q[:lead], q[-lead:] = math.nan, math.nan
    out = torch.full_like(wide, 5.0)
    got = out[:, :heads * dim].unflatten(1, (heads, dim))
    lse = torch.full((rows_all, heads), 5.0, device="cuda")
    status = call(netkv, netkv.KvPages(k, v, ks, vs), q, offsets(new) + lead, ints(total), table, got,
                  lse=lse, scale=scale, stream=stream)
    assert status == 0
    sc = dim ** -0.5 if scale is None else scale
    rng = np.random.default_rng(seed)
    at = lead
    for i, (a, x) in enumerate(zip(new, total)):
        pages = table[i, :blocks[i]].long()
        sel = np.arange(a) if rows is None or a <= rows else \
            np.unique(np.concatenate([[0, a - 1], rng.integers(0, a, rows)]))
        sel = torch.from_numpy(sel).cuda()
        see = torch.arange(x, device="cuda")[None] <= sel[:, None] + x - a
        for h in range(heads) if only_heads is None else only_heads:
            hk = h // group
            kh = (k[pages, hk].double() * ks[pages, hk].double()[:, None, None]).flatten(0, 1)[:x]
            vh = (v[pages, hk].double() * vs[pages, hk].double()[:, None, None]).flatten(0, 1)[:x]
            qh = q[at:at + a, h].double()[sel]
            if a == 0:
                continue
            if x == 0:
                o, z, weight, size = torch.zeros_like(qh), torch.full((len(sel),), -math.inf).cuda(), 0.0, 0.0
            else:
                o, z, _, weight, size = plain.attention(qh, kh, vh, sc, see)
            # a weight below fp16's smallest step is off by at most half of it, against a sum of at
            # least 1, times the largest value its block can hold
            slack = x * 2.0 ** -25 * float(vs[pages, hk].max()) * plain.TOP[fmt] if x else 0.0
            plain.close_out(got[at:at + a, h][sel], o, weight, size, dim, dtype, WEIGHT_UNIT, slack)
            plain.close_lse(lse[at:at + a, h][sel], z.double(), size, dim)
        at += a
    if lead:
        assert (got[:lead] == 5).all() and (got[-lead:] == 5).all()
        assert (lse[:lead] == 5).all() and (lse[-lead:] == 5).all()
    if pad:
        assert (out[:, heads * dim:] == 5).all()
    return got, lse


NEW = [1, 2, 0, 5, 16, 17, 1, 40, 3, 130]
HELD = [0, 0, 9, 11, 0, 127, 128, 300, 1000, 200]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (4, 4, 64), (7, 1, 128), (16, 2, 64),
                                                (3, 1, 64), (32, 1, 128), (300, 1, 64)])
def test_shapes(netkv, fmt, dtype, heads, kv_heads, dim):
    check(netkv, NEW, HELD, heads, kv_heads, dim, dtype, fmt, seed=heads, pad=16, lead=3)


@pytest.mark.parametrize("new,held", [([1], [0]), ([1], [511]), ([4], [500]), ([128], [0]), ([129], [0]),
                                      ([16], [112]), ([16], [113]), ([256], [256]), ([33], [4000])])
def test_one_sequence(netkv, new, held):
    check(netkv, new, held, 8, 1, 128, torch.bfloat16, "int8", seed=new[0])
    check(netkv, new, held, 2, 2, 64, torch.float16, "e4m3", seed=new[0])


@pytest.mark.parametrize("new,held,heads,kv_heads,dim", [
    ([600], [0], 4, 2, 128), ([513, 1, 700], [900, 2000, 0], 6, 2, 64), ([1000], [3000], 16, 2, 128),
    ([2000, 30, 1], [100, 3000, 777], 2, 1, 128)])
def test_longer_chunks(netkv, new, held, heads, kv_heads, dim):
    check(netkv, new, held, heads, kv_heads, dim, torch.bfloat16, "int8", rows=60, seed=5)
    check(netkv, new, held, heads, kv_heads, dim, torch.float16, "e4m3", rows=60, seed=6)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_long_context(netkv, fmt):
    """Few rows over a long axis, which is split and joined."""
    check(netkv, [5, 1], [70000, 40001], 16, 2, 128, torch.bfloat16, fmt, only_heads=[0, 7, 15])
    check(netkv, [9], [100000], 4, 4, 64, torch.float16, fmt, only_heads=[0, 3])


@pytest.mark.parametrize("n", [130, 700])
def test_many_sequences(netkv, n):
    """Ragged, with sequences without tokens and without rows."""
    rng = np.random.default_rng(n)
    new = (rng.integers(0, 4, n) * rng.integers(0, 9, n)).tolist()
    held = (rng.integers(0, 3, n) * rng.integers(0, 200, n)).tolist()
    check(netkv, new, held, 4, 2, 64, torch.bfloat16, "int8", seed=n, only_heads=[0, 3])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scales_and_sharp_scores(netkv, fmt, dtype):
    """Scales over 32 powers of two and zeros among them, and scores of which one takes all."""
    check(netkv, [3, 50, 200], [700, 300, 90], 8, 2, 128, dtype, fmt, spread=True, seed=2)
    check(netkv, [3, 50, 200], [700, 300, 90], 4, 2, 64, dtype, fmt, sharp=30.0, seed=3)
    check(netkv, [3, 50], [700, 300], 8, 1, 64, dtype, fmt, scale=1e-3, seed=4)


def test_more_rows_than_tokens(netkv):
    """Rows that see nothing give 0 and -inf."""
    check(netkv, [20, 1, 300, 5, 40], [-7, -1, -200, -5, 10], 4, 2, 64, torch.bfloat16, "int8")
    check(netkv, [20, 1, 300, 5, 40], [-7, -1, -200, -5, 10], 8, 1, 128, torch.float16, "e4m3")


@pytest.mark.parametrize("gone", [1, 2, 3, 9, 40])
def test_sequences_without_tokens_between_others(netkv, gone):
    """Many rows in a row that see nothing, in one run of the line and across runs."""
    new = [3, 1] + [2] * gone + [4, 1] + [1] * gone + [2]
    held = [50, 400] + [-2] * gone + [60, 200] + [-1] * gone + [30]
    check(netkv, new, held, 8, 1, 128, torch.bfloat16, "int8", seed=gone)
    check(netkv, new * 3, held * 3, 4, 4, 64, torch.float16, "e4m3", seed=gone)
    check(netkv, [300] * gone + [2], [-300] * gone + [40], 4, 2, 64, torch.float16, "int8", seed=gone)


@pytest.mark.parametrize("dim", [64, 128])
def test_absent_pages(netkv, dim):
    """Pages out of range hold no tokens: their block is not seen, ERANGE is said, and a row that sees
    nothing else gives 0 and -inf."""
    heads, kv_heads, new, held = 4, 2, [30, 20, 5], [300, 0, 100]
    total = [a + b for a, b in zip(new, held)]
    blocks = [-(-x // 16) for x in total]
    k, v, ks, vs = pool(sum(blocks) + 1, kv_heads, dim, "int8")
    table = tables(blocks, max(blocks), sum(blocks) + 1)
    gone = [(0, 0), (0, 7), (0, 20), (1, 0), (1, 1)] + [(2, b) for b in range(7)]
    for j, (i, b) in enumerate(gone):
        table[i, b] = (-1, sum(blocks) + 1, 2 ** 31 - 1, -2 ** 31)[j % 4]
    q = torch.randn((sum(new), heads, dim), device="cuda").half()
    out, lse = torch.full_like(q, 5), torch.full((sum(new), heads), 5.0, device="cuda")
    status = call(netkv, netkv.KvPages(k, v, ks, vs), q, offsets(new), ints(total), table, out, lse=lse)
    assert status == netkv.NETKV_DEV_ERANGE
    at = 0
    for i, (a, x) in enumerate(zip(new, total)):
        there = torch.tensor([(i, b) not in gone for b in range(blocks[i])]).repeat_interleave(16)[:x]
        pages = table[i, :blocks[i]].clamp(0, sum(blocks)).long()
        pages[~torch.tensor([(i, b) not in gone for b in range(blocks[i])])] = 0
        see = (torch.arange(x)[None] <= torch.arange(a)[:, None] + x - a) & there
        for h in range(heads):
            hk = h // 2
            kh = (k[pages, hk].double() * ks[pages, hk].double()[:, None, None]).flatten(0, 1)[:x].cpu()
            vh = (v[pages, hk].double() * vs[pages, hk].double()[:, None, None]).flatten(0, 1)[:x].cpu()
            o, z, _, weight, size = plain.attention(q[at:at + a, h].cpu().double(), kh, vh, dim ** -0.5, see)
            plain.close_out(out[at:at + a, h].cpu(), o, weight, size, dim, torch.float16, WEIGHT_UNIT,
                            x * 2.0 ** -25 * float(vs.max()) * 127)
            plain.close_lse(lse[at:at + a, h].cpu(), z, size, dim)
        at += a
    assert (out[30:50] == 0).all() and (lse[30:50] == -math.inf).all()


def test_bad_lengths_and_offsets(netkv):
    """A length past the table is cut and said; offsets that decrease or pass the rows have no rows."""
    k, v, ks, vs = pool(8, 1, 64, "int8")
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    q = torch.randn((12, 2, 64), device="cuda").bfloat16()
    pages = netkv.KvPages(k, v, ks, vs)
    want, got = torch.full_like(q, 5), torch.full_like(q, 5)
    assert call(netkv, pages, q, offsets([6, 6]), ints([64, 30]), table, want) == 0
    assert call(netkv, pages, q, offsets([6, 6]), ints([-1, 30]), table, got) == netkv.NETKV_DEV_ERANGE
    assert torch.equal(want, got)
    for off in ([6, 0, 6], [0, 6, 13]):
        got.fill_(5)
        assert call(netkv, pages, q, ints(off, torch.int64), ints([64, 30]), table, got) == netkv.NETKV_DEV_ERANGE
        lo, hi = (0, 6)
        other = torch.full_like(q, 5)
        seq = 1 if off[0] else 0
        call(netkv, pages, q, ints([lo, hi], torch.int64), ints([[64, 30][seq]]), table[seq:seq + 1].contiguous(), other)
        assert torch.equal(got[:6], other[:6]) and (got[6:] == 5).all()


@pytest.mark.parametrize("gap", [10, 18, 22])
@pytest.mark.parametrize("new,heads,kv_heads,dim", [(2, 2, 1, 64), (2, 16, 2, 128), (300, 8, 1, 128)])
def test_sinks(netkv, gap, new, heads, kv_heads, dim):
    """A sink 2^gap above the other tokens whose value is 0: what the others add comes to its full
    precision down to 2^-20 of the largest weight, and by 2^-31 of it for each token below."""
    n = 4096
    g = torch.Generator().manual_seed(gap)
    q = 0.02 * torch.randn((new, heads, dim), generator=g)
    q[..., 0] = 1.0
    q = q.half().cuda()
    pages = n // 16
    k = torch.randint(-127, 128, (pages, kv_heads, 16, dim), generator=g, dtype=torch.int8)
    v = torch.randint(64, 128, (pages, kv_heads, 16, dim), generator=g, dtype=torch.int8)
    ks, vs = torch.full((pages, kv_heads), 1 / 127), torch.full((pages, kv_heads), 1 / 127)
    k[..., 0] = 0
    k[0, :, 0], v[0, :, 0] = 0, 0
    k[0, :, 1:], v[0, :, 1:] = 0, 0
    k[0, :, 0, 0] = 127
    ks[0] = gap * math.log(2) / 127
    k, v, ks, vs = k.cuda(), v.cuda(), ks.cuda(), vs.cuda()
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    out, lse = torch.empty_like(q), torch.empty((new, heads), device="cuda")
    assert call(netkv, netkv.KvPages(k, v, ks, vs), q, offsets([new]), ints([n]), table, out, lse=lse,
                scale=1.0) == 0
    at = torch.tensor(sorted({0, new // 2, new - 1}), device="cuda")
    see = torch.arange(n, device="cuda")[None] <= at[:, None] + n - new
    for h in {0, heads - 1}:
        hk = h // (heads // kv_heads)
        kh = (k[:, hk].double() * ks[:, hk].double()[:, None, None]).flatten(0, 1)
        vh = (v[:, hk].double() * vs[:, hk].double()[:, None, None]).flatten(0, 1)
        o, z, _, weight, size = plain.attention(q[at, h].double(), kh, vh, 1.0, see)
        plain.close_out(out[at, h], o, weight, size, dim, torch.float16, WEIGHT_UNIT, n * 2.0 ** -31)
        plain.close_lse(lse[at, h], z, size, dim)


def test_nan_and_infinite_queries_stay_in_their_rows(netkv):
    new, held = [40, 3], [500, 700]
    k, v, ks, vs = pool(100, 2, 64, "int8")
    table = tables([34, 44], 50, 100)
    q = torch.randn((43, 8, 64), device="cuda").bfloat16()
    pages, off, length = netkv.KvPages(k, v, ks, vs), offsets(new), ints([540, 703])
    want, got = torch.empty_like(q), torch.empty_like(q)
    call(netkv, pages, q, off, length, table, want)
    bad = q.clone()
    bad[7, 3, 5], bad[41, 0, 0], bad[20, 6, 63] = math.nan, math.inf, -math.inf
    call(netkv, pages, bad, off, length, table, got)
    fine = torch.ones((43, 8), dtype=torch.bool, device="cuda")
    for r, h in ((7, 3), (41, 0), (20, 6)):
        fine[r, h] = False
    assert torch.equal(got[fine], want[fine])
    assert not torch.isfinite(got[7, 3]).any()


def test_wide_range_of_bf16_queries(netkv):
    """Small channels of a bf16 row beside large ones, and rows of very large and very small values."""
    g = torch.Generator().manual_seed(1)
    k, v, ks, vs = pool(40, 1, 128, "int8")
    table = torch.arange(40, dtype=torch.int32, device="cuda")[None]
    q = torch.randn((6, 2, 128), generator=g)
    q[0, :, 3] *= 2.0 ** 20
    q[1] *= 2.0 ** 100
    q[2] *= 2.0 ** -100
    q[3] = 0
    q[4] *= 2.0 ** -126
    k[:, :, :, 3] = 0
    q = q.bfloat16().cuda()
    out, lse = torch.empty_like(q), torch.empty((6, 2), device="cuda")
    pages = netkv.KvPages(k, v, ks, vs)
    assert call(netkv, pages, q, offsets([6]), ints([640]), table, out, lse=lse) == 0
    kh, vh = ((x.double() * s.double()[..., None, None]).flatten(0, 2) for x, s in ((k, ks), (v, vs)))
    see = torch.arange(640, device="cuda")[None] <= torch.arange(6, device="cuda")[:, None] + 634
    for h in range(2):
        for r in (0, 2, 3, 4):
            # a channel above 2^20 meets zeros: it adds nothing, and takes nothing from the others
            qr = q[r:r + 1, h].double()
            small = qr.clone()
            small[:, 3] = 0
            o, z, _, weight, _ = plain.attention(qr, kh, vh, 128 ** -0.5, see[r:r + 1])
            _, _, _, _, size = plain.attention(small, kh, vh, 128 ** -0.5, see[r:r + 1])
            plain.close_out(out[r:r + 1, h], o, weight, size, 128, torch.bfloat16, WEIGHT_UNIT, 1e-5)
            plain.close_lse(lse[r:r + 1, h], z, size, 128)
        # scores of 2^100: the largest takes all
        top = int((q[1, h].double() @ kh.T).masked_fill(~see[1], -math.inf).argmax())
        assert ((out[1, h].double() - vh[top]).abs() <= 2.0 ** -7 * vh[top].abs() + 1e-6).all()


def test_equal_calls_give_equal_bits(netkv):
    new, held = [70, 1, 4, 500], [3000, 20000, 900, 1000]
    total = [a + b for a, b in zip(new, held)]
    blocks = [-(-x // 16) for x in total]
    pages = netkv.KvPages(*pool(sum(blocks), 2, 128, "int8"))
    table = tables(blocks, max(blocks), sum(blocks))
    q = torch.randn((sum(new), 16, 128), device="cuda").bfloat16()
    runs = []
    for _ in range(4):
        out, lse = torch.full_like(q, 5), torch.empty(q.shape[:2], device="cuda")
        call(netkv, pages, q, offsets(new), ints(total), table, out, lse=lse)
        runs.append((out, lse))
    assert all(torch.equal(out, runs[0][0]) and torch.equal(lse, runs[0][1]) for out, lse in runs)


def test_a_graph_and_two_streams(netkv):
    """A captured call with other lengths at its replay, and calls on two streams with workspaces of
    their own."""
    new, held = [20, 3], [2000, 900]
    k, v, ks, vs = pool(300, 2, 64, "e4m3")
    pages, table = netkv.KvPages(k, v, ks, vs), tables([150, 150], 150, 300)
    q = torch.randn((23, 8, 64), device="cuda").half()
    off, length = offsets(new), ints([2020, 903])
    size = netkv.netkv_attn_chunk_workspace_size(pages, 23, 2, 8)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.full_like(q, 5) for _ in range(3)]
    netkv.netkv_attn_chunk(pages, q, off, length, table, outs[0], workspace=ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        netkv.netkv_attn_chunk(pages, q, off, length, table, outs[0], workspace=ws[0])
    off.copy_(offsets([1, 22]))
    length.copy_(ints([1500, 2400]))
    graph.replay()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            for _ in range(3):
                netkv.netkv_attn_chunk(pages, q, off, length, table, outs[1 + i], workspace=ws[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("n", [5, 5000])
def test_single_tokens_are_decode(netkv, n):
    """One new token a sequence: what netkv_attn_decode gives, up to both sides' rounding; among 5,000
    sequences some without tokens."""
    rng = np.random.default_rng(n)
    lengths = [1, 17, 300, 5000, 64] + (rng.integers(0, 3, n - 5) * rng.integers(1, 60, n - 5)).tolist()
    blocks = [-(-x // 16) for x in lengths]
    pages = netkv.KvPages(*pool(sum(blocks), 2, 128, "int8"))
    table = tables(blocks, max(blocks), sum(blocks))
    q = torch.randn((n, 16, 128), device="cuda").half()
    a, b, la, lb = torch.empty_like(q), torch.empty_like(q), *(torch.empty((n, 16), device="cuda") for _ in "ab")
    ws = torch.empty(netkv.netkv_attn_decode_workspace_size(pages, n, 16, max(blocks)),
                     dtype=torch.uint8, device="cuda")
    netkv.netkv_attn_decode(pages, q, ints(lengths), table, a, lse=la, workspace=ws)
    assert call(netkv, pages, q, offsets([1] * n), ints(lengths), table, b, lse=lb) == 0
    none = torch.tensor(lengths, device="cuda") == 0
    assert (b[none] == 0).all() and (lb[none] == -math.inf).all() and (la[none] == -math.inf).all()
    la[none], lb[none] = 0, 0
    # each: weights to 2^-11 and the output to 2^-11, of values up to 4 (codes of up to 127 at 1.25 / 127)
    assert ((a.float() - b.float()).abs() <= 4 * 2.0 ** -11 * 4).all()
    assert ((la - lb).abs() <= 1e-5 * (1 + la.abs())).all()
