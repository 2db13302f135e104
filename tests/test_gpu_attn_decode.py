"""Attention of one query a sequence over 8-bit blocks, against its definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_kv_blocks import FMT, ints, pool, tables  # noqa: E402

WEIGHT_UNIT = 2.0 ** -11  # the softmax weights may be rounded to fp16 for the second product


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


def call(netkv, pages, q, length, table, out, mass=None, same=False, stream=None, lse=None, **kw):
    n, heads = q.shape[:2]
    size = netkv.netkv_attn_decode_workspace_size(pages, n, heads, table.shape[1], mass is not None)
    assert size > 0
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda")  # no initial value
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mo = None
    if mass is not None:
        mo = mass if same else torch.full_like(mass, 7.0)
    torch.cuda.synchronize()
    netkv.netkv_attn_decode(pages, q, length, table, out, lse=lse, mass_in=mass, mass_out=mo,
                            workspace=ws, status=status, stream=stream, **kw)
    torch.cuda.synchronize()
    return mo, int(status.item())


def check(netkv, lengths, heads, kv_heads, dim, dtype, fmt, seed=0, mass=True, scale=None, pad=0,
          sharp=1.0, spread=False, width=None, garbage=True, same=False, stream=None):
    n, group = len(lengths), heads // kv_heads
    blocks = [-(-x // 16) for x in lengths]
    width = width or max(max(blocks), 1) + 2
    n_pages = sum(blocks) + 3
    k, v, ks, vs = pool(n_pages, kv_heads, dim, fmt, seed)
    g = torch.Generator().manual_seed(seed + 9)
    if spread:  # scales over many orders, some of them zero
        for s in (ks, vs):
            s *= torch.exp2(torch.randint(-24, 8, s.shape, generator=g).float()).cuda()
        vs[0] = 0
    table = tables(blocks, width, n_pages, seed)
    if garbage:  # codes past the last token: the NaN of e4m3, the unused code of int8
        bad = 0x7F if fmt == "e4m3" else 0x80
        for i, x in enumerate(lengths):
            if x % 16:
                for c in (k, v):
                    c.view(torch.uint8)[int(table[i, x // 16]), :, x % 16:] = bad
    wide = (torch.randn((n, heads * dim + pad), generator=g) * sharp).to(dtype).cuda()
    q = wide[:, :heads * dim].unflatten(1, (heads, dim))
    out = torch.full_like(wide, 5.0)
    got = out[:, :heads * dim].unflatten(1, (heads, dim))
    lse = torch.empty((n, heads), device="cuda")
    m0 = torch.rand((n, width), generator=g).cuda() if mass else None
    before = m0.clone() if mass else None
    length = ints(lengths)
    m1, status = call(netkv, netkv.KvPages(k, v, ks, vs), q, length, table, got, mass=m0, same=same,
                      lse=lse, scale=scale, stream=stream)
    assert status == 0
    sc = dim ** -0.5 if scale is None else scale
    kk, vv = plain.codes_value(k), plain.codes_value(v)
    ks64, vs64 = ks.cpu().double(), vs.cpu().double()
    for i, x in enumerate(lengths):
        pages = table[i, :blocks[i]].cpu().long()
        see = (torch.arange(blocks[i] * 16) < x).expand(group, -1)
        drawn, err = torch.zeros(blocks[i] * 16, dtype=torch.float64), 0.0
        for h in range(kv_heads):
            kh = (kk[pages, h] * ks64[pages, h][:, None, None]).flatten(0, 1)
            vh = (vv[pages, h] * vs64[pages, h][:, None, None]).flatten(0, 1)
            kh = torch.where(see[0][:, None], kh, torch.zeros_like(kh)) if x else kh
            vh = torch.where(see[0][:, None], vh, torch.zeros_like(vh)) if x else vh
            at = slice(h * group, (h + 1) * group)
            o, z, p, weight, size = plain.attention(q[i, at].cpu().double(), kh, vh, sc, see)
            # a weight below fp16's smallest step is off by at most half of it, against a sum
            # of at least 1, times the largest value its block can hold
            slack = x * 2.0 ** -25 * float(vs64[pages, h].max()) * plain.TOP[fmt] if x else 0.0
            plain.close_out(got[i, at].cpu(), o, weight, size, dim, dtype, WEIGHT_UNIT, slack)
            plain.close_lse(lse[i, at].cpu(), z, size, dim)
            drawn += p.sum(0)
            err = max(err, plain.score_error(size, dim))
        if mass:
            want = before[i, :blocks[i]].cpu().double() + drawn.view(-1, 16).sum(1)
            tol = (2 * err + 2.0 ** -18) * drawn.view(-1, 16).sum(1) + 2.0 ** -22 * want + 1e-30
            assert ((m1[i, :blocks[i]].cpu().double() - want).abs() <= tol).all()
            rest = m1[i, blocks[i]:]
            assert torch.equal(rest, before[i, blocks[i]:]) if same else bool((rest == 7).all())
    if pad:
        assert (out[:, heads * dim:] == 5).all()


LENGTHS = [0, 1, 15, 16, 17, 100, 128, 129, 1000]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads", [(16, 2), (1, 1), (7, 1), (8, 8), (9, 3), (18, 2), (32, 2), (40, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_heads_types_and_lengths(netkv, fmt, dtype, heads, kv_heads, dim):
    check(netkv, LENGTHS, heads, kv_heads, dim, dtype, fmt, seed=heads, pad=8)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("lengths", [[1], [16], [513], [5000], [40000], [70000, 3]])
def test_few_sequences(netkv, fmt, lengths):
    check(netkv, lengths, 16, 2, 128, torch.bfloat16, fmt, seed=1)


@pytest.mark.parametrize("n", [130, 700])
def test_many_ragged_sequences(netkv, n):
    rng = np.random.default_rng(n)
    lengths = np.where(rng.random(n) < 0.1, 0, np.exp(rng.normal(4.5, 1.2, n))).astype(int).tolist()
    check(netkv, lengths, 8, 1, 64, torch.float16, "int8", seed=n)
    check(netkv, lengths, 3, 3, 128, torch.bfloat16, "e4m3", seed=n, same=True)


@pytest.mark.parametrize("n,heads,kv_heads", [(6, 16, 2), (40, 8, 8), (700, 6, 3), (300, 60, 5)])
@pytest.mark.parametrize("width", [1, 31, 32, 33])
def test_short_tables(netkv, n, heads, kv_heads, width):
    """Tables at and next to the width up to which no segment is shared between runs."""
    rng = np.random.default_rng(width + n)
    lengths = np.where(rng.random(n) < 0.1, 0, rng.integers(1, width * 16 + 1, n)).tolist()
    lengths[0] = width * 16
    check(netkv, lengths, heads, kv_heads, 64, torch.bfloat16, "int8", seed=n, width=width)


@pytest.mark.parametrize("n,heads,kv_heads", [(620, 36, 3), (1900, 2, 1)])
@pytest.mark.parametrize("mass", [False, True])
def test_a_run_for_each_warp(netkv, n, heads, kv_heads, mass):
    """Enough segments that warps have runs of their own, which cut some of them."""
    rng = np.random.default_rng(n)
    lengths = np.exp(rng.normal(3.5, 1.5, n)).astype(int).clip(0, 4000)
    lengths[5] = 4000
    check(netkv, lengths.tolist(), heads, kv_heads, 128, torch.float16, "e4m3", seed=n, mass=mass)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_sharp_scores_and_spread_scales(netkv, fmt):
    """One token takes nearly all of a row's weight; scales of blocks orders apart."""
    check(netkv, [33, 400, 3000], 8, 2, 128, torch.bfloat16, fmt, sharp=20.0)
    check(netkv, [33, 400, 3000], 16, 1, 64, torch.float16, fmt, spread=True)
    check(netkv, [33, 400, 3000], 8, 1, 128, torch.bfloat16, fmt, scale=3.0, sharp=1e-3)


def test_large_and_small_queries(netkv):
    """bf16 queries beyond fp16's range either way."""
    check(netkv, [200], 8, 2, 128, torch.bfloat16, "int8", sharp=1e6, scale=1e-7)
    check(netkv, [200], 8, 2, 128, torch.bfloat16, "int8", sharp=1e-9, scale=1e8)


def test_without_mass_and_on_another_stream(netkv):
    s = torch.cuda.Stream()
    check(netkv, [70, 0, 900], 16, 2, 128, torch.bfloat16, "int8", mass=False, stream=s)
    check(netkv, [70, 0, 900], 16, 2, 128, torch.bfloat16, "int8", same=True, stream=s)


def test_bad_lengths_and_pages(netkv):
    """A page out of range counts as absent, a length past the table is cut; both are flagged,
    and the other sequences are as without them."""
    k, v, ks, vs = pool(12, 2, 64, "e4m3")
    pages = netkv.KvPages(k, v, ks, vs)
    q = torch.randn((4, 4, 64)).half().cuda()
    good = ints(range(12)).view(4, 3)
    want, got = torch.empty_like(q), torch.empty_like(q)
    m = torch.zeros((4, 3), device="cuda")
    assert call(netkv, pages, q, ints([48, 20, 33, 48]), good, want, mass=m)[1] == 0
    bad = good.clone()
    bad[1, 1] = 12
    bad[2, :] = -1
    m1, status = call(netkv, pages, q, ints([48, 20, 33, 49]), bad, got, mass=m)
    assert status == netkv.NETKV_DEV_ERANGE
    assert torch.equal(got[[0, 3]], want[[0, 3]]) and (got[2] == 0).all()
    assert (m1[2] == 0).all() and float(m1[1, 1]) == 0 and abs(float(m1[1, 0]) - 4) < 1e-4
    short = torch.empty_like(q)
    call(netkv, pages, q, ints([48, 16, 33, 48]), good, short)
    assert torch.equal(got[1], short[1])


def test_query_infinities_stay_in_their_head(netkv):
    k, v, ks, vs = pool(8, 1, 64, "int8")
    q = torch.randn((2, 8, 64)).bfloat16().cuda()
    pages, table, length = netkv.KvPages(k, v, ks, vs), ints(range(8)).view(2, 4), ints([64, 50])
    want, got = torch.empty_like(q), torch.empty_like(q)
    call(netkv, pages, q, length, table, want)
    q[0, 3, 5] = float("nan")
    q[1, 0, 0] = float("inf")
    call(netkv, pages, q, length, table, got)
    keep = torch.ones((2, 8), dtype=torch.bool)
    keep[0, 3] = keep[1, 0] = False
    assert torch.equal(got[keep.cuda()], want[keep.cuda()])
    assert got[0, 3].isnan().all() and not got[1, 0].float().isfinite().all()


def test_repeated_calls_give_the_same_bits(netkv):
    k, v, ks, vs = pool(600, 2, 128, "int8")
    q = torch.randn((3, 16, 128)).bfloat16().cuda()
    pages = netkv.KvPages(k, v, ks, vs)
    table, length = ints(range(600)).view(3, 200), ints([3200, 1500, 77])
    m = torch.zeros((3, 200), device="cuda")
    first = torch.empty_like(q)
    m1, _ = call(netkv, pages, q, length, table, first, mass=m)
    for _ in range(3):
        out = torch.empty_like(q)
        m2, _ = call(netkv, pages, q, length, table, out, mass=m)
        assert torch.equal(out, first) and torch.equal(m1[:, :5], m2[:, :5])


def test_pool_past_32_bits(netkv):
    heads, dim = 16, 128
    n_pages = (1 << 32) // (heads * 16 * dim) + 40
    k = torch.zeros((n_pages, heads, 16, dim), dtype=torch.int8, device="cuda")
    v, ks = torch.zeros_like(k), torch.ones((n_pages, heads), device="cuda")
    v[-1] = 3
    v[-2] = 5
    q = torch.randn((1, heads, dim)).half().cuda()
    out = torch.empty_like(q)
    call(netkv, netkv.KvPages(k, v, ks, ks.clone()), q, ints([24]),
         ints([n_pages - 1, n_pages - 2]).view(1, 2), out)
    assert ((out.float() - (16 * 3 + 8 * 5) / 24).abs() < 4e-3).all()


def test_refusals(netkv):
    k, v, ks, vs = pool(4, 2, 64, "int8")
    pages = netkv.KvPages(k, v, ks, vs)
    q = torch.zeros((1, 4, 64), dtype=torch.float16, device="cuda")
    out, length, table = torch.empty_like(q), ints([16]), ints([0]).view(1, 1)
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    go = lambda **kw: netkv.netkv_attn_decode(**{**dict(  # noqa: E731
        pages=pages, q=q, length=length, table=table, out=out, workspace=ws), **kw})
    go()
    m = torch.zeros((1, 1), device="cuda")
    for bad in (dict(workspace=None), dict(workspace=ws[:1]), dict(workspace=ws[1:]),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                dict(mass_in=m), dict(q=q[:, :3], out=out[:, :3])):
        with pytest.raises(netkv.NetKVError) as e:
            go(**bad)
        assert e.value.code == netkv.NETKV_EINVAL
    for bad in (dict(out=out.bfloat16()), dict(q=q.float()), dict(mass_out=m.double()),
                dict(length=length.long())):
        with pytest.raises(TypeError):
            go(**bad)
    for bad in (dict(out=out[:, :2]), dict(length=ints([1, 2])), dict(table=ints([0, 1]).view(2, 1)),
                dict(mass_out=torch.zeros((1, 2), device="cuda")), dict(lse=m)):
        with pytest.raises(ValueError):
            go(**bad)
    torch.cuda.synchronize()
    assert netkv.netkv_attn_decode_workspace_size(pages, 1, 3, 1) == 0
    go(q=q[:0], out=out[:0], length=length[:0], table=table[:0])


@pytest.mark.parametrize("n", [4097, 4500])
def test_thousands_of_sequences(netkv, n):
    """More sequences than a warp keeps sums of chunks for, some without tokens."""
    rng = np.random.default_rng(n)
    lengths = np.where(rng.random(n) < 0.3, 0, rng.integers(1, 60, n))
    lengths[[0, n // 2, n - 1]] = 700
    check(netkv, lengths.tolist(), 2, 1, 64, torch.float16, "int8", seed=n, width=44)
