"""Causal attention of packed prompts against its definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets  # noqa: E402


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


def strided(rows, heads, dim, dtype, pad, g, sharp=1.0):
    x = (torch.randn((rows, heads * dim + pad), generator=g) * sharp).to(dtype).cuda()
    return x[:, :heads * dim].unflatten(1, (heads, dim))


def check(netkv, lq, lk, heads, kv_heads, dim, dtype, seed=0, pad=0, sharp=1.0, scale=None,
          rows=None, lead=0, stream=None, only_heads=None):
    """lead: rows before the first sequence, filled with NaN, as are those after the last."""
    g = torch.Generator().manual_seed(seed)
    tq, tk = sum(lq) + 2 * lead, sum(lk) + 2 * lead
    q = strided(tq, heads, dim, dtype, pad, g, sharp)
    k = strided(tk, kv_heads, dim, dtype, 2 * pad, g)
    v = strided(tk, kv_heads, dim, dtype, pad, g)
    if lead:
        for x in (q, k, v):
            x[:lead] = math.nan
            x[-lead:] = math.nan
    out = torch.full((tq, heads * dim + pad), 5.0, dtype=dtype, device="cuda")
    got = out[:, :heads * dim].unflatten(1, (heads, dim))
    lse = torch.full((tq, heads), 5.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_off, k_off = offsets(lq) + lead, offsets(lk) + lead
    torch.cuda.synchronize()
    netkv.netkv_attn_prompt(q, k, v, q_off, k_off, got, lse=lse, scale=scale, status=status,
                            stream=stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    sc = dim ** -0.5 if scale is None else scale
    group = heads // kv_heads
    rng = np.random.default_rng(seed)
    dev = "cuda" if max(lk + [0]) > 1500 else "cpu"
    qa = ka = lead
    for a, b in zip(lq, lk):
        at = np.arange(a) if rows is None or a <= rows else \
            np.unique(np.concatenate([[0, a - 1], rng.integers(0, a, rows)]))
        sel = torch.from_numpy(at).to(dev)
        see = torch.arange(b, device=dev)[None] <= sel[:, None] + b - a
        for h in (range(heads) if only_heads is None else only_heads):
            pick = lambda x, n, s, hh: x[s:s + n, hh].to(dev).double()  # noqa: E731
            o, z, _, weight, size = plain.attention(
                pick(q, a, qa, h)[sel], pick(k, b, ka, h // group), pick(v, b, ka, h // group), sc, see)
            # weights of fp16 below its smallest step, against a sum of at least 1
            slack = b * 2.0 ** -24 * 6.0 if dtype == torch.float16 else 0.0
            plain.close_out(pick(got, a, qa, h)[sel].to(dtype), o, weight, size, dim, dtype,
                            plain.U[dtype], slack)
            plain.close_lse(lse[qa:qa + a, h].to(dev)[sel], z, size, dim)
        qa, ka = qa + a, ka + b
    if lead:
        assert (got[:lead] == 5).all() and (got[-lead:] == 5).all()
        assert (lse[:lead] == 5).all() and (lse[-lead:] == 5).all()
    if pad:
        assert (out[:, heads * dim:] == 5).all()


LENGTHS = [1, 0, 2, 16, 63, 64, 65, 127, 128, 129, 200, 257, 300]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (1, 1), (7, 1), (2, 2), (3, 3), (8, 1)])
@pytest.mark.parametrize("dim", [64, 128])
def test_whole_prompts(netkv, dtype, heads, kv_heads, dim):
    check(netkv, LENGTHS, LENGTHS, heads, kv_heads, dim, dtype, seed=heads, pad=8, lead=3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_cached_prefixes_and_empty_rows(netkv, dtype, dim):
    """More keys than rows (a prefix), no keys at all, and fewer keys than rows: the rows that
    see nothing give 0 and -inf."""
    lq = [1, 1, 5, 40, 128, 130, 300, 7, 33, 200, 0, 300]
    lk = [1, 400, 133, 300, 256, 131, 1000, 0, 10, 199, 50, 20]
    check(netkv, lq, lk, 4, 2, dim, dtype, seed=dim, pad=16, lead=1)


@pytest.mark.parametrize("n", [1, 31, 64, 96, 128, 160, 255, 256, 384, 385, 511, 640, 1000])
def test_single_prompts(netkv, n):
    check(netkv, [n], [n], 2, 1, 128, torch.bfloat16, seed=n)
    check(netkv, [n], [n], 3, 1, 64, torch.float16, seed=n)


def test_many_short_prompts(netkv):
    rng = np.random.default_rng(0)
    lq = rng.integers(0, 40, 300).tolist()
    lk = [a + int(b) for a, b in zip(lq, rng.integers(0, 30, 300))]
    check(netkv, lq, lk, 2, 2, 64, torch.bfloat16, lead=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv_heads", [(64, 8), (63, 9)])
@pytest.mark.parametrize("dim", [64, 128])
def test_more_items_than_the_card_takes_at_once(netkv, dtype, heads, kv_heads, dim):
    """Even and odd groups, enough row blocks that blocks of the grid take several: ordered by
    their keys, with prefixes, empty rows and empty sequences among them."""
    lq = [300, 1, 0, 700, 128, 257, 40, 900, 129, 5]
    lk = [300, 500, 20, 1100, 100, 257, 0, 900, 1000, 5]
    pick = sorted({0, 1, heads // kv_heads - 1, heads // 2, heads - 2, heads - 1})
    check(netkv, lq, lk, heads, kv_heads, dim, dtype, seed=dim + heads, pad=8, lead=2,
          only_heads=pick, rows=60)


@pytest.mark.parametrize("heads,kv_heads", [(16, 2), (15, 3)])
def test_more_sequences_than_are_ordered(netkv, heads, kv_heads):
    """More than 128 sequences, each with a few row blocks or less."""
    rng = np.random.default_rng(heads)
    lq = rng.integers(0, 300, 150).tolist()
    lk = [a + int(b) for a, b in zip(lq, rng.integers(0, 200, 150))]
    check(netkv, lq, lk, heads, kv_heads, 64, torch.bfloat16, only_heads=[0, heads - 1], rows=20)


def test_one_long_prompt_of_many_items(netkv):
    check(netkv, [20000], [20000], 16, 2, 128, torch.bfloat16, rows=40, only_heads=[0, 7, 8, 15])
    check(netkv, [16000], [20000], 15, 5, 128, torch.float16, rows=40, only_heads=[0, 3, 14])


def test_no_keys_at_all(netkv):
    """Rows without any key row in the call: zeros and -inf."""
    q = torch.randn((300, 4, 128)).bfloat16().cuda()
    k = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 5.0), torch.full((300, 4), 5.0, device="cuda")
    netkv.netkv_attn_prompt(q, k, k, offsets([300]), offsets([0]), out, lse=lse)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()


def test_long_prompts(netkv):
    check(netkv, [9000, 2500], [9000, 4000], 4, 1, 128, torch.bfloat16, rows=40)
    check(netkv, [40000], [40000], 2, 1, 64, torch.float16, rows=40)
    check(netkv, [300], [131072], 2, 1, 128, torch.bfloat16, rows=30)


def test_sharp_and_growing_scores(netkv):
    """Scores of hundreds, where one key takes a row's weight, and other scales."""
    check(netkv, [700, 129], [700, 400], 2, 1, 128, torch.bfloat16, sharp=30.0)
    check(netkv, [700, 129], [700, 400], 2, 1, 64, torch.float16, sharp=10.0)
    check(netkv, [300], [300], 2, 1, 128, torch.bfloat16, scale=1e-6)
    check(netkv, [300], [300], 2, 1, 128, torch.float16, scale=2.5)


def test_growing_maximum(netkv):
    """Keys whose scores grow along the row, so that the running maximum changes at every key."""
    n, dim = 1000, 128
    for dtype, step in ((torch.bfloat16, 0.05), (torch.float16, 0.5)):
        q = torch.zeros((n, 2, dim))
        q[..., 0] = 1.0
        k = torch.zeros((n, 1, dim))
        k[:, 0, 0] = torch.arange(n) * step
        v = torch.randn((n, 1, dim), generator=torch.Generator().manual_seed(1))
        q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
        out, off = torch.empty_like(q), offsets([n])
        netkv.netkv_attn_prompt(q, k, v, off, off, out, scale=1.0)
        torch.cuda.synchronize()
        see = torch.ones((n, n), dtype=torch.bool).tril()
        o, _, _, w, size = plain.attention(q[:, 0].cpu().double(), k[:, 0].cpu().double(),
                                           v[:, 0].cpu().double(), 1.0, see)
        for h in (0, 1):
            plain.close_out(out[:, h].cpu(), o, w, size, dim, dtype, plain.U[dtype], n * 2.0 ** -22)


def test_infinities_outside_a_sequence(netkv):
    """A neighbour of infinities and NaN in a packed batch reaches nothing."""
    dim = 128
    lq = [70, 130, 50]
    g = torch.Generator().manual_seed(2)
    q, k, v = (strided(sum(lq), h, dim, torch.bfloat16, 0, g).contiguous() for h in (2, 1, 1))
    off = offsets(lq)
    want, got = torch.empty_like(q), torch.empty_like(q)
    netkv.netkv_attn_prompt(q, k, v, off, off, want)
    for x in (q, k, v):
        x[70:200] = math.nan
        x[75:80] = math.inf
    netkv.netkv_attn_prompt(q, k, v, off, off, got)
    torch.cuda.synchronize()
    assert torch.equal(got[:70], want[:70]) and torch.equal(got[200:], want[200:])
    assert got[70:200].isnan().any()


def test_query_nan_stays_in_its_row(netkv):
    dim, n = 64, 300
    g = torch.Generator().manual_seed(2)
    q, k, v = (strided(n, h, dim, torch.float16, 0, g).contiguous() for h in (2, 1, 1))
    off = offsets([n])
    want, got = torch.empty_like(q), torch.empty_like(q)
    netkv.netkv_attn_prompt(q, k, v, off, off, want)
    q[17, 1] = math.nan
    q[200, 0, 3] = math.inf
    netkv.netkv_attn_prompt(q, k, v, off, off, got)
    torch.cuda.synchronize()
    keep = torch.ones((n, 2), dtype=torch.bool, device="cuda")
    keep[17, 1] = keep[200, 0] = False
    assert torch.equal(got[keep], want[keep]) and got[17, 1].isnan().all()


def test_streams_no_lse_and_repeats(netkv):
    s = torch.cuda.Stream()
    check(netkv, [300, 10], [300, 20], 4, 2, 128, torch.bfloat16, stream=s)
    g = torch.Generator().manual_seed(2)
    q, k, v = (strided(500, h, 128, torch.bfloat16, 0, g).contiguous() for h in (4, 2, 2))
    off = offsets([500])
    a, b = torch.empty_like(q), torch.empty_like(q)
    netkv.netkv_attn_prompt(q, k, v, off, off, a)
    netkv.netkv_attn_prompt(q, k, v, off, off, b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_bad_offsets(netkv):
    """Offsets that decrease or pass the rows: flagged, the other sequences as without them."""
    g = torch.Generator().manual_seed(2)
    q, k, v = (strided(100, h, 64, torch.float16, 0, g).contiguous() for h in (2, 1, 1))
    for off in ([0, 30, 20, 100], [0, 30, 101, 101], [0, 30, 1 << 40, 100]):
        want, got = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        good = offsets([30])
        netkv.netkv_attn_prompt(q, k, v, good, good, want)
        o = ints(off, torch.int64)
        netkv.netkv_attn_prompt(q, k, v, o, o, got, status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == netkv.NETKV_DEV_ERANGE
        assert torch.equal(got[:20], want[:20])


def test_refusals(netkv):
    z = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")  # noqa: E731
    q, k, v, out, off = z(4, 2, 64), z(4, 1, 64), z(4, 1, 64), z(4, 2, 64), offsets([4])
    go = lambda **kw: netkv.netkv_attn_prompt(**{**dict(  # noqa: E731
        q=q, k=k, v=v, q_off=off, k_off=off, out=out), **kw})
    go()
    narrow = dict(q=z(4, 2, 32), k=z(4, 1, 32), v=z(4, 1, 32), out=z(4, 2, 32))
    odd = z(4 * 128 + 8)[4:-4].view(4, 2, 64)
    for bad in (dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), narrow,
                dict(q=z(4, 3, 64), out=z(4, 3, 64), k=z(4, 2, 64), v=z(4, 2, 64)),
                dict(q=odd), dict(out=odd)):
        with pytest.raises(netkv.NetKVError) as e:
            go(**bad)
        assert e.value.code == netkv.NETKV_EINVAL
    for bad in (dict(k=k.bfloat16()), dict(q=q.float()), dict(lse=z(4, 2)), dict(q_off=off.int())):
        with pytest.raises(TypeError):
            go(**bad)
    for bad in (dict(v=z(3, 1, 64)), dict(out=z(3, 2, 64)), dict(k_off=offsets([2, 2])),
                dict(q=z(4, 64, 2).transpose(1, 2)), dict(lse=torch.zeros((2, 4), device="cuda"))):
        with pytest.raises(ValueError):
            go(**bad)
    torch.cuda.synchronize()
    go(q=q[:0], out=out[:0], q_off=offsets([0]))
