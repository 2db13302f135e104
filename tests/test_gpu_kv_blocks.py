"""8-bit KV blocks: rows into blocks and back, and eviction by attention weight, value for value
against the definitions."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402

FMT = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


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


def ints(x, dtype=torch.int32):
    return torch.tensor(list(x), dtype=dtype, device="cuda")


def offsets(counts):
    return ints(np.concatenate([[0], np.cumsum(counts)]).tolist(), torch.int64)


def pool(n_pages, heads, dim, fmt, seed=0):
    """Pages with codes in every place, and scales."""
    g = torch.Generator().manual_seed(seed)
    top = plain.TOP[fmt]

    def codes():
        x = (torch.randn((n_pages, heads, 16, dim), generator=g) * top / 3).clamp(-top, top)
        return (x.round() if fmt == "int8" else x).to(FMT[fmt]).cuda()

    def scales():
        return (0.25 + torch.rand((n_pages, heads), generator=g)).cuda() / top

    return codes(), codes(), scales(), scales()


def tables(blocks, width, n_pages, seed=0):
    rng = np.random.default_rng(seed)
    pages = rng.permutation(n_pages)[:sum(blocks)]
    t = np.full((len(blocks), width), -1, np.int32)
    at = 0
    for i, b in enumerate(blocks):
        t[i, :b] = pages[at:at + b]
        at += b
    return torch.from_numpy(t).cuda()


def check_store(netkv, held, new, heads, dim, fmt, dtype, seed=0, special=None, stream=None,
                pad=0):
    total = sum(new)
    blocks = [-(-(a + b) // 16) for a, b in zip(held, new)]
    width, n_pages = max(blocks) + 1, sum(blocks) + 3
    k, v, ks, vs = pool(n_pages, heads, dim, fmt, seed)
    table = tables(blocks, width, n_pages, seed)
    g = torch.Generator().manual_seed(seed + 1)
    wide = torch.randn((2, max(total, 1), heads * dim + pad), generator=g) * torch.exp(
        torch.randn((2, max(total, 1), 1), generator=g))
    wide = wide.to(dtype)
    if special is not None:
        special(wide)
    wide = wide.cuda()
    rows = wide[:, :total, :heads * dim].unflatten(2, (heads, dim))
    old = [x.clone() for x in (k, v, ks, vs)]
    pages = netkv.KvPages(k, v, ks, vs)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    start = ints(held)
    torch.cuda.synchronize()
    netkv.netkv_kv_store(pages, rows[0], rows[1], offsets(new), start, table, status=status,
                         stream=stream)
    torch.cuda.synchronize()
    want = [plain.codes_value(x).float().numpy() if x.dim() == 4 else x.cpu().numpy().copy()
            for x in old]
    host = rows.float().cpu().numpy()
    at = 0
    for i, (a, b) in enumerate(zip(held, new)):
        done = 0
        while done < b:
            pos = a + done
            lead, page = pos % 16, int(table[i, pos // 16])
            n = min(16 - lead, b - done)
            for h in range(heads):
                for which in (0, 1):
                    c, s = plain.store_block(want[which][page, h], want[2 + which][page, h], lead,
                                             host[which, at + done:at + done + n, h], fmt)
                    want[which][page, h], want[2 + which][page, h] = c, s
            done += n
        at += b
    for got, exp in zip((k, v), want[:2]):
        assert np.array_equal(plain.codes_value(got).float().numpy(), exp)
    for got, exp in zip((ks, vs), want[2:]):
        assert np.array_equal(got.cpu().numpy(), exp)
    return pages, table, int(status.item())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,heads", [(128, 2), (64, 3), (128, 1), (64, 8)])
def test_store_fresh_and_merged_blocks(netkv, fmt, dtype, dim, heads):
    held = [0, 0, 0, 5, 16, 15, 31, 1, 40, 0]
    new = [1, 16, 33, 3, 1, 1, 20, 15, 0, 0]
    assert check_store(netkv, held, new, heads, dim, fmt, dtype, seed=dim + heads, pad=24)[2] == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_store_many_sequences(netkv, fmt):
    """More sequences than one step of the search counts, some without rows."""
    rng = np.random.default_rng(5)
    held = rng.integers(0, 40, 300).tolist()
    new = (rng.integers(0, 3, 300) * rng.integers(1, 20, 300)).tolist()
    assert check_store(netkv, held, new, 1, 64, fmt, torch.bfloat16, seed=3)[2] == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_store_special_values(netkv, fmt):
    """Zeros, tiny values, infinities and NaN: zeros in their place, the status word set."""
    def special(x):
        x[:, 0:16] = 0
        x[:, 16:32] = 1e-38
        x[0, 40] = float("inf")
        x[1, 41] = float("nan")
        x[1, 48:64] = float("nan")
    status = check_store(netkv, [0, 7], [70, 30], 2, 64, fmt, torch.bfloat16, special=special)[2]
    assert status == netkv.NETKV_DEV_EDOMAIN


def test_store_one_token_after_another(netkv):
    """A block filled token by token holds every token to half a step of its last scale, plus
    half a step for each time the scale grew."""
    dim, heads = 64, 2
    k, v, ks, vs = pool(2, heads, dim, "int8")
    pages = netkv.KvPages(k, v, ks, vs)
    rows = torch.randn((2, 20, heads, dim)).to(torch.bfloat16).cuda()
    table = ints([1, 0]).view(1, 2)
    grew = torch.zeros(2, 2, heads)
    last = None
    for t in range(20):
        netkv.netkv_kv_store(pages, rows[0, t:t + 1], rows[1, t:t + 1], offsets([1]), ints([t]), table)
        now = torch.stack([ks[[1, 0]], vs[[1, 0]]]).cpu()
        if last is not None:
            grew += now > last
        last = now
    back = torch.zeros_like(rows)
    netkv.netkv_kv_load(pages, back[0], back[1], offsets([20]), ints([0]), table)
    err = (back.float() - rows.float()).abs().cpu()
    for w in range(2):
        for t in range(20):
            step = last[w, t // 16] * (0.5 + 0.5 * grew[w, t // 16])
            tol = step[:, None] + 2.0 ** -8 * rows[w, t].float().abs().cpu() + 1e-6
            assert (err[w, t] <= tol * 1.01).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,heads", [(128, 2), (64, 5)])
def test_load(netkv, fmt, dtype, dim, heads):
    start, count = [0, 3, 16, 0, 47, 9], [1, 30, 16, 0, 2, 100]
    blocks = [-(-(a + b) // 16) for a, b in zip(start, count)]
    k, v, ks, vs = pool(sum(blocks) + 2, heads, dim, fmt, 7)
    table = tables(blocks, max(blocks), sum(blocks) + 2, 7)
    out = torch.full((2, sum(count) + 1, heads * dim + 16), 9.0, dtype=dtype, device="cuda")
    rows = out[:, :sum(count), :heads * dim].unflatten(2, (heads, dim))
    netkv.netkv_kv_load(netkv.KvPages(k, v, ks, vs), rows[0], rows[1], offsets(count), ints(start),
                        table)
    torch.cuda.synchronize()
    at = 0
    for i, (a, b) in enumerate(zip(start, count)):
        for t in range(a, a + b):
            page = int(table[i, t // 16])
            for got, codes, scale in ((rows[0], k, ks), (rows[1], v, vs)):
                want = (codes[page, :, t % 16].cpu().float() * scale[page].cpu()[:, None]).to(dtype)
                assert torch.equal(got[at].cpu(), want)
            at += 1
    assert (out[:, -1] == 9).all() and (out[:, :, heads * dim:] == 9).all()


def test_blocks_on_another_stream_and_past_32_bits(netkv):
    """A pool whose codes pass 2^32 bytes, written and read at its end, on a stream of its own."""
    heads, dim = 16, 128
    n_pages = (1 << 32) // (heads * 16 * dim) + 40
    k = torch.zeros((n_pages, heads, 16, dim), dtype=torch.int8, device="cuda")
    ks = torch.zeros((n_pages, heads), device="cuda")
    rows = torch.randn((35, heads, dim), device="cuda").half()
    v, vs = k.clone(), ks.clone()
    table = ints([n_pages - 1, 0, n_pages - 2]).view(1, 3)
    back = torch.zeros((2,) + rows.shape, dtype=torch.float16, device="cuda")
    pages = netkv.KvPages(k, v, ks, vs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    off, start = offsets([35]), ints([0])
    torch.cuda.synchronize()
    netkv.netkv_kv_store(pages, rows, rows * 2, off, start, table, stream=s)
    netkv.netkv_kv_load(pages, back[0], back[1], off, start, table, stream=s)
    s.synchronize()
    for got, src in ((back[0], rows), (back[1], rows * 2)):
        x = src.float().cpu().numpy()
        for at in range(0, 35, 16):
            for h in range(heads):
                n = min(16, 35 - at)
                codes, scale = plain.store_block(np.zeros((16, dim)), 0, 0, x[at:at + n, h], "int8")
                want = torch.from_numpy(codes[:n] * scale).half()
                assert torch.equal(got[at:at + n, h].cpu(), want)
    assert k[1:-2].view(torch.int64).count_nonzero() == 0


def test_bad_pages_offsets_and_tables(netkv):
    """Page numbers, offsets and tables out of range: flagged, and nothing else is touched."""
    k, v, ks, vs = pool(8, 2, 64, "int8")
    old = [x.clone() for x in (k, v, ks, vs)]
    pages = netkv.KvPages(k, v, ks, vs)
    rows = torch.ones((40, 2, 64), dtype=torch.float16, device="cuda")

    def call(off, start, table, load=False):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        f = netkv.netkv_kv_load if load else netkv.netkv_kv_store
        out = [rows.clone(), rows.clone()]
        f(pages, out[0], out[1], ints(off, torch.int64), ints(start), ints(table).view(len(start), -1),
          status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == netkv.NETKV_DEV_ERANGE
        return out

    call([0, 16], [0], [8])
    call([0, 16], [0], [-1])
    call([0, 41], [0], [0, 1, 2])          # past the rows
    call([9, 0], [0], [0])                 # decreasing
    call([0, 16], [48], [0, 1, 2])         # past the table
    call([0, 3], [-1], [0, 1])             # a start of 2^32 - 1
    for x, y in zip((k, v, ks, vs), old):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    out = call([0, 20], [0], [3, 9], load=True)
    assert (out[0][16:20] == 0).all() and (out[0][20:] == 1).all()
    assert torch.equal(out[0][:16].cpu(), (k[3].cpu().float() * ks[3].cpu()[:, None, None]).half().permute(1, 0, 2))


def test_move_refusals(netkv):
    k, v, ks, vs = pool(4, 2, 64, "int8")
    pages = netkv.KvPages(k, v, ks, vs)
    r = torch.zeros((4, 2, 64), dtype=torch.float16, device="cuda")
    off, start, table = offsets([4]), ints([0]), ints([0]).view(1, 1)
    go = netkv.netkv_kv_store
    for bad in (r.float(), r.bfloat16()):
        with pytest.raises(TypeError):
            go(pages, r, bad, off, start, table)
    for bad in (r[:3], r[:, :1], torch.zeros((4, 64, 2), dtype=torch.float16, device="cuda")):
        with pytest.raises(ValueError):
            go(pages, r, bad, off, start, table)
    with pytest.raises(TypeError):
        go(pages, r, r, off.int(), start, table)
    with pytest.raises(TypeError):
        go(pages, r, r, off, start.float(), table)
    with pytest.raises(ValueError):
        go(pages, r, r, off, start, ints([0, 1]).view(2, 1))
    shifted = torch.zeros(4 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(4, 2, 64)
    odd = torch.zeros((4, 2 * 64 + 4), dtype=torch.float16, device="cuda")[:, :128].unflatten(1, (2, 64))
    for bad in (shifted, odd):
        with pytest.raises(netkv.NetKVError) as e:
            go(pages, r, bad, off, start, table)
        assert e.value.code == netkv.NETKV_EINVAL
    with pytest.raises(TypeError):
        netkv.KvPages(k.float(), v.float(), ks, vs)
    with pytest.raises(ValueError):
        netkv.KvPages(k[:, :, :8], v[:, :, :8], ks, vs)
    with pytest.raises(ValueError):
        netkv.KvPages(k, v, ks[:3], vs)
    with pytest.raises(netkv.NetKVError):
        go(netkv.KvPages(k[..., :32].contiguous(), v[..., :32].contiguous(), ks, vs),
           r[..., :32].contiguous(), r[..., :32].contiguous(), off, start, table)
    go(pages, r[:0], r[:0], offsets([0]), start, table)  # no rows: nothing to do


# ---------------------------------------------------------------- eviction
def check_evict(netkv, lengths, width, budget, sink, recent, mass, seed=0):
    n = len(lengths)
    rng = np.random.default_rng(seed)
    table = rng.permutation(n * width).astype(np.int32).reshape(n, width)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    to, fr = (torch.full((n, width), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    mo = torch.full((n, width), 77.0, device="cuda")
    lo, nf = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    netkv.netkv_kv_evict(dev(table), ints(lengths), dev(mass), ints(budget), sink, recent, to, lo,
                         mo, fr, nf, status=status)
    torch.cuda.synchronize()
    for i in range(n):
        t, m, length, gone = plain.evict(lengths[i], table[i].tolist(), mass[i].tolist(),
                                         budget[i], sink, recent)
        assert to[i].tolist() == t + [-1] * (width - len(t))
        assert np.array_equal(mo[i].cpu().numpy(), np.float32(m + [0.0] * (width - len(m))),
                              equal_nan=True)
        assert int(lo[i]) == length and int(nf[i]) == len(gone)
        assert fr[i].tolist() == gone + [-1] * (width - len(gone))
    assert int(status.item()) == 0


@pytest.mark.parametrize("width", [1, 2, 31, 512, 513, 1500, 4097])
@pytest.mark.parametrize("sink,recent", [(0, 1), (4, 16), (1, 600)])
def test_evict(netkv, width, sink, recent):
    rng = np.random.default_rng(width + recent)
    lengths = [width * 16, width * 16 - 15, 0, 1, max(1, width * 8), width * 16 - 3]
    budget = [max(1, width // 2), 1, 3, 1, width, max(1, width * 3 // 4)]
    mass = np.exp(3 * rng.standard_normal((6, width))).astype(np.float32)
    check_evict(netkv, lengths, width, budget, sink, recent, mass)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "special", "negative", "close"])
def test_evict_ties_and_special_weights(netkv, kind):
    rng = np.random.default_rng(4)
    width = 1300
    mass = {"equal": np.ones((3, width)), "few": rng.integers(0, 3, (3, width)),
            "zeros": np.where(rng.random((3, width)) < 0.5, -0.0, 0.0),
            "special": rng.choice([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-45, 3e38], (3, width)),
            "negative": rng.standard_normal((3, width)),
            "close": 1 + np.arange(3 * width).reshape(3, width) % 97 * 2.0 ** -23}[kind]
    check_evict(netkv, [width * 16] * 3, width, [700, 20, 1299], 3, 5, mass.astype(np.float32))


@pytest.mark.parametrize("width", [8192, 8193, 20001])
def test_evict_long_tables(netkv, width):
    """Rows at and past what one block of threads holds at a time."""
    rng = np.random.default_rng(width)
    mass = rng.choice(np.exp(rng.standard_normal(width // 3)), (3, width)).astype(np.float32)
    check_evict(netkv, [width * 16, width * 16 - 9, 77], width, [width // 2, 30, 9], 4, 16, mass)


def test_evict_refusals_and_long_lengths(netkv):
    t = ints(range(4)).view(1, 4)
    m = torch.ones((1, 4), device="cuda")
    one = ints([1])
    to, fr, mo = torch.empty_like(t), torch.empty_like(t), torch.empty_like(m)
    lo, nf = torch.empty_like(one), torch.empty_like(one)
    call = lambda *a, **k: netkv.netkv_kv_evict(*a, **k)  # noqa: E731
    for bad in (lambda: call(t, one, m, one, 0, 0, to, lo, mo, fr, nf),
                lambda: call(t, one, m, one, 0, 1, t, lo, mo, fr, nf),
                lambda: call(t, one, m, one, 0, 1, to, lo, m, fr, nf),
                lambda: call(t, one, m, one, 0, 1, to, lo, mo, to, nf)):
        with pytest.raises(netkv.NetKVError) as e:
            bad()
        assert e.value.code == netkv.NETKV_EINVAL
    with pytest.raises(ValueError):
        call(t, one, m, one, 0, 1, to[:, :3], lo, mo, fr, nf)
    with pytest.raises(TypeError):
        call(t, one, m.double(), one, 0, 1, to, lo, mo, fr, nf)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call(t, ints([65]), m, ints([2]), 1, 1, to, lo, mo, fr, nf, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == netkv.NETKV_DEV_ERANGE
    assert to[0].tolist() == [0, 3, -1, -1] and int(lo[0]) == 32
    assert fr[0].tolist() == [1, 2, -1, -1]
