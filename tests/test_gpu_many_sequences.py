"""Calls with thousands of sequences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_kv_blocks import check_store, ints, offsets, pool, tables  # noqa: E402


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


@pytest.mark.parametrize("n,at", [(9000, 8990), (9000, 5000), (9000, 100), (20000, 19999)])
@pytest.mark.parametrize("which", ["q", "k"])
def test_bad_prompt_offsets_far_back(netkv, n, at, which):
    """One bad pair among thousands of sequences, most of them empty: flagged, every time."""
    rng = np.random.default_rng(n)
    count = (rng.random(n) < 0.2).astype(np.int64)
    count[at - 1:at + 1] = 1
    off = np.concatenate([[0], np.cumsum(count)])
    rows = int(off[-1])
    bad = off.copy()
    bad[at] += 2 if at + 1 < n else rows  # the next pair decreases, or this one passes the rows
    q = torch.ones((rows, 2, 64), dtype=torch.float16, device="cuda")
    k = torch.ones((rows, 1, 64), dtype=torch.float16, device="cuda")
    good, wrong = ints(off.tolist(), torch.int64), ints(bad.tolist(), torch.int64)
    for k_off, q_off, want in ((good, good, 0),
                               (wrong if which == "k" else good, wrong if which == "q" else good,
                                netkv.NETKV_DEV_ERANGE)):
        for _ in range(3):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            netkv.netkv_attn_prompt(q, k, k, q_off, k_off, torch.empty_like(q), status=status)
            torch.cuda.synchronize()
            assert int(status.item()) == want


def test_what_follows_a_batch_without_tokens(netkv):
    """Rows and lse of empty sequences are there for whatever comes next in the stream, block
    weights or not."""
    n, heads, dim = 30000, 16, 128
    k, s = torch.zeros((2, 2, 16, dim), dtype=torch.int8, device="cuda"), torch.ones((2, 2), device="cuda")
    pages = netkv.KvPages(k, k.clone(), s, s.clone())
    q = torch.ones((n, heads, dim), dtype=torch.bfloat16, device="cuda")
    length, table = ints([0] * n), torch.zeros((n, 40), dtype=torch.int32, device="cuda")
    for mass in (None, torch.ones((n, 40), device="cuda")):
        ws = torch.empty(netkv.netkv_attn_decode_workspace_size(pages, n, heads, 40, mass is not None),
                         dtype=torch.uint8, device="cuda")
        out, lse = torch.full_like(q, 5.0), torch.full((n, heads), 5.0, device="cuda")
        torch.cuda.synchronize()
        netkv.netkv_attn_decode(pages, q, length, table, out, lse=lse, mass_out=mass, workspace=ws)
        seen, seen_lse = out.clone(), lse.clone()
        torch.cuda.synchronize()
        assert not seen.any() and bool((seen_lse == -float("inf")).all())
        assert mass is None or bool((mass == 1).all())


def milliseconds(f):
    """GPU time of the second of two calls."""
    f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b)


@pytest.mark.parametrize("n", [512, 513, 2500])
@pytest.mark.parametrize("fmt,dim", [("int8", 64), ("e4m3", 128)])
def test_store_of_thousands(netkv, n, fmt, dim):
    """Rows into blocks of many sequences, some without rows and some far longer than the average."""
    rng = np.random.default_rng(n)
    held = rng.integers(0, 40, n).tolist()
    new = (rng.integers(0, 2, n) * rng.integers(1, 20, n)).tolist()
    new[0], new[n // 2], new[n - 1] = 900, 0, 300
    assert check_store(netkv, held, new, 1, dim, fmt, torch.bfloat16, seed=n)[2] == 0


@pytest.mark.parametrize("dim,heads", [(64, 3), (128, 1)])
def test_load_of_thousands(netkv, dim, heads):
    """One call for all sequences gives what calls for 500 at a time give."""
    rng = np.random.default_rng(dim)
    n = 2000
    start, count = rng.integers(0, 40, n), rng.integers(0, 2, n) * rng.integers(1, 60, n)
    count[7], count[n - 1] = 1500, 600
    blocks = (-(-(start + count) // 16)).tolist()
    pages = netkv.KvPages(*pool(sum(blocks) + 2, heads, dim, "int8", 7))
    table = tables(blocks, max(blocks), sum(blocks) + 2, 7)
    got, want = (torch.full((2, int(count.sum()), heads, dim), 9.0, dtype=torch.float16, device="cuda")
                 for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    netkv.netkv_kv_load(pages, got[0], got[1], offsets(count), ints(start.tolist()), table, status=status)
    at = 0
    for i in range(0, n, 500):
        rows = int(count[i:i + 500].sum())
        netkv.netkv_kv_load(pages, want[0, at:at + rows], want[1, at:at + rows], offsets(count[i:i + 500]),
                            ints(start[i:i + 500].tolist()), table[i:i + 500], status=status)
        at += rows
    torch.cuda.synchronize()
    assert torch.equal(got, want) and int(status) == 0


def test_bad_rows_among_thousands(netkv):
    """Pages, offsets and tables out of range in a long batch: flagged, the others stored."""
    n = 3000
    rows = torch.ones((n, 1, 64), dtype=torch.float16, device="cuda")
    off = np.arange(n + 1)
    off[1000] = n + 5          # pair 999 passes the rows, pair 1000 decreases
    table = np.arange(n).reshape(n, 1)
    table[2000] = n            # no such page
    start = np.zeros(n, np.int64)
    start[2500] = 16           # past the table
    k, s = torch.zeros((n, 1, 16, 64), dtype=torch.int8, device="cuda"), torch.zeros((n, 1), device="cuda")
    pages = netkv.KvPages(k, k.clone(), s, s.clone())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    netkv.netkv_kv_store(pages, rows, rows, ints(off.tolist(), torch.int64), ints(start.tolist()),
                         ints(table.ravel().tolist()).view(n, 1), status=status)
    torch.cuda.synchronize()
    assert int(status) == netkv.NETKV_DEV_ERANGE
    written = set(torch.nonzero(s[:, 0]).ravel().tolist())
    assert written == set(range(n)) - {999, 1000, 2000, 2500}
    assert (k[list(written)][:, :, 0] == 127).all() and (k[:, :, 1:] == 0).all()


def test_time_of_a_token_for_each_of_many(netkv):
    """A warp that looks for its block among all sequences makes the call quadratic: the limit of
    2^24 - 1 sequences would take minutes."""
    n = 1 << 18
    rows = torch.ones((n, 1, 64), dtype=torch.float16, device="cuda")
    k, s = torch.zeros((n, 1, 16, 64), dtype=torch.int8, device="cuda"), torch.zeros((n, 1), device="cuda")
    pages = netkv.KvPages(k, k.clone(), s, s.clone())
    off = torch.arange(n + 1, device="cuda")
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
    back = torch.zeros((2,) + rows.shape, dtype=rows.dtype, device="cuda")
    assert milliseconds(lambda: netkv.netkv_kv_store(pages, rows, rows, off, None, table)) < 10
    assert milliseconds(lambda: netkv.netkv_kv_load(pages, back[0], back[1], off, None, table)) < 10
    assert torch.equal(back[0], rows) and torch.equal(back[1], rows)


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 64), (3, 1, 128)])
@pytest.mark.parametrize("n", [1024, 1025, 2000])
def test_prompts_of_thousands(netkv, n, heads, kv_heads, dim):
    """Many prompts with prefixes, some without rows and some of several row blocks, with rows that
    see no key among them: as calls for a hundred at a time give them."""
    rng = np.random.default_rng(n)
    lq = rng.integers(0, 2, n) * rng.integers(1, 40, n)
    lq[[3, n // 2, n - 1]] = 1500, 700, 900
    lk = np.maximum(lq + rng.integers(-5, 100, n), 0)
    q, k, v = (torch.randn((int(r.sum()), h, dim), device="cuda").half()
               for r, h in ((lq, heads), (lk, kv_heads), (lk, kv_heads)))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(a, b, out, lse):
        i, j = int(lq[:a].sum()), int(lk[:a].sum())
        x, y = i + int(lq[a:b].sum()), j + int(lk[a:b].sum())
        netkv.netkv_attn_prompt(q[i:x], k[j:y], v[j:y], offsets(lq[a:b]), offsets(lk[a:b]), out[i:x],
                                lse=lse[i:x], status=status)

    got, want = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
    lse, want_lse = (torch.full((len(q), heads), 5.0, device="cuda") for _ in range(2))
    call(0, n, got, lse)
    for a in range(0, n, 100):
        call(a, min(n, a + 100), want, want_lse)
    torch.cuda.synchronize()
    assert int(status) == 0
    # the two may take a row's keys in another order; outputs are sums of weights of at most 1
    finite = want_lse > -float("inf")
    assert torch.equal(finite, lse > -float("inf")) and bool((got[~finite] == 0).all())
    assert (lse - want_lse)[finite].abs().max() < 1e-5 * (1 + want_lse[finite].abs().max())
    assert (got.float() - want.float()).abs().max() < 4 * 2.0 ** -11 * v.float().abs().max()


def test_time_of_a_row_for_each_of_many_prompts(netkv):
    n = 1 << 16
    q = torch.ones((n, 1, 64), dtype=torch.float16, device="cuda")
    k = q.clone()
    off, out = torch.arange(n + 1, device="cuda"), torch.empty_like(q)
    assert milliseconds(lambda: netkv.netkv_attn_prompt(q, k, k, off, off, out)) < 20
    assert torch.equal(out, k)
