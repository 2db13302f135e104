"""Calls with thousands of sequences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_kv_blocks import ints  # noqa: E402


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
