"""The KV-block calls captured in a CUDA graph: launches, the ones that start early among them, and
nothing else, so that a replay gives what the calls give."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_kv_blocks import ints, offsets  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("width", [20, 200])
def test_replay(width):
    from paper_2606_03910_gb300 import netkv
    n, heads, kv_heads, dim = 5, 8, 2, 128
    lengths = [min(x, width * 16) for x in (300, 17, 1, 3000, 900)]
    total, blocks = sum(lengths), [-(-x // 16) for x in lengths]
    g = torch.Generator().manual_seed(width)
    q, k, v = (torch.randn((total, h, dim), generator=g).bfloat16().cuda() for h in (heads, kv_heads, kv_heads))
    at, table = 0, torch.full((n, width), -1, dtype=torch.int32)
    for i, b in enumerate(blocks):
        table[i, :b] = torch.arange(at, at + b)
        at += b
    table, off, length = table.cuda(), offsets(lengths), ints(lengths)
    codes = torch.zeros((at, kv_heads, 16, dim), dtype=torch.int8, device="cuda")
    scale = torch.zeros((at, kv_heads), device="cuda")
    pages = netkv.KvPages(codes, codes.clone(), scale, scale.clone())
    ws = torch.empty(netkv.netkv_attn_decode_workspace_size(pages, n, heads, width, True),
                     dtype=torch.uint8, device="cuda")
    last = (off[1:] - 1).long()
    budget, status = ints([4] * n), torch.zeros(1, dtype=torch.int32, device="cuda")

    def outputs():
        return [torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0),
                torch.full_like(q[:n], 7.0), torch.full((n, width), 7.0, device="cuda"),
                torch.full_like(table, 7), torch.full_like(length, 7),
                torch.full((n, width), 7.0, device="cuda"), torch.full_like(table, 7),
                torch.full_like(length, 7)]

    def step(query, o):
        netkv.netkv_attn_prompt(q, k, v, off, off, o[0], status=status)
        netkv.netkv_kv_store(pages, k, v, off, None, table, status=status)
        netkv.netkv_kv_load(pages, o[1], o[2], off, None, table, status=status)
        netkv.netkv_attn_decode(pages, query, length, table, o[3], mass_out=o[4], workspace=ws, status=status)
        netkv.netkv_kv_evict(table, length, o[4], budget, 1, 1, *o[5:], status=status)

    query, want, got = q[last].clone(), outputs(), outputs()
    step(query, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(query, got)
    for other in (False, True):
        if other:  # new inputs in the same places
            for x in (q, k, v):
                x.copy_(torch.randn(x.shape, generator=g).to(x.dtype))
            query.copy_(q[last])
            want = outputs()
            step(query, want)
        for x, y in zip(got, outputs()):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_status_in_pinned_memory():
    """A status word that the host reads without a copy."""
    from paper_2606_03910_gb300 import netkv
    k, s = torch.zeros((1, 1, 16, 64), dtype=torch.int8, device="cuda"), torch.zeros((1, 1), device="cuda")
    pages = netkv.KvPages(k, k.clone(), s, s.clone())
    row = torch.full((1, 1, 64), float("inf"), dtype=torch.float16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, pin_memory=True)
    netkv.netkv_kv_store(pages, row, row, offsets([1]), None, ints([0]).view(1, 1), status=status)
    torch.cuda.synchronize()
    assert int(status) == netkv.NETKV_DEV_EDOMAIN
