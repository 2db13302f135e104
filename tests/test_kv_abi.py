"""The KV-block entry points refuse bad arguments on the host, before any GPU work: no GPU here."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import netkv
    return netkv


def pages(lib, dtype=torch.int8, shape=(4, 2, 16, 64)):
    k = torch.zeros(shape, dtype=dtype)
    s = torch.zeros(shape[:2])
    return lib.KvPages(k, k.clone(), s, s.clone())


def test_pages_layout(lib):
    """Four pointers and four uint32 in 48 bytes."""
    assert C.sizeof(lib.KvPages) == 48
    assert [getattr(lib.KvPages, f).offset for f, _ in lib.KvPages._fields_] == [0, 8, 16, 24, 32, 36, 40, 44]
    p = pages(lib, torch.float8_e4m3fn)
    assert (p.n_pages, p.kv_heads, p.head_dim, p.format) == (4, 2, 64, lib.NETKV_KV_E4M3)


def test_workspace_sizes(lib):
    p = pages(lib)
    size = lib.netkv_attn_decode_workspace_size
    small, mass = size(p, 3, 8, 10), size(p, 3, 8, 10, True)
    assert 0 < small < mass and mass - small >= 3 * 10 * 8 * 4
    assert size(p, 3, 7, 10) == 0 and size(p, 3, 8, 0) == 0 and size(p, 3, 0, 10) == 0
    assert size(pages(lib, shape=(4, 2, 16, 32)), 3, 8, 10) == 0


def test_null_and_misaligned_pointers(lib):
    so, p = lib._lib, pages(lib)
    E, a = lib.NETKV_EINVAL, 1 << 20  # an address that is never read
    move = lambda *x: (so.netkv_kv_store(*x), so.netkv_kv_load(*x))  # noqa: E731
    assert move(None, 0, a, 128, a, 128, 1, a, 1, None, a, 1, None, None) == (E, E)
    assert move(p.ref, 2, a, 128, a, 128, 1, a, 1, None, a, 1, None, None) == (E, E)   # dtype
    assert move(p.ref, 0, a + 8, 128, a, 128, 1, a, 1, None, a, 1, None, None) == (E, E)
    assert move(p.ref, 0, a, 120, a, 128, 1, a, 1, None, a, 1, None, None) == (E, E)   # short row
    assert move(p.ref, 0, a, 132, a, 128, 1, a, 1, None, a, 1, None, None) == (E, E)   # odd stride
    assert move(p.ref, 0, a, 128, a, 128, 1, None, 1, None, a, 1, None, None) == (E, E)
    assert move(p.ref, 0, a, 128, a, 128, 1, a, 1, None, None, 1, None, None) == (E, E)
    assert move(p.ref, 0, a, 128, a, 128, 1, a, 1, None, a, 0, None, None) == (E, E)
    assert move(p.ref, 0, a, 128, a, 128, 1, a, 1 << 31, None, a, 1, None, None) == (E, E)
    assert move(p.ref, 0, None, 0, None, 0, 0, None, 0, None, None, 0, None, None) == (0, 0)
    prompt = lambda **k: so.netkv_attn_prompt(*{**dict(  # noqa: E731
        dtype=0, q=a, qs=128, k=a, ks=64, v=a, vs=64, heads=2, kv=1, dim=64, n=1, qo=a, ko=a,
        qr=1, kr=1, scale=1.0, out=a, os=128, lse=None, st=None, stream=None), **k}.values())
    for bad in (dict(dtype=2), dict(dim=96), dict(heads=0), dict(kv=0), dict(heads=3, kv=2),
                dict(q=None), dict(q=a + 2), dict(qs=64), dict(k=None), dict(vs=60), dict(out=None),
                dict(qo=None), dict(ko=a + 4), dict(scale=0.0), dict(scale=float("nan")),
                dict(qr=1 << 31), dict(n=1 << 24), dict(lse=a + 2)):
        assert prompt(**bad) == E, bad
    assert prompt(qr=0, q=None) == 0 and prompt(n=0) == 0
    need = lib.netkv_attn_decode_workspace_size(p, 1, 4, 1)
    decode = lambda **k: so.netkv_attn_decode(*{**dict(  # noqa: E731
        p=p.ref, dtype=0, q=a, qs=256, heads=4, n=1, len=a, table=a, width=1, scale=1.0, out=a,
        os=256, lse=None, mi=None, mo=None, ws=a, wb=need, st=None, stream=None), **k}.values())
    for bad in (dict(p=None), dict(dtype=5), dict(heads=3), dict(q=None), dict(qs=8), dict(len=None),
                dict(table=None), dict(width=0), dict(scale=-1.0), dict(out=a + 4), dict(mi=a),
                dict(ws=None), dict(ws=a + 4), dict(wb=need - 1), dict(mo=a, wb=need)):
        assert decode(**bad) == E, bad
    assert decode(n=0) == 0
    evict = lambda **k: so.netkv_kv_evict(*{**dict(  # noqa: E731
        n=1, t=a, l=a, m=a, w=4, b=a, sink=0, recent=1, to=2 * a, lo=a, mo=2 * a, f=3 * a, nf=a,
        st=None, stream=None), **k}.values())
    for bad in (dict(t=None), dict(recent=0), dict(w=0), dict(to=a), dict(mo=a), dict(f=a),
                dict(f=2 * a), dict(nf=None), dict(l=a + 1)):
        assert evict(**bad) == E, bad
    assert evict(n=0) == 0
