"""The calls on new tokens refuse bad arguments on the host, before any GPU work, and take tensors of
the current CUDA device only: no GPU here."""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_kv_devices import on, pages as device_pages, rows  # noqa: E402


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


def test_rotary_layout_and_steps(lib):
    """64 uint64, 64 bytes and four uint32 in 592 bytes; a step is a part of a turn times 2^64."""
    R = lib.Rotary
    assert C.sizeof(R) == 592
    assert [getattr(R, f).offset for f, _ in R._fields_] == [0, 512, 576, 580, 584, 588]
    r = R(24, base=1000.0, sections=[4, 0, 20], interleaved=True)
    assert (r.pairs, r.axes, r.interleaved, r.reserved) == (24, 3, 1, 0)
    assert list(r.axis)[:24] == [0] * 4 + [2] * 20
    for p in range(24):
        assert abs(r.step[p] / 2.0 ** 64 * 2 * math.pi - 1000.0 ** (-p / 24)) <= 2.0 ** -51
    assert list(r.step)[24:] == [0] * 40


@pytest.mark.parametrize("bad", [
    dict(pairs=0), dict(pairs=65), dict(pairs=12), dict(pairs=-8), dict(pairs=8, sections=[4, 3]),
    dict(pairs=8, sections=[9, -1]), dict(pairs=8, sections=[2, 2, 2, 1, 1]), dict(pairs=8, sections=[]),
    dict(pairs=8, frequencies=[1.0] * 7), dict(pairs=8, frequencies=[1.0] * 7 + [-1.0]),
    dict(pairs=8, frequencies=[1.0] * 7 + [math.nan]), dict(pairs=8, frequencies=[1.0] * 7 + [2 * math.pi])])
def test_rotary_refusals(lib, bad):
    with pytest.raises((ValueError, lib.NetKVError)):
        lib.Rotary(**bad)


def test_rotary_set_refuses_without_writing(lib):
    so, r, f = lib._lib, lib.Rotary(8), (C.c_double * 8)(*[1.0] * 8)
    n = (C.c_uint32 * 2)(4, 4)
    before = bytes(r)
    for args in ((None, 8, f, 1, None, 0), (r.ref, 8, None, 1, None, 0), (r.ref, 8, f, 2, None, 0),
                 (r.ref, 8, f, 0, n, 0), (r.ref, 8, f, 5, n, 0), (r.ref, 8, f, 2, n, 2),
                 (r.ref, 16, f, 2, n, 0), (r.ref, 8, f, 1, n, 0)):
        assert so.netkv_rotary_set(*args) == lib.NETKV_EINVAL
    assert bytes(r) == before
    assert so.netkv_rotary_set(r.ref, 8, f, 2, n, 1) == 0 and r.axes == 2


def broken(lib, **fields):
    r = lib.Rotary(8)
    for k, v in fields.items():
        if k == "axis0":
            r.axis[0] = v
        else:
            setattr(r, k, v)
    return r


BROKEN = [dict(pairs=0), dict(pairs=4), dict(pairs=40), dict(pairs=1 << 31), dict(axes=0), dict(axes=5),
          dict(axis0=1), dict(interleaved=2), dict(reserved=1)]


def test_rotate_refusals(lib):
    so, E, a = lib._lib, lib.NETKV_EINVAL, 1 << 20  # an address that is never read
    r = lib.Rotary(32)
    call = lambda **k: so.netkv_rotate(*{**dict(  # noqa: E731
        rot=r.ref, dtype=0, x=a, xs=128, heads=2, dim=64, rows=1, pos=a, out=2 * a, os=128, stream=None),
        **k}.values())
    for bad in (dict(rot=None), dict(dtype=2), dict(dim=96), dict(heads=0), dict(heads=65536), dict(x=None),
                dict(x=a + 2), dict(xs=64), dict(xs=132), dict(rows=1 << 31), dict(pos=None),
                dict(pos=a + 2), dict(out=None), dict(os=120), dict(out=a, os=136),
                dict(rot=lib.Rotary(64).ref)):
        assert call(**bad) == E, bad
    for fields in BROKEN:
        assert call(rot=broken(lib, **fields).ref) == E, fields
    assert call(rows=0, x=None) == 0


def test_append_refusals(lib):
    so, E, a, p = lib._lib, lib.NETKV_EINVAL, 1 << 20, pages(lib)
    r, two = lib.Rotary(32), lib.Rotary(32, sections=[16, 16])
    call = lambda **k: so.netkv_kv_append(*{**dict(  # noqa: E731
        p=p.ref, rot=r.ref, dtype=0, k=a, ks=128, v=a, vs=128, n=1, off=a, rows=1, start=None, table=a,
        width=1, pos=None, heads=4, q=a, qs=256, qo=2 * a, qos=256, st=None, stream=None), **k}.values())
    for bad in (dict(p=None), dict(rot=None), dict(rot=two.ref), dict(rot=lib.Rotary(64).ref), dict(dtype=2),
                dict(k=None), dict(k=a + 8), dict(ks=120), dict(vs=132), dict(v=None), dict(off=None),
                dict(off=a + 4), dict(table=None), dict(table=a + 2), dict(width=0), dict(width=1 << 28),
                dict(rows=1 << 31), dict(n=1 << 24), dict(start=a + 2), dict(pos=a + 2), dict(heads=0),
                dict(heads=65536), dict(qs=248), dict(q=a + 4), dict(qo=None), dict(qos=128),
                dict(qo=a, qos=264), dict(st=a + 2)):
        assert call(**bad) == E, bad
    for fields in BROKEN:
        assert call(rot=broken(lib, **fields).ref) == E, fields
    assert call(rows=0, k=None) == 0 and call(n=0) == 0
    assert call(p=pages(lib, shape=(4, 2, 16, 32)).ref) == E


def test_chunk_refusals_and_workspace(lib):
    so, E, a, p = lib._lib, lib.NETKV_EINVAL, 1 << 20, pages(lib)
    size = lib.netkv_attn_chunk_workspace_size
    need = size(p, 3, 1, 4)
    assert need > 0 and need % 16 == 0
    assert size(p, 3, 1, 5) == 0 and size(p, 3, 1, 0) == 0 and size(p, 1 << 31, 1, 4) == 0
    assert size(p, 3, 1 << 24, 4) == 0 and size(pages(lib, shape=(4, 2, 16, 32)), 3, 1, 4) == 0
    # no larger call of the same pool needs less
    assert need <= size(p, 30, 2, 4) <= size(p, 3000, 5, 8)
    call = lambda **k: so.netkv_attn_chunk(*{**dict(  # noqa: E731
        p=p.ref, dtype=0, q=a, qs=256, heads=4, n=1, off=a, rows=3, len=a, table=a, width=1, scale=1.0,
        out=a, os=256, lse=None, ws=a, wb=need, st=None, stream=None), **k}.values())
    for bad in (dict(p=None), dict(dtype=2), dict(heads=3), dict(heads=0), dict(q=None), dict(q=a + 4),
                dict(qs=8), dict(off=None), dict(off=a + 4), dict(len=None), dict(len=a + 2), dict(table=None),
                dict(width=0), dict(width=1 << 28), dict(scale=-1.0), dict(scale=0.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(out=None), dict(out=a + 4), dict(os=128), dict(lse=a + 2),
                dict(ws=None), dict(ws=a + 8), dict(wb=need - 1), dict(wb=0), dict(st=a + 2),
                dict(rows=1 << 31), dict(n=1 << 24)):
        assert call(**bad) == E, bad
    assert call(rows=0, q=None) == 0 and call(n=0) == 0


# ---------------------------------------------------------------- the binding
@pytest.fixture
def kv(monkeypatch, lib):
    lib._ask_torch()
    calls = []
    for f in ("netkv_rotate", "netkv_kv_append", "netkv_attn_chunk"):
        monkeypatch.setattr(lib._lib, f, lambda *a: calls.append(a) or 0)
    monkeypatch.setattr(lib, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(lib, "_current_device", lambda: 0)
    return lib, calls


I, L = torch.int32, torch.int64
ARGS = {
    "netkv_rotate": dict(x=rows(3, 2), pos=torch.zeros((1, 3), dtype=I), out=rows(3, 2)),
    "netkv_kv_append": dict(k=rows(3, 1), v=rows(3, 1), off=torch.zeros(3, dtype=L),
                            start=torch.zeros(2, dtype=I), table=torch.zeros((2, 4), dtype=I),
                            pos=torch.zeros((1, 3), dtype=I), q=rows(3, 2), q_out=rows(3, 2),
                            status=torch.zeros(1, dtype=I)),
    "netkv_attn_chunk": dict(q=rows(3, 2), off=torch.zeros(3, dtype=L), length=torch.zeros(2, dtype=I),
                             table=torch.zeros((2, 4), dtype=I), out=rows(3, 2), lse=torch.zeros((3, 2)),
                             workspace=torch.zeros(1 << 10, dtype=torch.uint8),
                             status=torch.zeros(1, dtype=I)),
}
PAGED = ("netkv_kv_append", "netkv_attn_chunk")


def run(netkv, name, where=None, change=None, stream=None):
    """One call, the argument named in `where` on another device than 0, those in `change` others."""
    args = {k: t if t is None else on(t, (where or {}).get(k, 0))
            for k, t in {**ARGS[name], **(change or {})}.items()}
    if name in PAGED:
        args["pages"] = device_pages(netkv, (where or {}).get("pages", 0))
    if name != "netkv_attn_chunk":
        args["rotary"] = netkv.Rotary(32)
    getattr(netkv, name)(**args, stream=stream)


@pytest.mark.parametrize("stream", [None, 5])
@pytest.mark.parametrize("name", sorted(ARGS))
def test_every_argument_is_on_the_current_device(kv, name, stream):
    netkv, calls = kv
    run(netkv, name, stream=stream)
    assert len(calls) == 1
    for arg in list(ARGS[name]) + (["pages"] if name in PAGED else []):
        for device in (-1, 1):
            with pytest.raises((TypeError, ValueError)):
                run(netkv, name, {arg: device}, stream=stream)
    with pytest.raises(ValueError):
        run(netkv, name, {k: 1 for k in list(ARGS[name]) + ["pages"]})
    assert len(calls) == 1


@pytest.mark.parametrize("name,change", [
    ("netkv_rotate", dict(out=rows(4, 2))), ("netkv_rotate", dict(out=rows(3, 1))),
    ("netkv_rotate", dict(out=rows(3, 2).bfloat16())), ("netkv_rotate", dict(x=rows(3, 2).float())),
    ("netkv_rotate", dict(pos=torch.zeros((2, 3), dtype=I))), ("netkv_rotate", dict(pos=torch.zeros((1, 4), dtype=I))),
    ("netkv_rotate", dict(pos=torch.zeros((1, 3), dtype=L))), ("netkv_rotate", dict(pos=None)),
    ("netkv_rotate", dict(pos=torch.zeros((1, 6), dtype=I)[:, ::2])),
    ("netkv_rotate", dict(x=torch.zeros((3, 64, 2), dtype=torch.float16).transpose(1, 2))),
    ("netkv_kv_append", dict(v=rows(4, 1))), ("netkv_kv_append", dict(k=rows(3, 2))),
    ("netkv_kv_append", dict(q=None)), ("netkv_kv_append", dict(q_out=None)),
    ("netkv_kv_append", dict(q=rows(2, 2))), ("netkv_kv_append", dict(q_out=rows(4, 2))),
    ("netkv_kv_append", dict(q=rows(3, 2).bfloat16(), q_out=rows(3, 2).bfloat16())),
    ("netkv_kv_append", dict(start=torch.zeros(3, dtype=I))), ("netkv_kv_append", dict(table=torch.zeros((3, 4), dtype=I))),
    ("netkv_kv_append", dict(off=torch.zeros(3, dtype=I))), ("netkv_kv_append", dict(pos=torch.zeros((3, 1), dtype=I))),
    ("netkv_attn_chunk", dict(out=rows(2, 2))), ("netkv_attn_chunk", dict(q=rows(3, 2).bfloat16())),
    ("netkv_attn_chunk", dict(length=torch.zeros(3, dtype=I))), ("netkv_attn_chunk", dict(table=torch.zeros((2, 8), dtype=I)[:, ::2])),
    ("netkv_attn_chunk", dict(lse=torch.zeros((3, 1)))), ("netkv_attn_chunk", dict(lse=torch.zeros((3, 2)).half())),
    ("netkv_attn_chunk", dict(q=torch.zeros((3, 2, 128), dtype=torch.float16), out=torch.zeros((3, 2, 128), dtype=torch.float16))),
    ("netkv_attn_chunk", dict(workspace=torch.zeros(1 << 11, dtype=torch.uint8)[::2]))])
def test_tensors_that_do_not_fit(kv, name, change):
    netkv, calls = kv
    with pytest.raises((TypeError, ValueError)):
        run(netkv, name, change=change)
    assert not calls


def test_absent_arguments(kv):
    netkv, calls = kv
    run(netkv, "netkv_kv_append", change=dict(pos=None, q=None, q_out=None, start=None, status=None))
    run(netkv, "netkv_kv_append", change=dict(pos=torch.zeros(3, dtype=I)))
    run(netkv, "netkv_attn_chunk", change=dict(lse=None, status=None, workspace=None))
    run(netkv, "netkv_rotate", change=dict(pos=torch.zeros(3, dtype=I)))
    assert len(calls) == 4
