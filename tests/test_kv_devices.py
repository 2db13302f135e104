"""The KV-block calls take tensors of the current CUDA device only: an address of the host or of
another GPU never reaches a kernel.  Tensors that say which device they are on, and a library
whose calls are counted: no GPU here."""
import pytest

torch = pytest.importorskip("torch")


class On(torch.Tensor):
    """A tensor that says it is on a CUDA device."""
    where = 0

    def get_device(self):
        return self.where


def on(t, device):
    t = t.as_subclass(On)
    t.where = device
    return t


@pytest.fixture
def kv(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_03910_gb300 import netkv
    netkv._ask_torch()
    calls = []
    for f in ("netkv_kv_store", "netkv_kv_load", "netkv_attn_prompt", "netkv_attn_decode",
              "netkv_kv_evict"):
        monkeypatch.setattr(netkv._lib, f, lambda *a: calls.append(a) or 0)
    monkeypatch.setattr(netkv, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(netkv, "_current_device", lambda: 0)
    return netkv, calls


def rows(n, heads):
    return torch.zeros((n, heads, 64), dtype=torch.float16)


def pages(netkv, device):
    k, s = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1))
    return netkv.KvPages(*(on(x.clone(), device) for x in (k, k, s, s)))


I, L, F = torch.int32, torch.int64, torch.float32
ARGS = {
    "netkv_kv_store": dict(k=rows(3, 1), v=rows(3, 1), off=torch.zeros(3, dtype=L),
                           start=torch.zeros(2, dtype=I), table=torch.zeros((2, 4), dtype=I),
                           status=torch.zeros(1, dtype=I)),
    "netkv_attn_prompt": dict(q=rows(3, 2), k=rows(5, 1), v=rows(5, 1), q_off=torch.zeros(2, dtype=L),
                              k_off=torch.zeros(2, dtype=L), out=rows(3, 2),
                              lse=torch.zeros((3, 2)), status=torch.zeros(1, dtype=I)),
    "netkv_attn_decode": dict(q=rows(2, 2), length=torch.zeros(2, dtype=I),
                              table=torch.zeros((2, 4), dtype=I), out=rows(2, 2),
                              lse=torch.zeros((2, 2)), mass_in=torch.zeros((2, 4)),
                              mass_out=torch.zeros((2, 4)),
                              workspace=torch.zeros(1 << 10, dtype=torch.uint8),
                              status=torch.zeros(1, dtype=I)),
    "netkv_kv_evict": dict(table=torch.zeros((2, 4), dtype=I), length=torch.zeros(2, dtype=I),
                           mass=torch.zeros((2, 4)), budget=torch.zeros(2, dtype=I),
                           table_out=torch.zeros((2, 4), dtype=I),
                           length_out=torch.zeros(2, dtype=I), mass_out=torch.zeros((2, 4)),
                           freed=torch.zeros((2, 4), dtype=I), n_freed=torch.zeros(2, dtype=I),
                           status=torch.zeros(1, dtype=I)),
}
ARGS["netkv_kv_load"] = ARGS["netkv_kv_store"]
PAGED = ("netkv_kv_store", "netkv_kv_load", "netkv_attn_decode")


def run(netkv, name, where, stream=None):
    """One call, the argument named in `where` on another device than 0."""
    args = {k: on(t, where.get(k, 0)) for k, t in ARGS[name].items()}
    if name in PAGED:
        args["pages"] = pages(netkv, where.get("pages", 0))
    if name == "netkv_kv_evict":
        args.update(sink=0, recent=1)
    getattr(netkv, name)(**args, stream=stream)


@pytest.mark.parametrize("stream", [None, 5])
@pytest.mark.parametrize("name", sorted(ARGS))
def test_every_argument_is_on_the_current_device(kv, name, stream):
    netkv, calls = kv
    run(netkv, name, {}, stream)
    assert len(calls) == 1
    for arg in list(ARGS[name]) + (["pages"] if name in PAGED else []):
        for device in (-1, 1):
            with pytest.raises((TypeError, ValueError)):
                run(netkv, name, {arg: device}, stream)
    assert len(calls) == 1


@pytest.mark.parametrize("name", sorted(ARGS))
def test_all_on_a_device_that_is_not_current(kv, name):
    netkv, calls = kv
    with pytest.raises(ValueError):
        run(netkv, name, {k: 1 for k in list(ARGS[name]) + ["pages"]})
    assert not calls


def test_pages_of_two_devices(kv):
    netkv, _ = kv
    k, s = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1))
    with pytest.raises(ValueError):
        netkv.KvPages(on(k, 0), on(k.clone(), 0), on(s, 0), on(s.clone(), 1))


def test_addresses_and_absent_arguments(kv):
    """A status or workspace may be an address, as everywhere in the binding."""
    netkv, calls = kv
    a = {k: on(t, 0) for k, t in ARGS["netkv_attn_decode"].items()}
    a.update(status=1 << 20, lse=None, mass_in=None, mass_out=None)
    netkv.netkv_attn_decode(pages(netkv, 0), **a)
    a = {k: on(t, 0) for k, t in ARGS["netkv_kv_store"].items()}
    a.update(status=None, start=None)
    netkv.netkv_kv_store(pages(netkv, 0), **a)
    assert len(calls) == 2


def test_a_status_in_pinned_memory(kv, monkeypatch):
    """The host may poll it: the kernels' atomics reach pinned memory."""
    netkv, calls = kv
    a = {k: on(t, 0) for k, t in ARGS["netkv_kv_store"].items()}
    a.update(status=on(torch.zeros(1, dtype=I), -1))
    monkeypatch.setattr(On, "is_pinned", lambda t: True, raising=False)
    netkv.netkv_kv_store(pages(netkv, 0), **a)
    assert len(calls) == 1
    a.update(table=on(ARGS["netkv_kv_store"]["table"], -1))
    with pytest.raises(ValueError):
        netkv.netkv_kv_store(pages(netkv, 0), **a)


def test_a_workspace_that_is_not_as_large_as_it_says(kv):
    """Elements that lie on one another or apart: their number is not the buffer's size."""
    netkv, calls = kv
    one = torch.zeros(1, dtype=torch.uint8)
    for bad in (one.expand(1 << 10), torch.zeros(1 << 11, dtype=torch.uint8)[::2]):
        a = {k: on(t, 0) for k, t in ARGS["netkv_attn_decode"].items()}
        a.update(workspace=on(bad, 0))
        with pytest.raises(ValueError):
            netkv.netkv_attn_decode(pages(netkv, 0), **a)
    assert not calls
