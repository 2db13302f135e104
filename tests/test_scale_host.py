"""The softmax scale of the attention calls: it and its product with log2(e), which the exponentials go
by, are finite, or a score of 0 would become NaN.  Refused on the host: no GPU here."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_chunk_host import lib, pages  # noqa: E402,F401

# 2^128 / log2(e) is 2.3587e38
TOO_LARGE, LARGEST = (2.36e38, 3.0e38, 3.4e38), 2.358e38


def test_chunk(lib):  # noqa: F811
    p, a = pages(lib), 1 << 20
    need = lib.netkv_attn_chunk_workspace_size(p, 3, 1, 4)
    call = lambda rows, scale: lib._lib.netkv_attn_chunk(  # noqa: E731
        p.ref, 0, a, 256, 4, 1, a, rows, a, a, 1, scale, a, 256, None, a, need, None, None)
    assert all(call(3, s) == lib.NETKV_EINVAL for s in TOO_LARGE)
    assert call(0, LARGEST) == 0


def test_prompt(lib):  # noqa: F811
    a = 1 << 20
    call = lambda rows, scale: lib._lib.netkv_attn_prompt(  # noqa: E731
        0, a, 128, a, 64, a, 64, 2, 1, 64, 1, a, a, rows, 1, scale, a, 128, None, None, None)
    assert all(call(1, s) == lib.NETKV_EINVAL for s in TOO_LARGE)
    assert call(0, LARGEST) == 0


def test_decode(lib):  # noqa: F811
    p, a = pages(lib), 1 << 20
    need = lib.netkv_attn_decode_workspace_size(p, 1, 4, 1)
    for scale in TOO_LARGE:
        assert lib._lib.netkv_attn_decode(p.ref, 0, a, 256, 4, 1, a, a, 1, scale, a, 256, None, None, None,
                                          a, need, None, None) == lib.NETKV_EINVAL
