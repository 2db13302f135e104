"""Rows turned by their positions, and new tokens into 8-bit blocks with the rotation on the way,
against the definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import kv_plain as plain  # noqa: E402
from tests.test_gpu_kv_blocks import ints, offsets, pool, tables  # noqa: E402

# A turned value in fp32: an angle to 2^-22 of a radian (32 bits of a turn, rounded to fp32's 24), its
# cosine and sine to 2 units of 2^-24, and three roundings of products and their sum, of |x| + |y|.
ANGLE = 2.0 ** -21


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


def exact(x, pos, frequencies, sections, interleaved):
    """x [rows, heads, dim], pos [axes, rows] (CPU): the turned rows, and the sum |x| + |y| of each
    channel's pair, in float64."""
    x, n = x.cpu().double(), len(frequencies)
    y, size = x.clone(), torch.zeros_like(x)
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    for p in range(n):
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + n)
        # whole turns leave before the product loses bits
        angle = torch.tensor([math.fmod(t * frequencies[p], 2 * math.pi) for t in pos[axis[p]].tolist()],
                             dtype=torch.float64)[:, None]
        u, v = x[..., a], x[..., b]
        y[..., a], y[..., b] = u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()
        size[..., a] = size[..., b] = u.abs() + v.abs()
    return y, size


def rows(n, heads, dim, dtype, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads * dim + pad), generator=g).to(dtype).cuda()
    return x, x[:, :heads * dim].unflatten(1, (heads, dim))


def close(got, want, size, dtype):
    err = (got.cpu().double() - want).abs()
    tol = plain.U[dtype] * (want.abs() + ANGLE * size) + ANGLE * size + 2.0 ** -25
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs,sections", [(128, 64, [64]), (64, 32, [32]), (128, 64, [16, 24, 24]),
                                                (128, 16, [16]), (64, 8, [3, 5]), (128, 56, [20, 1, 0, 35]),
                                                (64, 24, [24])])
def test_rotate(netkv, dtype, interleaved, dim, pairs, sections):
    n, heads = 37, 5
    wide, x = rows(n, heads, dim, dtype, pad=24, seed=pairs)
    rng = np.random.default_rng(pairs)
    pos = torch.from_numpy(rng.integers(-5000, 200000, (len(sections), n)).astype(np.int32))
    out = torch.full((n, heads * dim + 8), 5.0, dtype=dtype, device="cuda")
    got = out[:, :heads * dim].unflatten(1, (heads, dim))
    rot = netkv.Rotary(pairs, base=10000.0, sections=sections, interleaved=interleaved)
    netkv.netkv_rotate(rot, x, pos.cuda(), got)
    torch.cuda.synchronize()
    f = [10000.0 ** (-p / pairs) for p in range(pairs)]
    want, size = exact(x, pos, f, sections, interleaved)
    close(got, want, size, dtype)
    assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])
    assert (out[:, heads * dim:] == 5).all()
    # and in place
    inside = wide.clone()
    at = inside[:, :heads * dim].unflatten(1, (heads, dim))
    netkv.netkv_rotate(rot, at, pos.cuda(), at)
    torch.cuda.synchronize()
    assert torch.equal(at, got) and torch.equal(inside[:, heads * dim:], wide[:, heads * dim:])


@pytest.mark.parametrize("n,heads", [(1, 1), (1, 200), (15, 3), (16, 17), (17, 1), (5000, 2)])
def test_rotate_sizes(netkv, n, heads):
    _, x = rows(n, heads, 64, torch.bfloat16, seed=n)
    pos = torch.arange(n, dtype=torch.int32)[None]
    out = torch.empty_like(x)
    netkv.netkv_rotate(netkv.Rotary(32), x, pos[0].cuda(), out)
    want, size = exact(x, pos, [10000.0 ** (-p / 32) for p in range(32)], [32], False)
    close(out, want, size, torch.bfloat16)


@pytest.mark.parametrize("at", [0, 1 << 20, (1 << 24) + 1, 2 ** 31 - 64, -(2 ** 31)])
def test_far_positions(netkv, at):
    """Angles of hundreds of millions of turns are right to their last digits: only whole turns go.
    The error grows by the frequencies' own rounding, position * 2^-53 of a radian, twice."""
    n = 33
    _, x = rows(n, 2, 128, torch.float16, seed=3)
    pos = (torch.arange(n, dtype=torch.int64) + at).to(torch.int32)[None]
    f = [1.0 - p / 100 for p in range(64)]
    # exact whole turns in integers: position * (f / 2 pi) with 80 bits behind the point
    from fractions import Fraction
    pi = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)
    turns = [Fraction(v) / (2 * pi) for v in f]
    angle = torch.tensor([[float((int(t) * w) % 1 * 2 * pi) for w in turns] for t in pos[0]],
                         dtype=torch.float64)[:, None]
    u, v = x[..., :64].cpu().double(), x[..., 64:].cpu().double()
    want = torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], 2)
    size = torch.cat([u.abs() + v.abs()] * 2, 2)
    out = torch.empty_like(x)
    netkv.netkv_rotate(netkv.Rotary(64, frequencies=f), x, pos.cuda(), out)
    err = (out.cpu().double() - want).abs()
    far = abs(at) * 2.0 ** -52
    tol = plain.U[torch.float16] * want.abs() + (ANGLE + far) * 1.01 * size + 2.0 ** -25
    assert (err <= tol).all(), float((err / tol).max())


def test_negated_positions_undo(netkv):
    """The inverse, and so the gradient of what goes through a rotation: the transposed matrix.  Each
    way rounds once, by 2^-8 of a value that is at most |x| + |y|."""
    _, x = rows(40, 3, 128, torch.bfloat16)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")[None] * 1000
    rot = netkv.Rotary(64, base=500000.0)
    there, back = torch.empty_like(x), torch.empty_like(x)
    netkv.netkv_rotate(rot, x, pos, there)
    netkv.netkv_rotate(rot, there, -pos, back)
    size = torch.cat([x[..., :64].float().abs() + x[..., 64:].float().abs()] * 2, 2)
    assert ((back.float() - x.float()).abs() <= 2.1 * 2.0 ** -8 * 1.5 * size).all()


def test_rotate_on_a_stream(netkv):
    _, x = rows(64, 2, 64, torch.float16)
    pos = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    a, b = torch.empty_like(x), torch.empty_like(x)
    netkv.netkv_rotate(netkv.Rotary(32), x, pos, a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        netkv.netkv_rotate(netkv.Rotary(32), x, pos, b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


# ---------------------------------------------------------------- append
def setup(netkv, held, new, kv_heads, heads, dim, fmt, dtype, seed=0, pad=0, short=0):
    blocks = [-(-(a + b) // 16) for a, b in zip(held, new)]
    width, n_pages = max(max(blocks) - short, 1), sum(blocks) + 3
    codes = pool(n_pages, kv_heads, dim, fmt, seed)
    table = tables(blocks, max(blocks) + 1, n_pages, seed)[:, :width].contiguous()
    total = sum(new)
    q, k, v = (rows(total, h, dim, dtype, pad, seed + i) for i, h in ((1, heads), (2, kv_heads), (3, kv_heads)))
    return codes, table, q, k[1], v[1]


def turned_blocks(codes, table, held, new, want, size, fmt, before, scale_before):
    """The blocks' keys after a call against turned rows `want` in float64 (rows of all sequences)."""
    top = plain.TOP[fmt]
    got, scale = plain.codes_value(codes[0]), codes[2].cpu().double()
    at = 0
    for i, (a, b) in enumerate(zip(held, new)):
        done = 0
        while done < b:
            t = a + done
            lead, page = t % 16, int(table[i, t // 16])
            n = min(16 - lead, b - done)
            x, e = want[at + done:at + done + n], ANGLE * size[at + done:at + done + n]
            largest, off = x.abs().amax((0, 2)), e.amax((0, 2))
            fresh = largest / top
            was = scale_before[page] if lead else torch.zeros_like(fresh)
            now = scale[page]
            assert ((now - torch.maximum(was, fresh)).abs() <= off / top + 2.0 ** -22 * now).all()
            # a code is the nearest to a value that is `e` off at most (2^-22: fp32's 1 / s and product)
            back = got[page, :, lead:lead + n].permute(1, 0, 2) * now[:, None]
            step = 0.5 if fmt == "int8" else torch.maximum(x.abs() / now[:, None] * 2.0 ** -4,
                                                           torch.tensor(2.0 ** -10))
            tol = step * now[:, None] * (1 + 2.0 ** -20) + 1.1 * e + 2.0 ** -21 * x.abs()
            assert ((back - x).abs() <= tol).all()
            if lead:  # the tokens before: by the ratio of the scales, from fp32
                f = np.float32
                old = before[page, :, :lead].numpy().astype(f)
                ratio = (scale_before[page].numpy().astype(f) / now.numpy().astype(f))[:, None, None]
                grown = (now > scale_before[page]).numpy()[:, None, None]
                exp = np.where(grown, plain.to_codes(old * ratio, fmt), old)
                assert np.array_equal(got[page, :, :lead].numpy().astype(f), exp)
            rest = got[page, :, lead + n:]
            assert torch.equal(rest, before[page, :, lead + n:])
            done += n
        at += b


HELD = [0, 0, 0, 5, 16, 15, 31, 1, 40, 0]
NEW = [1, 16, 33, 3, 1, 1, 20, 15, 0, 0]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,kv_heads,heads,pairs,interleaved,axes",
                         [(128, 2, 4, 64, False, 1), (64, 3, 21, 32, True, 1), (128, 1, 1, 64, False, 3),
                          (64, 8, 8, 16, False, 2)])
def test_append(netkv, fmt, dtype, dim, kv_heads, heads, pairs, interleaved, axes):
    held, new = HELD, NEW
    codes, table, (qw, q), k, v = setup(netkv, held, new, kv_heads, heads, dim, fmt, dtype, seed=dim, pad=16)
    total = sum(new)
    rng = np.random.default_rng(axes)
    sections = [pairs // axes + (pairs % axes if i == 0 else 0) for i in range(axes)]
    rot = netkv.Rotary(pairs, base=500000.0, sections=sections, interleaved=interleaved)
    pos = torch.from_numpy(rng.integers(0, 100000, (axes, total)).astype(np.int32))
    before, scale_before = plain.codes_value(codes[0]), codes[2].cpu().double()
    other = [x.clone() for x in codes]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((total + 2, heads * dim), 5.0, dtype=dtype, device="cuda")
    got = out[:total].unflatten(1, (heads, dim))
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), ints(held), table, rot,
                          pos=pos.cuda(), q=q, q_out=got, status=status)
    netkv.netkv_kv_store(netkv.KvPages(*other), k, v, offsets(new), ints(held), table)
    torch.cuda.synchronize()
    assert int(status) == 0
    f = [500000.0 ** (-p / pairs) for p in range(pairs)]
    want, size = exact(q, pos, f, sections, interleaved)
    close(got, want, size, dtype)
    assert (out[total:] == 5).all()
    want, size = exact(k, pos, f, sections, interleaved)
    turned_blocks(codes, table, held, new, want, size, fmt, before, scale_before)
    # values as netkv_kv_store has them, and pages without new tokens as they were
    assert torch.equal(codes[1].view(torch.uint8), other[1].view(torch.uint8))
    assert torch.equal(codes[3], other[3])
    touched = {int(table[i, b]) for i, (a, n) in enumerate(zip(held, new)) if n
               for b in range(a // 16, -(-(a + n) // 16))}
    still = [p for p in range(len(before)) if p not in touched]
    assert torch.equal(plain.codes_value(codes[0])[still], before[still])
    assert torch.equal(codes[2].cpu().double()[still], scale_before[still])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [3, 600])
def test_append_without_turning_is_store(netkv, fmt, dtype, n):
    """At frequency 0 cosines are 1 and sines 0, and everything is as netkv_kv_store has it to the bit;
    600 sequences take the other way to find their blocks."""
    rng = np.random.default_rng(n)
    held, new = rng.integers(0, 50, n).tolist(), (rng.integers(0, 3, n) * rng.integers(1, 30, n)).tolist()
    codes, table, (_, q), k, v = setup(netkv, held, new, 2, 6, 64, fmt, dtype, seed=n)
    other = [x.clone() for x in codes]
    out = torch.empty_like(q)
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), ints(held), table,
                          netkv.Rotary(32, frequencies=[0.0] * 32), q=q, q_out=out)
    netkv.netkv_kv_store(netkv.KvPages(*other), k, v, offsets(new), ints(held), table)
    torch.cuda.synchronize()
    assert torch.equal(out, q)
    for a, b in zip(codes, other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("start", [True, False])
def test_positions_from_the_blocks(netkv, start):
    """No positions given: a token's place in its sequence, in one call or token by token."""
    held, new = ([7, 0, 40], [20, 3, 9]) if start else ([0, 0, 0], [20, 3, 9])
    codes, table, (_, q), k, v = setup(netkv, held, new, 2, 4, 128, "int8", torch.float16)
    other = [x.clone() for x in codes]
    pos = torch.cat([torch.arange(a, a + b) for a, b in zip(held, new)]).to(torch.int32).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    at = ints(held) if start else None
    rot = netkv.Rotary(64)
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), at, table, rot, q=q, q_out=a)
    netkv.netkv_kv_append(netkv.KvPages(*other), k, v, offsets(new), at, table, rot, pos=pos, q=q, q_out=b)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(codes, other))
    # again: what is appended twice is the same
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), at, table, rot)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(codes, other))
    # and the queries where they are
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), at, table, rot, q=q, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(q, a)


@pytest.mark.parametrize("n", [1, 600])
def test_append_past_the_table(netkv, n):
    """Tokens without a place are not written; their queries are turned all the same, and so are those
    of a page number out of range.  Offsets that decrease have no rows."""
    held, new = [10] * n, [30] * n
    codes, table, (_, q), k, v = setup(netkv, held, new, 1, 2, 64, "int8", torch.float16, short=1)
    table[n // 2, 0] = 1 << 30
    want, out = torch.empty_like(q), torch.empty_like(q)
    pos = torch.arange(10, 40, dtype=torch.int32, device="cuda").repeat(n)
    rot, status = netkv.Rotary(32), torch.zeros(1, dtype=torch.int32, device="cuda")
    netkv.netkv_rotate(rot, q, pos, want)
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets(new), ints(held), table, rot, q=q,
                          q_out=out, status=status)
    torch.cuda.synchronize()
    assert int(status) == netkv.NETKV_DEV_ERANGE
    assert torch.equal(out, want)
    off = offsets(new)
    off[0] = 1 << 40
    status.zero_()
    out.fill_(5)
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, off, ints(held), table, rot, q=q, q_out=out,
                          status=status)
    torch.cuda.synchronize()
    assert int(status) == netkv.NETKV_DEV_ERANGE
    assert (out[:30] == 5).all() and torch.equal(out[30:], want[30:])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_special_values(netkv, fmt):
    """An infinity or NaN spreads over its pair and is held as zeros there, the status word set; tiny
    blocks are zeros of scale 0."""
    codes, table, (_, q), k, v = setup(netkv, [0], [48], 1, 2, 64, fmt, torch.bfloat16)
    k[3, 0, 5], k[20, 0, 40], k[32:] = math.inf, math.nan, 1e-38
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    netkv.netkv_kv_append(netkv.KvPages(*codes), k, v, offsets([48]), None, table, netkv.Rotary(32),
                          status=status)
    torch.cuda.synchronize()
    assert int(status) == netkv.NETKV_DEV_EDOMAIN
    got = plain.codes_value(codes[0])
    page = lambda t: int(table[0, t // 16])  # noqa: E731
    for t, c in ((3, 5), (3, 37), (20, 8), (20, 40)):
        assert got[page(t), 0, t % 16, c] == 0
    assert torch.isfinite(got).all() and torch.isfinite(codes[2]).all()
    assert (got[page(32)] == 0).all() and float(codes[2][page(32), 0]) == 0
    assert (got[page(3), 0, 3] != 0).sum() > 40


def test_rotate_and_append_replay(netkv):
    """Captured in a graph, with other rows, positions and lengths at the replay."""
    held, new = [3, 20], [30, 5]
    codes, table, (_, q), k, v = setup(netkv, held, new, 2, 4, 64, "int8", torch.bfloat16)
    table = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    codes = pool(10, 2, 64, "int8")
    pages, rot, out = netkv.KvPages(*codes), netkv.Rotary(32), torch.empty_like(q)
    off, start, pos = offsets(new), ints(held), torch.arange(35, dtype=torch.int32, device="cuda")
    turned = torch.empty_like(q)

    def step():
        netkv.netkv_kv_append(pages, k, v, off, start, table, rot, pos=pos, q=q, q_out=out)
        netkv.netkv_rotate(rot, out, pos, turned)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    q.copy_(torch.randn_like(q))
    k.copy_(torch.randn_like(k))
    off.copy_(offsets([12, 23]))
    start.copy_(ints([0, 33]))
    pos += 1000
    again = [x.clone() for x in codes]
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in codes] + [out.clone(), turned.clone()]
    for x, y in zip(codes, again):
        x.copy_(y)
    step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, [*codes, out, turned]))
