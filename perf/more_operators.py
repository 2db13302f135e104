"""Cases of the operators on new tokens of a running batch: their positions, their way into the
blocks, and their attention over everything that the blocks hold.

- ``rotate``  rows turned by their positions, on one axis (text) or several (time, height, width);
- ``append``  new keys, turned on the way, and values into 8-bit blocks behind what these hold, the
              queries of the same tokens turned beside them, and the touched blocks read back;
- ``chunk``   causal attention of each sequence's new tokens over its 8-bit blocks: a part of a long
              prompt, drafted tokens to verify, single tokens, or a batch of all of them.

The heads are those of Llama-3-70B (64 query and 8 KV heads of 128, a fourth of them at TP=4)
where a case does not say otherwise; lengths are lognormal around a median, as the request
lengths of the scoring workloads are, and are part of the case; blocks hold 16 tokens and lie in
the page pool in random order.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
LARGEST = {"int8": 127.0, "e4m3": 448.0}   # the largest code of each 8-bit format
SMALLEST = 2.0 ** -100                     # blocks of smaller values are held as zeros

# n sequences with `new` tokens each (median; `single` of them with one) behind `held` (median; 0:
# none) that their blocks hold; spread is that of both lognormals
_BASE = dict(kind="chunk", n=1, new=512, held=8192, longest=32768, spread=1.0, single=0.0, mix=0,
             heads=16, kv_heads=2, dim=128, dtype="bf16", format="int8", pairs=64, axes=1,
             interleaved=False, base=500000.0, far=0)


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # queries and keys of a decode batch far into their contexts: latency
        _case("rotate_tokens", kind="rotate", new=64, heads=18, far=1 << 20),
        # a prompt's queries, a fourth of the channels turned, in neighbouring pairs
        _case("rotate_prompt", kind="rotate", new=16384, heads=16, pairs=16, interleaved=True,
              base=10000.0, dtype="f16"),
        # frames of a video for a whole model's queries and keys: three axes
        _case("rotate_video", kind="rotate", new=32768, heads=72, axes=3, base=1000000.0),
        # a decode batch's new tokens, each into a partly filled block
        _case("append_tokens", kind="append", n=96, new=1, held=2048, spread=0.7, heads=64,
              kv_heads=8, format="e4m3"),
        # parts of prompts behind what their blocks hold already; 64-wide heads, in neighbouring pairs
        _case("append_chunks", kind="append", n=12, new=400, held=3000, spread=0.8, heads=12,
              kv_heads=4, dim=64, pairs=32, interleaved=True, dtype="f16"),
        # a prefill batch with images in its prompts, the whole model's heads
        _case("append_prompts", kind="append", n=20, new=2500, longest=16384, held=0, heads=64,
              kv_heads=8, axes=3),
        # four drafted tokens of one short chat: latency
        _case("chunk_draft", new=4, held=500, spread=0.0),
        # drafted tokens of a decode batch, verified together
        _case("chunk_verify", n=64, new=5, held=8192, spread=0.6, longest=24000, format="e4m3"),
        # a batch of decoded tokens with parts of two prompts among them
        _case("chunk_mixed", n=26, new=900, held=5000, spread=0.8, longest=12000, single=0.92, mix=4),
        # one part of a prompt, two KV heads
        _case("chunk_part", new=512, held=7680, spread=0.0),
        # several short prompts' parts; 64-wide heads without groups, fp16
        _case("chunk_heads", n=10, new=300, held=2000, spread=0.7, longest=5000, heads=8, kv_heads=8,
              dim=64, dtype="f16"),
        # a large part of a very long prompt
        _case("chunk_long", new=2048, held=65536, longest=65536, spread=0.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "chunk", "chunk"])
    heads, kv_heads = rng.choice([(16, 2), (16, 2), (64, 8), (8, 8), (7, 1), (32, 2), (12, 4)])
    dim = rng.choice([128, 128, 64])
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, dtype=rng.choice(["bf16", "f16"]),
             format=rng.choice(["int8", "e4m3"]), mix=rng.randrange(1 << 20),
             spread=rng.choice([0.0, 0.5, 1.0]), interleaved=rng.random() < 0.3,
             pairs=rng.choice([dim // 2, dim // 2, dim // 2, dim // 4, 8]),
             base=rng.choice([10000.0, 500000.0, 1000000.0]))
    c["axes"] = rng.choice([1, 1, 2, 3]) if c["pairs"] > 8 else 1
    if kind == "rotate":
        c["heads"] = heads + kv_heads
        c["new"] = _log_int(rng, 1, 32768 * 72 * 128 // (c["heads"] * dim))
        c["far"] = rng.choice([0, 0, 1 << 20])
    elif kind == "append":
        if rng.random() < 0.4:
            c["n"], c["new"] = _log_int(rng, 1, 400), 1
        else:
            c["n"] = _log_int(rng, 1, 40)
            c["new"] = _log_int(rng, 2, max(3, 4_000_000 // ((heads + 2 * kv_heads) * dim * c["n"])))
        c["longest"] = max(4 * c["new"], 64)
        c["held"] = 0 if rng.random() < 0.3 else \
            _log_int(rng, 16, 400_000 // (c["n"] * kv_heads) + 17)
        c["longest"] = max(c["longest"], 2 * c["held"])
    else:
        c["n"] = _log_int(rng, 1, 100)
        # scores of the padded batch, and its keys, are kept below the largest listed case's
        scores = 16 * 2048 * 66000 // (c["n"] * heads)
        keys = min(66000, 64 * 2 * 24000 * 128 // (c["n"] * kv_heads * dim))
        most = min(4096, max(1, int(math.sqrt(scores) / 2)))
        c["new"] = _log_int(rng, 1, most)
        c["longest"] = max(c["new"], min(keys, scores // (2 * c["new"])))
        c["held"] = 0 if rng.random() < 0.15 else _log_int(rng, min(64, c["longest"]), c["longest"])
        c["single"] = rng.choice([0.0, 0.0, 0.8])
        if c["spread"]:  # the longest of a ragged batch
            c["new"] = max(1, c["new"] // 2)
    return _case(**c)


# ---------------------------------------------------------------- inputs
def _lengths(c):
    """New tokens of each sequence, and those that it holds before them."""
    r = random.Random(c["mix"] * 1009 + c["n"])

    def some(median, most):
        far = c["spread"] * r.gauss(0, 1) if median > 1 else 0.0
        return max(1, min(most, int(median * math.exp(far))))

    most = 2 * c["new"] if c["kind"] == "chunk" else c["longest"]
    new = [1 if r.random() < c["single"] else some(c["new"], most) for _ in range(c["n"])]
    held = [some(c["held"], c["longest"]) if c["held"] else 0 for _ in range(c["n"])]
    return new, held


def _offsets(lengths):
    t = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    t[1:] = torch.tensor(lengths, dtype=torch.int64).cumsum(0)
    return t.cuda()


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def _rows(g, rows, heads, dim, dtype):
    """Rows whose channels differ in size, as those after a projection do."""
    size = torch.exp(0.5 * torch.randn((1, heads, dim), generator=g, device="cuda"))
    return (torch.randn((rows, heads, dim), generator=g, device="cuda") * size).to(dtype)


def _pages(c, g, held):
    """A pool of 8-bit pages in random order, a block table, and codes as stored blocks have."""
    blocks = [-(-x // BLOCK) for x in held]
    width, used = max(blocks), sum(blocks)
    n_pages = used + used // 16 + 1
    order = torch.randperm(n_pages, generator=g, device="cuda")[:used].to(torch.int32)
    at = torch.arange(width, device="cuda")[None] < torch.tensor(blocks, device="cuda")[:, None]
    table = torch.full((c["n"], width), -1, dtype=torch.int32, device="cuda")
    table[at] = order
    shape = (n_pages, c["kv_heads"], BLOCK, c["dim"])
    top = LARGEST[c["format"]]

    def codes():
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16) * (top / 4)
        x = x.clamp_(-top, top)
        return x.round_().to(torch.int8) if c["format"] == "int8" else x.to(torch.float8_e4m3fn)

    def scales():
        return (0.5 + torch.rand(shape[:2], generator=g, device="cuda")) * 4 / top

    return dict(k=codes(), v=codes(), k_scale=scales(), v_scale=scales(), table=table)


def _sections(c):
    """Pairs of each axis, in order: time has the fewest where there are three."""
    p, n = c["pairs"], c["axes"]
    rest = (p * 3 // 8) if n == 3 else p // n
    return [p - rest * (n - 1)] + [rest] * (n - 1)


def _frequencies(c):
    """Radians a position of each pair."""
    p = c["pairs"]
    return [c["base"] ** (-i / p) for i in range(p)]


def _positions(c, g, first):
    """[axes][rows]: text counts up alike on every axis; images count frames, rows and columns."""
    rows = len(first)
    if c["axes"] == 1:
        return first[None].to(torch.int32).contiguous()
    side = 24
    at = torch.arange(rows, device="cuda")
    image = (at // 1024) % 2 == 0
    grid = [at // (side * side), at // side % side, at % side][-c["axes"]:]
    jump = torch.randint(0, 500, (1,), generator=g, device="cuda")
    return torch.stack([torch.where(image, x + jump, first) for x in grid]).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=c, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    dt = _dtype(c)
    if c["kind"] == "rotate":
        first = torch.arange(c["new"], device="cuda")
        if c["far"]:  # a token of each of many sequences
            first = torch.randint(0, c["far"], (c["new"],), generator=g, device="cuda")
        x = _rows(g, c["new"], c["heads"], c["dim"], dt)
        s.update(x=x, out=torch.empty_like(x), pos=_positions(c, g, first))
        return s
    new, held = _lengths(c)
    s.update(_pages(c, g, [a + b for a, b in zip(new, held)]))
    q = _rows(g, sum(new), c["heads"], c["dim"], dt)
    s.update(q=q, out=torch.empty_like(q), off=_offsets(new),
             start=torch.tensor(held, dtype=torch.int32).cuda(),
             length=torch.tensor([a + b for a, b in zip(new, held)], dtype=torch.int32).cuda())
    if c["kind"] == "chunk":
        s["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        return s
    first = [x // BLOCK * BLOCK for x in held]
    back = [a + b - f for a, b, f in zip(new, held, first)]
    seq, at = _sequence_of(s["off"], sum(new))
    k = _rows(g, sum(new), c["kv_heads"], c["dim"], dt)
    s.update(k_new=k, v_new=_rows(g, sum(new), c["kv_heads"], c["dim"], dt),
             pos=_positions(c, g, at - s["off"][seq] + s["start"].long()[seq]),
             back_off=_offsets(back), back_start=torch.tensor(first, dtype=torch.int32).cuda(),
             k_back=torch.empty((sum(back),) + k.shape[1:], dtype=dt, device="cuda"),
             v_back=torch.empty((sum(back),) + k.shape[1:], dtype=dt, device="cuda"))
    return s


# ---------------------------------------------------------------- plain forms
def _sequence_of(off, rows):
    at = torch.arange(rows, device="cuda")
    return torch.searchsorted(off[1:].contiguous(), at, right=True), at


def _axis_of(c):
    n = torch.tensor(_sections(c), device="cuda")
    return torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), n)


def _turned(c, x, pos):
    """x in fp32; the angles in 64 bits, since positions are far."""
    p = c["pairs"]
    angle = pos.double()[_axis_of(c)].T * torch.tensor(_frequencies(c), dtype=torch.float64,
                                                       device="cuda")
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float().clone()
    first, second = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if c["interleaved"] else \
        (slice(0, p), slice(p, 2 * p))
    a, b = x[..., first].float(), x[..., second].float()
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y


def _touched(start, count):
    """(sequence, block) of every block that tokens [start, start + count) touch."""
    first = start // BLOCK
    n = (start + count + BLOCK - 1) // BLOCK - first
    seq = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
    at = torch.arange(len(seq), device="cuda") - (n.cumsum(0) - n)[seq]
    return seq, at + first[seq]


def _to_codes(x, fmt):
    top = LARGEST[fmt]
    x = x.clamp(-top, top)
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _plain_store(s, codes, scale, rows, seq, block):
    fmt = s["case"]["format"]
    start, count = s["start"].long()[seq], s["off"].diff()[seq]
    pos = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    fresh = ((pos >= start[:, None]) & (pos < (start + count)[:, None]))[:, None, :, None]
    older = (pos < start[:, None])[:, None, :, None]
    row = (s["off"][seq][:, None] + pos - start[:, None]).clamp(0, len(rows) - 1)
    x = rows[row].permute(0, 2, 1, 3) * fresh
    page = s["table"].long()[seq, block]
    was = scale[page] * older.any(2)[..., 0]
    largest = x.abs().amax((2, 3))
    new = torch.where(largest < SMALLEST, torch.zeros_like(largest), largest / LARGEST[fmt])
    now = torch.maximum(was, new)
    inv = torch.where(now > 0, 1 / now, torch.zeros_like(now))
    ratio = torch.where(now > 0, was / now, torch.zeros_like(now))
    kept = codes[page].float()
    grown = torch.where(now > was, 1.0, 0.0)[..., None, None] * older
    y = torch.where(fresh, x * inv[..., None, None], kept)
    y = torch.where(grown > 0, kept * ratio[..., None, None], y)
    codes[page] = _to_codes(y, fmt)
    scale[page] = now


def _plain_load(s, codes, scale, seq, pos, dtype):
    page = s["table"].long()[seq, pos // BLOCK]
    x = codes.permute(0, 2, 1, 3)[page, pos % BLOCK].float()
    return (x * scale[page][..., None]).to(dtype)


def _plain_append(s):
    c, dt = s["case"], s["q"].dtype
    seq, block = _touched(s["start"].long(), s["off"].diff())
    _plain_store(s, s["k"], s["k_scale"], _turned(c, s["k_new"], s["pos"]), seq, block)
    _plain_store(s, s["v"], s["v_scale"], s["v_new"].float(), seq, block)
    rs, at = _sequence_of(s["back_off"], len(s["k_back"]))
    pos = at - s["back_off"][rs] + s["back_start"].long()[rs]
    return dict(q=_turned(c, s["q"], s["pos"]).to(dt),
                k=_plain_load(s, s["k"], s["k_scale"], rs, pos, dt),
                v=_plain_load(s, s["v"], s["v_scale"], rs, pos, dt),
                k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain_chunk(s):
    c = s["case"]
    rows, h, d = s["q"].shape
    n, new = c["n"], s["off"].diff()
    most = max(_lengths(c)[0])
    seq, at = _sequence_of(s["off"], rows)
    at = at - s["off"][seq]
    q = torch.zeros((n, most, h, d), device="cuda")
    q[seq, at] = s["q"].float() * d ** -0.5
    page = s["table"].long().clamp_min(0)

    def tokens(codes, scale):  # [n, kv heads, tokens, dim]
        x = codes[page].float() * scale[page][..., None, None]
        return x.permute(0, 2, 1, 3, 4).flatten(2, 3)

    k = tokens(s["k"], s["k_scale"])
    hk, width = k.shape[1:3]
    x = q.view(n, most, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d)
    x = (x @ k.transpose(2, 3)).view(n, h, most, width)
    last = (s["length"] - new)[:, None] + torch.arange(most, device="cuda")  # the row's own token
    hidden = torch.arange(width, device="cuda") > last[..., None]
    x.masked_fill_(hidden[:, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    v = tokens(s["v"], s["v_scale"])
    past = torch.arange(width, device="cuda")[None] >= s["length"][:, None]
    v.masked_fill_(past[:, None, :, None], 0.0)
    o = (x.view(n, hk, -1, width) @ v).view(n, h, most, d) / total.clamp_min(1e-38)
    lse = (m + total.log())[..., 0]
    return dict(out=o.permute(0, 2, 1, 3)[seq, at].to(s["q"].dtype),
                lse=lse.transpose(1, 2)[seq, at])


# ---------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2606_03910_gb300 import netkv
    c, status = s["case"], s["status"]
    # the handles and the workspace that a program keeps with its model and its pool
    if c["kind"] != "chunk" and "rotary" not in s:
        s["rotary"] = netkv.Rotary(c["pairs"], base=c["base"], sections=_sections(c),
                                   interleaved=c["interleaved"])
    if c["kind"] == "rotate":
        netkv.netkv_rotate(s["rotary"], s["x"], s["pos"], s["out"])
        return s["out"]
    if "pages" not in s:
        s["pages"] = netkv.KvPages(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if c["kind"] == "chunk":
            size = netkv.netkv_attn_chunk_workspace_size(s["pages"], s["q"].shape[0], c["n"],
                                                         c["heads"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if c["kind"] == "chunk":
        netkv.netkv_attn_chunk(s["pages"], s["q"], s["off"], s["length"], s["table"], s["out"],
                               lse=s["lse"], workspace=s["workspace"], status=status)
        return dict(out=s["out"], lse=s["lse"])
    netkv.netkv_kv_append(s["pages"], s["k_new"], s["v_new"], s["off"], s["start"], s["table"],
                          s["rotary"], pos=s["pos"], q=s["q"], q_out=s["out"], status=status)
    netkv.netkv_kv_load(s["pages"], s["k_back"], s["v_back"], s["back_off"], s["back_start"],
                        s["table"], status=status)
    return dict(q=s["out"], k=s["k_back"], v=s["v_back"], k_scale=s["k_scale"],
                v_scale=s["v_scale"])


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["kind"] == "rotate":
        return _turned(c, state["x"], state["pos"]).to(state["x"].dtype)
    return _plain_append(state) if c["kind"] == "append" else _plain_chunk(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    if c["kind"] == "rotate":
        return dict(bytes=c["new"] * (4 * h * d + 4 * c["axes"]), flops=6 * c["new"] * h * c["pairs"])
    new, held = _lengths(c)
    rows = sum(new)
    if c["kind"] == "append":
        older = sum(b % BLOCK for b in held)
        blocks = sum(-(-(a + b) // BLOCK) - b // BLOCK for a, b in zip(new, held))
        back = older + rows
        # rows in, codes out, and back: codes in, rows out; older codes in as well
        one = hk * (d * (2 * rows + older + back + back + 2 * back) + 8 * blocks)
        return dict(bytes=2 * one + rows * (4 * h * d + 4 * c["axes"]),
                    flops=6 * rows * (h + hk) * c["pairs"])
    pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, held))
    blocks = sum(-(-(a + b) // BLOCK) for a, b in zip(new, held))
    total = (rows + sum(held)) * 2 * d * hk + blocks * (8 * hk + 4) + rows * h * (4 * d + 4)
    return dict(bytes=total, flops=4 * d * h * pairs)


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_turn(c, x, pos):
    """Pair by pair, as products of complex numbers."""
    y, p, at = x.double().clone(), c["pairs"], 0
    for axis, n in enumerate(_sections(c)):
        for i in range(at, at + n):
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + p)
            angle = pos[axis].double() * c["base"] ** (-i / p)
            z = torch.complex(x[..., a].double(), x[..., b].double())
            z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        at += n
    return y


def _exact_round(x, fmt):
    if fmt == "int8":
        return x.round()
    # e4m3: 3 bits behind the leading one, exponents from -6, nearest, ties to even
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return ((x / step).round() * step).clamp(-448, 448)


def _exact_append(c, s):
    top = LARGEST[c["format"]]
    got = dict(q=_exact_turn(c, s["q"], s["pos"]))
    new, held = _lengths(c)
    rows = dict(k=_exact_turn(c, s["k_new"], s["pos"]), v=s["v_new"].double())
    for name, src in rows.items():
        scale, back, at = s[name + "_scale"].double(), [], 0
        for i, (a, b) in enumerate(zip(new, held)):
            lead = b % BLOCK
            n = -(-(lead + a) // BLOCK)
            pages = s["table"][i, b // BLOCK:b // BLOCK + n].long()
            x = torch.zeros((n * BLOCK,) + src.shape[1:], dtype=torch.float64, device="cuda")
            x[lead:lead + a] = src[at:at + a]
            at += a
            x = x.view(n, BLOCK, *src.shape[1:])
            now = x.abs().amax((1, 3)) / top
            if lead:
                was, older = scale[pages[0]], s[name][pages[0], :, :lead].double()
                now[0] = torch.maximum(now[0], was)
                older = _exact_round(older * (was / now[0])[:, None, None], c["format"])
            y = _exact_round(x / now[:, None, :, None], c["format"])
            if lead:
                y[0, :lead] = older.permute(1, 0, 2)
            scale[pages] = now
            back.append((y * now[:, None, :, None]).flatten(0, 1)[:lead + a])
        got[name], got[name + "_scale"] = torch.cat(back), scale
    return got


def _exact_chunk(c, s):
    group = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (a, b) in enumerate(zip(*_lengths(c))):
        n = a + b
        pages = s["table"][i, :-(-n // BLOCK)].long()
        for hk in range(c["kv_heads"]):
            k = s["k"][pages, hk].double() * s["k_scale"][pages, hk].double()[:, None, None]
            v = s["v"][pages, hk].double() * s["v_scale"][pages, hk].double()[:, None, None]
            k, v = k.flatten(0, 1)[:n], v.flatten(0, 1)[:n]
            for head in range(hk * group, (hk + 1) * group):
                for lo in range(0, a, 2048):
                    hi = min(a, lo + 2048)
                    x = (s["q"][at + lo:at + hi, head].double() @ k.T) / math.sqrt(c["dim"])
                    token = torch.arange(b + lo, b + hi, device="cuda")
                    x = x.masked_fill(torch.arange(n, device="cuda")[None] > token[:, None], -math.inf)
                    z = torch.logsumexp(x, 1)
                    out[at + lo:at + hi, head] = torch.exp(x - z[:, None]) @ v
                    lse[at + lo:at + hi, head] = z
        at += a
    return dict(out=out, lse=lse)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "rotate":
        return _exact_turn(c, s["x"], s["pos"])
    if c["kind"] == "append":
        return _exact_append(c, s)
    return _exact_chunk(c, s) if work(c)["flops"] < 4e12 else None
