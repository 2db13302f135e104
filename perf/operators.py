"""Cases of the KV-block operators: what prefill and decode instances do with the caches that the
scorer places.

- ``prompt``  causal attention of packed prompts, grouped heads, some after a cached prefix;
- ``cache``   new keys and values into 8-bit blocks (a scale for each block and head), and the
              touched blocks read back as rows, as a prefill reads a cached prefix;
- ``decode``  one query a sequence over its blocks, with the attention weight that each block
              has drawn where eviction follows;
- ``evict``   block tables cut to a budget by accumulated attention weight.

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

_BASE = dict(kind="decode", n=1, median=8192, longest=32768, spread=1.0, mix=0, heads=16,
             kv_heads=2, dim=128, dtype="bf16", format="int8", prefix=0.0, mass=False,
             append=False, blocks=0, sink=4, recent=16, keep=0.5)


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short request arrives alone at an idle prefill instance: latency
        _case("prompt_one", kind="prompt", median=512, spread=0.0),
        # a prefill batch of ragged prompts packed up to 16K tokens
        _case("prompt_packed", kind="prompt", n=10, median=1500, longest=6000),
        # one long prompt
        _case("prompt_long", kind="prompt", median=32768, spread=0.0),
        # requests whose longer part is cached: the rest attends to prefix and itself; 64-wide heads
        _case("prompt_prefix", kind="prompt", n=6, median=700, longest=2000, heads=8, kv_heads=8,
              dim=64, dtype="f16", prefix=1.5),
        # the blocks of a prefill batch, to be moved to their decode instances
        _case("cache_prompts", kind="cache", n=24, median=4096, longest=32768, kv_heads=8),
        # a decode batch's new tokens: each lands in a partly filled block
        _case("cache_tokens", kind="cache", n=96, median=2048, append=True, format="e4m3"),
        # one stream of a chat: latency
        _case("decode_one", median=512, spread=0.0),
        # a decode batch under a memory budget: block weights gathered for eviction
        _case("decode_batch", n=64, mass=True),
        # two long contexts: few rows, long axis
        _case("decode_long", n=2, median=131072, longest=131072, spread=0.0, format="e4m3"),
        # the whole model's heads, many sequences
        _case("decode_wide", n=160, median=4096, longest=16384, heads=64, kv_heads=8, dtype="f16"),
        # long contexts cut to half their blocks
        _case("evict_long", kind="evict", n=4, blocks=8192),
        # a decode batch after a step, ragged
        _case("evict_batch", kind="evict", n=256, blocks=2048, keep=0.75),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "cache", "decode", "decode", "evict"])
    heads, kv_heads = rng.choice([(16, 2), (16, 2), (64, 8), (8, 8), (7, 1), (32, 2), (12, 4)])
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=rng.choice([128, 128, 64]),
             dtype=rng.choice(["bf16", "f16"]), format=rng.choice(["int8", "e4m3"]),
             mix=rng.randrange(1 << 20), spread=rng.choice([0.0, 0.5, 1.0]))
    if kind == "prompt":
        pairs = 16 * 32768 ** 2 // heads           # rows x columns of the largest listed case
        c["prefix"] = rng.choice([0.0, 0.0, 0.7, 2.0])
        whole = math.sqrt(pairs / (1 + 4 * c["prefix"])) * 0.95
        c["n"] = _log_int(rng, 1, 24)
        c["median"] = _log_int(rng, 16, max(17, int(whole / c["n"])))
        c["longest"] = max(c["median"], int(whole / c["n"]))
    elif kind == "cache":
        c["append"] = rng.random() < 0.4
        c["n"] = _log_int(rng, 1, 400 if c["append"] else 40)
        c["longest"] = (6_000_000 if c["append"] else 1_300_000) // (c["n"] * kv_heads)
        c["longest"] = min(32768, c["longest"])
        c["median"] = _log_int(rng, 16, c["longest"])
    elif kind == "decode":
        c["n"] = _log_int(rng, 1, 300)
        c["longest"] = min(131072, 160 * 16384 * 8 // (c["n"] * kv_heads))
        c["median"] = _log_int(rng, 16, c["longest"])
        c["mass"] = rng.random() < 0.5
    else:
        c["n"] = _log_int(rng, 1, 400)
        c["blocks"] = _log_int(rng, 64, min(8192, 400_000 // c["n"]))
        c["sink"], c["recent"] = rng.choice([0, 1, 4]), rng.choice([1, 8, 33])
        c["keep"] = round(rng.uniform(0.1, 1.0), 3)
    return _case(**c)


# ---------------------------------------------------------------- inputs
def _lengths(c):
    """New tokens of each sequence (prompt, cache) or tokens it holds (decode)."""
    r = random.Random(c["mix"] * 1009 + c["n"])
    return [max(1, min(c["longest"], int(c["median"] * math.exp(c["spread"] * r.gauss(0, 1)))))
            for _ in range(c["n"])]


def _held(c):
    """Tokens that each sequence holds before the call: a cached prefix, or the decoded part."""
    new = _lengths(c)
    if c["kind"] == "prompt":
        r = random.Random(c["mix"] * 31 + 7)
        return [int(x * c["prefix"] * r.random() * 2) for x in new]
    return new if c["append"] else [0] * c["n"]


def _offsets(lengths):
    t = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    t[1:] = torch.tensor(lengths, dtype=torch.int64).cumsum(0)
    return t.cuda()


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float16


def _rows(g, rows, heads, dim, dtype):
    """Rows whose channels differ in size, as keys after a projection do."""
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


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=c, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if c["kind"] == "evict":
        r = random.Random(c["mix"] * 17 + 3)
        n = [c["blocks"] if i == 0 else r.randint(max(1, c["blocks"] // 4), c["blocks"])
             for i in range(c["n"])]
        tokens = [x * BLOCK - r.randrange(BLOCK) for x in n]
        perm = torch.randperm(c["n"] * c["blocks"], generator=g, device="cuda").to(torch.int32)
        # weights fall over many orders; a few blocks have drawn exactly nothing
        mass = torch.exp(3 * torch.randn((c["n"], c["blocks"]), generator=g, device="cuda"))
        mass = mass * (torch.rand(mass.shape, generator=g, device="cuda") > 0.02)
        s.update(table=perm.view(c["n"], c["blocks"]), mass=mass,
                 length=torch.tensor(tokens, dtype=torch.int32).cuda(),
                 budget=torch.tensor([max(1, int(x * c["keep"])) for x in n],
                                     dtype=torch.int32).cuda(),
                 table_out=torch.empty_like(perm).view(c["n"], c["blocks"]),
                 mass_out=torch.empty_like(mass),
                 length_out=torch.empty(c["n"], dtype=torch.int32, device="cuda"),
                 freed=torch.empty_like(perm).view(c["n"], c["blocks"]),
                 n_freed=torch.empty(c["n"], dtype=torch.int32, device="cuda"))
        return s
    new, held, dt = _lengths(c), _held(c), _dtype(c)
    if c["kind"] == "prompt":
        both = [a + b for a, b in zip(new, held)]
        q = _rows(g, sum(new), c["heads"], c["dim"], dt)
        s.update(q=q, k=_rows(g, sum(both), c["kv_heads"], c["dim"], dt),
                 v=_rows(g, sum(both), c["kv_heads"], c["dim"], dt),
                 q_off=_offsets(new), k_off=_offsets(both), out=torch.empty_like(q),
                 lse=torch.empty((sum(new), c["heads"]), dtype=torch.float32, device="cuda"))
    elif c["kind"] == "cache":
        add = [1] * c["n"] if c["append"] else new
        s.update(_pages(c, g, [a + b for a, b in zip(add, held)]))
        first = [x // BLOCK * BLOCK for x in held]
        back = [a + b - f for a, b, f in zip(add, held, first)]
        k = _rows(g, sum(add), c["kv_heads"], c["dim"], dt)
        s.update(k_new=k, v_new=_rows(g, sum(add), c["kv_heads"], c["dim"], dt),
                 off=_offsets(add), start=torch.tensor(held, dtype=torch.int32).cuda(),
                 back_off=_offsets(back), back_start=torch.tensor(first, dtype=torch.int32).cuda(),
                 k_back=torch.empty((sum(back),) + k.shape[1:], dtype=dt, device="cuda"),
                 v_back=torch.empty((sum(back),) + k.shape[1:], dtype=dt, device="cuda"))
    else:
        s.update(_pages(c, g, new))
        q = torch.randn((c["n"], c["heads"], c["dim"]), generator=g, device="cuda").to(dt)
        s.update(q=q, out=torch.empty_like(q),
                 length=torch.tensor(new, dtype=torch.int32).cuda(),
                 lse=torch.empty((c["n"], c["heads"]), dtype=torch.float32, device="cuda"))
        if c["mass"]:
            s["mass"] = torch.rand(s["table"].shape, generator=g, device="cuda")
            s["mass_out"] = torch.zeros_like(s["mass"])
    return s


# ---------------------------------------------------------------- plain forms
def _sequence_of(off, rows):
    at = torch.arange(rows, device="cuda")
    return torch.searchsorted(off[1:].contiguous(), at, right=True), at


def _plain_prompt(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    (tq, h, d), (tk, hk, _) = q.shape, k.shape
    sq, iq = _sequence_of(s["q_off"], tq)
    sk, ik = _sequence_of(s["k_off"], tk)
    before = (s["k_off"].diff() - s["q_off"].diff())[sq]
    last = iq - s["q_off"][sq] + before
    hidden = (sq[:, None] != sk[None]) | ((ik - s["k_off"][sk])[None] > last[:, None])
    x = q.view(tq, hk, h // hk, d).permute(1, 2, 0, 3).reshape(hk, -1, d) * d ** -0.5
    x = (x @ k.permute(1, 2, 0)).view(h, tq, tk)
    x.masked_fill_(hidden, -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(hk, -1, tk) @ v.permute(1, 0, 2)).view(h, tq, d) / total.clamp_min(1e-38)
    lse = (m + total.log())[..., 0]
    return dict(out=o.permute(1, 0, 2).to(s["q"].dtype).contiguous(), lse=lse.T.contiguous())


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
    x = rows[row].float().permute(0, 2, 1, 3) * fresh
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


def _plain_cache(s):
    seq, block = _touched(s["start"].long(), s["off"].diff())
    _plain_store(s, s["k"], s["k_scale"], s["k_new"], seq, block)
    _plain_store(s, s["v"], s["v_scale"], s["v_new"], seq, block)
    rs, at = _sequence_of(s["back_off"], len(s["k_back"]))
    pos = at - s["back_off"][rs] + s["back_start"].long()[rs]
    return dict(k=_plain_load(s, s["k"], s["k_scale"], rs, pos, s["k_new"].dtype),
                v=_plain_load(s, s["v"], s["v_scale"], rs, pos, s["k_new"].dtype),
                k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain_decode(s):
    n, h, d = s["q"].shape
    page = s["table"].long().clamp_min(0)

    def rows(codes, scale):  # [n, kv heads, tokens, dim]
        x = codes[page].float() * scale[page][..., None, None]
        return x.permute(0, 2, 1, 3, 4).flatten(2, 3)

    k = rows(s["k"], s["k_scale"])
    x = (s["q"].float().view(n, k.shape[1], -1, d) * d ** -0.5) @ k.transpose(2, 3)
    hidden = torch.arange(k.shape[2], device="cuda")[None] >= s["length"][:, None]
    x.masked_fill_(hidden[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    v = rows(s["v"], s["v_scale"]).masked_fill_(hidden[:, None, :, None], 0.0)
    o = (x @ v) / total.clamp_min(1e-38)
    got = dict(out=o.reshape(n, h, d).to(s["q"].dtype), lse=(m + total.log()).reshape(n, h))
    if "mass" in s:
        p = (x / total.clamp_min(1e-38)).sum((1, 2)).view(n, -1, BLOCK).sum(-1)
        held = torch.arange(p.shape[1], device="cuda") * BLOCK < s["length"][:, None]
        got["mass"] = torch.where(held, s["mass"] + p, s["mass_out"])
    return got


def _plain_evict(s):
    c, length = s["case"], s["length"]
    n = (length + BLOCK - 1) // BLOCK
    at = torch.arange(c["blocks"], device="cuda")[None]
    gone = (n - s["budget"].clamp_min(c["sink"] + c["recent"])).clamp_min(0)
    open_ = (at >= c["sink"]) & (at < (n - c["recent"])[:, None])
    weight = torch.where(open_, s["mass"], torch.full_like(s["mass"], math.inf))
    order = weight.sort(dim=1, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, at.expand_as(order).contiguous())
    held = at < n[:, None]
    out = (rank < gone[:, None]) & held
    stay = held & ~out
    width = c["blocks"]

    def pack(mark, x, fill):
        to = torch.where(mark, mark.long().cumsum(1) - 1, width)
        y = torch.full((len(x), width + 1), fill, dtype=x.dtype, device="cuda")
        return y.scatter_(1, to, x)[:, :width].contiguous()

    return dict(table=_tail(pack(stay, s["table"], -1), stay, -1),
                mass=_tail(pack(stay, s["mass"], 0.0), stay, 0.0),
                freed=_tail(pack(out, s["table"], -1), out, -1),
                length=length - BLOCK * gone, n_freed=gone)


def _tail(x, mark, fill):
    past = torch.arange(x.shape[1], device="cuda")[None] >= mark.sum(1, keepdim=True)
    return x.masked_fill_(past, fill)


# ---------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2606_03910_gb300 import netkv
    kind, status = s["case"]["kind"], s["status"]
    if kind == "prompt":
        netkv.netkv_attn_prompt(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], s["out"],
                                lse=s["lse"], status=status)
        return dict(out=s["out"], lse=s["lse"])
    if kind == "evict":
        c = s["case"]
        netkv.netkv_kv_evict(s["table"], s["length"], s["mass"], s["budget"], c["sink"],
                             c["recent"], s["table_out"], s["length_out"], s["mass_out"],
                             s["freed"], s["n_freed"], status=status)
        return dict(table=s["table_out"], mass=s["mass_out"], freed=s["freed"],
                    length=s["length_out"], n_freed=s["n_freed"])
    if "pages" not in s:  # the handle and the workspace that a program keeps with its pool
        s["pages"] = netkv.KvPages(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if kind == "decode":
            size = netkv.netkv_attn_decode_workspace_size(
                s["pages"], *s["q"].shape[:2], s["table"].shape[1], s["case"]["mass"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if kind == "cache":
        netkv.netkv_kv_store(s["pages"], s["k_new"], s["v_new"], s["off"], s["start"], s["table"],
                             status=status)
        netkv.netkv_kv_load(s["pages"], s["k_back"], s["v_back"], s["back_off"], s["back_start"],
                            s["table"], status=status)
        return dict(k=s["k_back"], v=s["v_back"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    netkv.netkv_attn_decode(s["pages"], s["q"], s["length"], s["table"], s["out"], lse=s["lse"],
                            mass_in=s.get("mass"), mass_out=s.get("mass_out"),
                            workspace=s["workspace"], status=status)
    got = dict(out=s["out"], lse=s["lse"])
    if "mass" in s:
        got["mass"] = s["mass_out"]
    return got


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "cache": _plain_cache, "decode": _plain_decode,
            "evict": _plain_evict}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "evict":
        # the entries of every block read once, written once as kept or freed, with the padding
        r = random.Random(c["mix"] * 17 + 3)
        n = sum(c["blocks"] if i == 0 else r.randint(max(1, c["blocks"] // 4), c["blocks"])
                for i in range(c["n"]))
        return dict(bytes=8 * n + 12 * c["n"] * c["blocks"] + 16 * c["n"], flops=0)
    new, held = _lengths(c), _held(c)
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    if c["kind"] == "prompt":
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, held))
        tq, tk = sum(new), sum(new) + sum(held)
        return dict(bytes=2 * d * (2 * tq * h + 2 * tk * hk) + 4 * tq * h, flops=4 * d * h * pairs)
    if c["kind"] == "cache":
        add = [1] * c["n"] if c["append"] else new
        older = sum(b % BLOCK for b in held)
        blocks = sum(-(-(a + b) // BLOCK) - b // BLOCK for a, b in zip(add, held))
        rows = older + sum(add)
        # rows in, codes out, and back: codes in, rows out; older codes in as well
        one = hk * (d * (2 * sum(add) + older + rows + rows + 2 * rows) + 8 * blocks)
        return dict(bytes=2 * one, flops=0)
    blocks = sum(-(-x // BLOCK) for x in new)
    total = sum(new) * 2 * d * hk + blocks * (8 * hk + 4) + c["n"] * h * (4 * d + 4)
    return dict(bytes=total + (8 * blocks if c["mass"] else 0), flops=4 * d * h * sum(new))


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_attention(q, k, v, see):
    """One head in float64: rows that see nothing give 0 and -inf."""
    x = (q @ k.T) / math.sqrt(q.shape[1])
    x = torch.where(see, x, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    return p, p @ v, lse


def _exact_prompt(c, s):
    new, held = _lengths(c), _held(c)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    group, qa, ka = c["heads"] // c["kv_heads"], 0, 0
    for a, b in zip(new, held):
        for head in range(c["heads"]):
            k = s["k"][ka:ka + a + b, head // group].double()
            v = s["v"][ka:ka + a + b, head // group].double()
            for lo in range(0, a, 4096):
                hi = min(a, lo + 4096)
                see = torch.arange(a + b, device="cuda")[None] <= \
                    torch.arange(lo + b, hi + b, device="cuda")[:, None]
                _, o, z = _exact_attention(s["q"][qa + lo:qa + hi, head].double(), k, v, see)
                out[qa + lo:qa + hi, head], lse[qa + lo:qa + hi, head] = o, z
        qa, ka = qa + a, ka + a + b
    return dict(out=out, lse=lse)


def _exact_round(x, fmt):
    if fmt == "int8":
        return x.round()
    # e4m3: 3 bits behind the leading one, exponents from -6, nearest, ties to even
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return ((x / step).round() * step).clamp(-448, 448)


def _exact_cache(c, s):
    top, got = LARGEST[c["format"]], {}
    add, held = s["off"].diff().tolist(), s["start"].tolist()
    for name in ("k", "v"):
        scale, back = s[name + "_scale"].double(), []
        src = s[name + "_new"].double()
        at = 0
        for i, (a, b) in enumerate(zip(add, held)):
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


def _exact_decode(c, s):
    group, got_mass = c["heads"] // c["kv_heads"], None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    if c["mass"]:
        got_mass = s["mass_out"].double()
    for i, length in enumerate(_lengths(c)):
        n = -(-length // BLOCK)
        pages = s["table"][i, :n].long()
        see = torch.arange(n * BLOCK, device="cuda")[None] < length
        drawn = torch.zeros(n * BLOCK, dtype=torch.float64, device="cuda")
        for hk in range(c["kv_heads"]):
            k = s["k"][pages, hk].double() * s["k_scale"][pages, hk].double()[:, None, None]
            v = s["v"][pages, hk].double() * s["v_scale"][pages, hk].double()[:, None, None]
            at = slice(hk * group, (hk + 1) * group)
            p, o, z = _exact_attention(s["q"][i, at].double(), k.flatten(0, 1), v.flatten(0, 1), see)
            out[i, at], lse[i, at] = o, z
            drawn += p.sum(0)
        if got_mass is not None:
            got_mass[i, :n] = s["mass"][i, :n].double() + drawn.view(n, BLOCK).sum(1)
    got = dict(out=out, lse=lse)
    if got_mass is not None:
        got["mass"] = got_mass
    return got


def exact(case, seed):
    if case["kind"] == "evict":  # whole numbers, and weights that only move
        return None
    s = prepare(case, seed)
    if case["kind"] == "prompt":
        return _exact_prompt(case, s) if work(case)["flops"] < 1e13 else None
    if case["kind"] == "cache":
        return _exact_cache(case, s)
    return _exact_decode(case, s) if case["n"] * case["kv_heads"] < 4000 else None
