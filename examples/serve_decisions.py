"""From decisions to tokens: the scorer places prefilled requests, and the blocks follow.

A small cluster's requests are scored and dispatched (``Scorer``).  Each prefill instance then
runs the prompts' attention and writes their keys and values into 8-bit blocks, the blocks move
to the decode instance that was chosen, and that instance decodes: a new token a step into its
block, attention over the blocks, and eviction of the least attended ones when the instance is
over its budget of pages.  Keys, values and queries are random rows: there is no model here, one
attention layer stands for all.

    python examples/serve_decisions.py [--steps 24] [--format int8|e4m3]
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

HEADS, KV_HEADS, DIM, LAYERS = 16, 2, 128, 80   # Llama-3-70B at TP=4
LONGEST = 4096                                  # tokens of a prompt that are kept, for size


def place(seed=0):
    """The decisions of one small stream: [(request, prefill, decode, tokens)]."""
    import synth
    from paper_2606_03910_gb300 import netkv
    from paper_2606_03910_gb300.blocks import bytes_per_token
    from paper_2606_03910_gb300.pipeline import Scorer, StepInputs, weights_tensor
    from synth import stage
    w = synth.make_workload(synth.tiny_spec(seed0=seed, n_streams=1))
    spec = w.spec
    sc = Scorer(spec.fanout, w.role, spec.tier_bw, spec.tier_lat, w.L, w.n_sets,
                netkv.index_log2_capacity(synth.distinct_keys_per_group(w)))
    sc.load_caches(stage.keys(w, 0, w.n_sets), stage.key_offsets(w, w.n_sets * w.D))
    ra = stage.request_arrays(w)
    # an 8-bit cache moves half the bytes, so its transfers are priced at half
    x = StepInputs(util=stage.util(w), chains=stage.chains(w), chain_off=ra["chain_off"],
                   set_off=ra["set_off"], length=ra["length"], prefill=ra["prefill"],
                   snap=ra["snap"], events=ra["events"], event_off=ra["event_off"],
                   weights=weights_tensor(w.weights, synth.THETA_S_PER_TOKEN, spec.cap_tokens,
                                          bytes_per_token(LAYERS, KV_HEADS, DIM)))
    out = sc.step(x, sc.alloc_outputs(x.n_snap, x.R, x.n_streams))
    dec, length, pre = out.dec.tolist(), ra["length"].tolist(), ra["prefill"].tolist()
    return [(r, pre[r], dec[r], min(length[r], LONGEST)) for r in range(x.R) if dec[r] >= 0]


def prefill(requests, fmt, g):
    """Prompts of one prefill instance, packed: the attention's output, and a pool that holds
    their blocks, a slot a request."""
    import torch
    from paper_2606_03910_gb300 import netkv
    from paper_2606_03910_gb300.blocks import BlockPool, blocks_of
    lengths = [n for *_, n in requests]
    total = sum(lengths)
    rows = lambda h: torch.randn((total, h, DIM), generator=g, device="cuda").bfloat16()  # noqa: E731
    q, k, v = rows(HEADS), rows(KV_HEADS), rows(KV_HEADS)
    pool = BlockPool(sum(map(blocks_of, lengths)), KV_HEADS, DIM, len(lengths),
                     max(map(blocks_of, lengths)), fmt)
    off = pool._offsets(lengths)
    out = torch.empty_like(q)
    netkv.netkv_attn_prompt(q, k, v, off, off, out, status=pool.status)
    pool.append(k, v, lengths)
    return out, pool


def serve(steps=24, fmt="int8", budget=0.6, seed=0, report=print):
    """Runs the whole path; returns what the last step's attention gave for each instance."""
    import torch
    from paper_2606_03910_gb300.blocks import BlockPool, blocks_of, move
    g = torch.Generator(device="cuda").manual_seed(seed)
    placed = place(seed)
    by_decode, results = {}, {}
    for r in placed:
        by_decode.setdefault(r[2], []).append(r)
    pools = {}
    for d, here in by_decode.items():
        room = sum(blocks_of(n + steps) for *_, n in here)
        pools[d] = BlockPool(room, KV_HEADS, DIM, len(here),
                             max(blocks_of(n + steps) for *_, n in here), fmt)
    moved = 0
    for p in sorted({r[1] for r in placed}):
        mine = [r for r in placed if r[1] == p]
        _, pool = prefill(mine, fmt, g)
        for slot, r in enumerate(mine):
            moved += move(pool, slot, pools[r[2]], by_decode[r[2]].index(r))
        if int(pool.status):
            raise RuntimeError(f"prefill instance {p}: status {int(pool.status)}")
    report(f"{len(placed)} requests, {sum(n for *_, n in placed)} tokens; {moved} bytes of blocks "
           f"moved to {len(pools)} decode instances")
    for d, pool in pools.items():
        keep = [max(9, int(blocks_of(t) * budget)) for t in pool.tokens]
        freed = 0
        for step in range(steps):
            row = lambda h: torch.randn((pool.slots, h, DIM), generator=g, device="cuda").bfloat16()  # noqa: E731
            pool.append(row(KV_HEADS), row(KV_HEADS), [1] * pool.slots)
            results[d] = pool.attend(row(HEADS))
            if step % 8 == 7:
                freed += sum(map(len, pool.evict(keep)))
        if int(pool.status):
            raise RuntimeError(f"decode instance {d}: status {int(pool.status)}")
        report(f"decode {d}: {pool.slots} sequences, {sum(pool.tokens)} tokens held after {steps} "
               f"steps, {freed} blocks given up")
    return results, pools


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--format", choices=("int8", "e4m3"), default="int8")
    a = ap.parse_args()
    serve(a.steps, a.format)
