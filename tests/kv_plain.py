"""The KV-block operators from their definitions in 64 bits, on the CPU, for the tests: one
sequence, head and block at a time."""
import math

import numpy as np
import torch

BLOCK = 16
TOP = {"int8": 127.0, "e4m3": 448.0}
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # unit roundoff


def attention(q, k, v, scale, see):
    """One head: q [m, d], k, v [n, d] float64, see [m, n].  Output, lse, weights, and what the
    rounding bounds go by: sum p |v| and the largest sum scale |q| |k|."""
    s = (q @ k.T) * scale
    size = float(((q.abs() @ k.abs().T) * scale).max()) if s.numel() else 0.0
    s = torch.where(see, s, torch.full_like(s, -math.inf))
    m = s.amax(1, keepdim=True) if s.shape[1] else torch.full((len(q), 1), -math.inf, dtype=s.dtype)
    e = torch.where(see, torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m)),
                    torch.zeros_like(s))
    t = e.sum(1, keepdim=True)
    p = torch.where(t > 0, e / t.clamp_min(1e-300), torch.zeros_like(e))
    lse = torch.where(t > 0, m + t.log(), torch.full_like(t, -math.inf))[:, 0]
    hidden = ~see.any(0)
    v = torch.where(hidden[:, None], torch.zeros_like(v), v)
    return p @ v, lse, p, p @ v.abs(), size


def score_error(size, dim):
    """A score's error: a sum of dim products in fp32, its scaling, and the exponential."""
    return (dim + 8) * 2.0 ** -24 * size + 2.0 ** -20


def close_out(got, want, weight, size, dim, dtype, weight_unit, slack=0.0):
    """got against the exact output: its own rounding, the weights' rounding, and the scores'
    error, which moves a weight and the sum it is divided by."""
    tol = U[dtype] * want.abs() + (weight_unit + 2.0 ** -18 + 2 * score_error(size, dim)) * \
        (1 + U[dtype]) * weight + slack + 1e-7
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all()
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))


def close_lse(got, want, size, dim):
    inf = want == -math.inf
    assert (got.double()[inf] == -math.inf).all()
    err = (got.double() - want).abs()[~inf]
    assert (err <= score_error(size, dim) + 2.0 ** -22 * want[~inf].abs() + 2.0 ** -19).all(), \
        float(err.max())


def codes_value(codes):
    """int8 or e4m3 codes (any device) as float64 on the CPU."""
    return codes.cpu().float().double()


def e4m3(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.float8_e4m3fn).float().numpy()


def to_codes(x, fmt):
    """fp32 values already divided by the scale, to the values of their codes."""
    top = np.float32(TOP[fmt])
    x = np.clip(x.astype(np.float32), -top, top)
    return np.rint(x) if fmt == "int8" else e4m3(x)


def store_block(old_codes, old_scale, lead, rows, fmt):
    """One block of one head by the definition, whose steps are in fp32: old codes [16, dim] as
    values, `lead` of them in use, then the new rows.  New codes (as values) and the scale."""
    f = np.float32
    out = np.array(old_codes, np.float32)
    x = np.where(np.isfinite(rows), rows, 0).astype(f)
    largest = np.abs(x).max() if x.size else f(0)
    fresh = f(0) if largest < f(2.0 ** -100) else f(largest) / f(TOP[fmt])
    was = f(old_scale) if lead else f(0)
    now = max(was, fresh)
    if lead and now > was:
        out[:lead] = to_codes(out[:lead] * (was / now), fmt)
    inv = f(1) / now if now > 0 else f(0)
    out[lead:lead + len(x)] = to_codes(x * inv, fmt)
    return out, now


def evict(length, table, mass, budget, sink, recent):
    """One sequence: (table, mass, length, freed) after eviction, as lists."""
    n = -(-length // BLOCK)
    gone = max(0, n - max(budget, sink + recent))
    between = range(sink, n - recent) if gone else []
    first = sorted(between, key=lambda j: (math.isnan(mass[j]), 0.0 if math.isnan(mass[j]) else mass[j], j))
    out = set(first[:gone])
    stay = [j for j in range(n) if j not in out]
    return ([table[j] for j in stay], [mass[j] for j in stay], length - BLOCK * gone,
            [table[j] for j in sorted(out)])
