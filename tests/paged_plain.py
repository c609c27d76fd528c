"""Attention over windows and paged caches in plain fp64 on the CPU, and how far fp32 / bf16 arithmetic may be off it."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


def sees(pos, n_keys, window, sinks):
    """[rows, keys] truth values; window 0: all keys up to the row."""
    j = torch.arange(n_keys)
    d = pos[:, None] - j[None, :]
    ok = d >= 0
    if window:
        ok &= (d < window) | (j[None, :] < sinks)
    return ok


def attend(q, k, v, pos, window, sinks, scale=None, valid=None):
    """q [G, n, D] of one kv-head at positions pos, k, v [m, D]; valid [m]: keys that count at all.
    (o, lse [G, n], got [m] per-row-summed weights) in fp64, and what each may be off by in the kernels' arithmetic."""
    dtype, D = q.dtype, q.shape[-1]
    scale = 1.0 / math.sqrt(D) if not scale else scale
    q, k, v = q.double(), k.double(), v.double()
    ok = sees(pos, k.shape[0], window, sinks)
    if valid is not None:
        ok = ok & valid[None, :]
    s = (q @ k.T * scale).masked_fill(~ok, -math.inf)
    m = s.amax(-1, keepdim=True) if k.shape[0] else torch.full(q.shape[:-1] + (1,), -math.inf, dtype=torch.float64)
    none = m == -math.inf
    e = torch.exp(s - m.masked_fill(none, 0.0))
    z = e.sum(-1, keepdim=True)
    w = e / z.masked_fill(none, 1.0)
    o = w @ v
    lse = (m + z.log()).squeeze(-1)
    # A score is a sum of D products in fp32, each sum off by a step of what it has reached at most: (D + 8) 2^-23 of the sum of
    # the products' sizes, and as much again of the scaled value for the products with the scale and the exponent reference.
    size = (q.abs() @ k.abs().T * scale).masked_fill(~ok, 0.0).amax((-1,), keepdim=True) if k.shape[0] else torch.zeros_like(m)
    off_s = (D + 8) * 2.0 ** -23 * size + 2.0 ** -21 * (size + 1)
    # sums over keys: a lane adds up at most every fourth key, then joins 64 states at most, a step each
    off_sum = (k.shape[0] / 4 + 64) * 2.0 ** -23
    rel = 2 * off_s + off_sum                                   # of a probability: its own exponent's and the sum's
    p_round = HALF[torch.bfloat16] if dtype == torch.bfloat16 else 0.0
    tol_o = HALF[dtype] * o.abs() + (rel + p_round) * (w @ v.abs()) * (1 + HALF[dtype]) + 1e-30
    tol_lse = (off_s + off_sum).squeeze(-1) + 2.0 ** -22 * lse.masked_fill(none.squeeze(-1), 0.0).abs()
    got, tol_got = w.sum((0, 1)), (w * (rel + off_sum)).sum((0, 1)) + q.shape[0] * q.shape[1] * 2.0 ** -23 * w.sum((0, 1)) + 1e-30
    return o, lse, got, tol_o, tol_lse, tol_got


def close(x, ref, tol, what):
    x, ref = x.double().cpu(), ref
    assert x.shape == ref.shape, (what, x.shape, ref.shape)
    gone = torch.isinf(ref)
    assert torch.equal(x[gone], ref[gone]), what
    off = ((x - ref).abs() - tol)[~gone]
    assert not torch.isnan(off).any(), f"{what}: NaN"
    if off.numel():
        assert off.max() <= 0, f"{what}: {float((x - ref)[~gone].abs().max()):.3e} off, {float(off.max()):.3e} more than it may be"
