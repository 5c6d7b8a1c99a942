"""Attention rows in 64 bits with bounds that scale with the softmax weights, for a ``Case`` of kv_support."""

import math

import torch

from tests.kv_support import UNIT


def visible(case, b, causal=True, window=0, hidden=()):
    """Which positions each new token of request ``b`` sees; ``hidden``: positions that nobody does."""
    n, kv = case.lens[b]
    p, j = torch.arange(n, device="cuda") + kv - n, torch.arange(kv, device="cuda")
    seen = torch.ones((n, kv), dtype=torch.bool, device="cuda")
    if causal:
        seen &= j[None] <= p[:, None]
    if window:
        seen &= j[None] > p[:, None] - window
    seen[:, list(hidden)] = False
    return seen


def worst(case, out, lse, b, scale=None, causal=True, window=0, hidden=()):
    """The largest error of request ``b`` in units of its bound, which is, with u the unit roundoff of the type, w the softmax
    weights and e_j = (D + 6) 2^-24 |scale| sum_d |q_d k_jd| (the FP32 score):  u |o| for the result's rounding,
    (u + 2 max e + 2^-18) sum w |v| for the weights' rounding, scores, exp and sum, and in FP16 2^-32 max(w) per position: a
    weight is held as 2^(s - m + 7), at least 2^7 for the largest, and below 2^-14 is off by 2^-25 absolutely."""
    u, f64 = UNIT[case.dt], torch.float64
    half = case.dt == torch.float16
    scale = case.D ** -0.5 if scale is None else scale
    kv, G = case.lens[b][1], case.Hq // case.Hkv
    rows = slice(int(case.off[b]), int(case.off[b + 1]))
    seen = visible(case, b, causal, window, hidden)
    some = seen.any(1)
    most = 0.0
    for h in range(case.Hq):
        q, k, v = case.q[rows, h].to(f64), case.keys[b][:, h // G].to(f64), case.values[b][:, h // G].to(f64)
        e = torch.where(seen, (case.D + 6) * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().T), 0.0).amax(1)
        s = (q @ k.T * scale).masked_fill(~seen, -math.inf)
        z = torch.logsumexp(s, 1)
        w = torch.exp(s - torch.where(some, z, 0.0)[:, None])
        ref = w @ v
        tol = u * ref.abs() + (u + 2 * e + 2.0 ** -18)[:, None] * (w @ v.abs())
        if half:
            tol = tol + (kv * 2.0 ** -32 * w.amax(1) * v.abs().max())[:, None] + 2.0 ** -25
        got = out[rows, h].to(f64)
        assert (got[~some] == 0).all()
        most = max(most, float(((got - ref).abs()[some] / tol[some]).max()))
        if lse is not None:
            d = (lse[rows, h].to(f64) - z).abs()[some]
            most = max(most, float((d / (e + 2.0 ** -20 * (1 + z.abs()) + kv * 2.0 ** -24)[some]).max()))
            assert (lse[rows, h][~some] == -math.inf).all()
    return most
