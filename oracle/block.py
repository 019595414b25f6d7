"""The attention block's operators from their definitions, in 64 bits (numpy, on the CPU): test infrastructure
that shares no code with the kernels.

Pools are [pages, kv heads, page size, head dim]; rows are [T, heads * head dim].
"""
from __future__ import annotations

import numpy as np
import torch


def rope_frequencies(rot, base=10000.0, factor=1.0, low=0.0, high=0.0, original=0.0):
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    share = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0) if high > low else np.zeros_like(f)
    return f * (share + (1.0 - share) / factor)


def rope_table(n_pos, rot, magnitude=1.0, **scaling):
    angle = np.arange(n_pos)[:, None] * rope_frequencies(rot, **scaling)
    return np.stack([np.cos(angle), np.sin(angle)], -1) * magnitude


def normed(x, w, partials, d_full, eps):
    """Phases B+C of the norm: x [T, d], partials [tp, T]."""
    return x * w / np.sqrt(partials.sum(0) / d_full + eps)[:, None]


def rotated(z, table, pos, D, rot, interleaved):
    """(rotated rows, the scale of each element's rounding errors): z [T, heads * D]."""
    T = z.shape[0]
    out = z.reshape(T, -1, D).copy()
    size = np.abs(out)
    for i in range(rot // 2):
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = table[pos, i, 0][:, None], table[pos, i, 1][:, None]
        a, b = out[..., ia].copy(), out[..., ib].copy()
        out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
        size[..., ia], size[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return out.reshape(z.shape), size.reshape(z.shape)


def attention(q, k, v, scale, causal=True, window=0):
    """One sequence and one head: q [n, D], k and v [m, D], query i at position m - n + i. Returns the output and
    the log-sum-exp; a query that sees no key has zeros and -inf. Keys that a query does not see take no part,
    whatever they hold."""
    n, m = len(q), len(k)
    out, lse = np.zeros((n, v.shape[1])), np.full(n, -np.inf)
    for i in range(n):
        at = m - n + i
        hi = min(m, at + 1) if causal else m
        lo = max(0, at - window + 1) if window else 0
        if lo >= hi:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = (k[lo:hi] @ q[i]) * scale
            top = s.max()
            if top == -np.inf:
                continue
            p = np.exp(s - top)
            out[i] = p @ v[lo:hi] / p.sum()
            lse[i] = top + np.log(p.sum())
    return out, lse


def adapted(base, x, a, b, ids, scale):
    """base + scale_i B_i A_i x, and the absolute sum of what is added to it: base [T, d], a [n, r, h], b [n, d, r]."""
    y, size = base.copy(), np.abs(base)
    for t in range(len(x)):
        i = ids[t]
        if i >= 0:
            inner = a[i] @ x[t]
            y[t] += scale[i] * (b[i] @ inner)
            size[t] += abs(scale[i]) * (np.abs(b[i]) @ (np.abs(a[i]) @ np.abs(x[t])))
    return y, size


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def _fp8(x):
    return torch.from_numpy(np.clip(x, -448.0, 448.0)).float().to(torch.float8_e4m3fn).double().numpy()


def check_rounded(got, ref, error, fmt, what):
    """Every value of `got` is the nearest bf16 value ("bf16"), or saturated e4m3fn value ("fp8"), of some value
    within `error` of `ref`. NaN stands where the reference has it."""
    got, ref, error = (np.asarray(z, dtype=np.float64) for z in (got, ref, error))
    to = _bf16 if fmt == "bf16" else _fp8
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    with np.errstate(invalid="ignore"):
        bad = ~((got >= to(ref - error)) & (got <= to(ref + error))) & ~np.isnan(ref)
    if bad.any():
        at = tuple(i[0] for i in np.nonzero(bad))
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} values, first at {at}: {got[at]!r} for {ref[at]!r} "
                             f"+- {np.broadcast_to(error, ref.shape)[at]!r}")
