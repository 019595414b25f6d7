"""The 4-bit cache's format from its definition, in 64 bits (numpy, on the CPU): test infrastructure that shares no code
with the kernels. Rows are [.., head dim]; codes [.., head dim / 2], exponents [.., head dim / 32], bytes."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponents(x):
    """The exponent byte of every 32 values: the least e of [-125, 125] with largest < 7 * 2^e, plus 127; NaN: 255."""
    most = np.abs(x.reshape(*x.shape[:-1], -1, 32)).max(-1)
    e = np.full(most.shape, 125)
    for cand in range(124, -126, -1):
        with np.errstate(invalid="ignore"):
            e = np.where(most < 7.0 * 2.0 ** cand, cand, e)
    return np.where(np.isnan(most), 255, e + 127).astype(np.uint8)


def _code(a):
    """The nearest value's code; of two as near the even one."""
    away = np.abs(np.minimum(np.nan_to_num(a, nan=0.0, posinf=8.0), 8.0)[..., None] - VALUES)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    return order[np.argmin(away[..., order], -1)]


def nearest(x):
    """The nearest value of the format to x, in units of a block."""
    return np.copysign(VALUES[_code(np.abs(x))], x)


def quantised(x):
    """Codes and exponents of 64-bit rows."""
    exps = exponents(x)
    unit = np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32, -1)
    with np.errstate(invalid="ignore", over="ignore"):
        code = _code(np.abs(x) / unit) + 8 * np.signbit(x)
    code = np.where(np.repeat(exps, 32, -1) == 255, 0, code).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, exps


def values(codes, exps):
    """What codes and exponents stand for."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    e = np.repeat(exps, 32, -1).astype(np.float64)
    return np.where(e >= 253, np.nan, v * 2.0 ** (e - 127))


def check_stored(codes, exps, x, error, what):
    """Codes and exponents are those of some rows within `error` of x. NaN stands where x has it."""
    got, (lo, hi) = values(codes, exps), (np.maximum(np.abs(x) - error, 0.0), np.abs(x) + error)
    least, most = exponents(lo), exponents(hi)
    assert np.array_equal(exps == 255, np.isnan(x.reshape(*exps.shape, 32)).any(-1)), f"{what}: NaN in other blocks"
    assert np.all((exps >= least) & (exps <= most)), f"{what}: exponents"
    unit = np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32, -1)
    with np.errstate(invalid="ignore", over="ignore"):
        low, high = (nearest((x + d) / unit) * unit for d in (-error, error))
        bad = ~((got >= low) & (got <= high)) & (np.repeat(exps, 32, -1) != 255)
    if bad.any():
        at = tuple(i[0] for i in np.nonzero(bad))
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} values, first at {at}: {got[at]!r} for {x[at]!r}")


def attention(q, k, v, scale, window, sinks):
    """One sequence and one head, causal: query i at position p = m - n + i sees the keys j <= p with j > p - window
    (window 0: all) or j < sinks. The output, the log-sum-exp, and the output for |v|; a row that sees none: 0, -inf."""
    n, m = len(q), len(k)
    out, size, lse = np.zeros((n, v.shape[1])), np.zeros((n, v.shape[1])), np.full(n, -np.inf)
    j = np.arange(m)
    for i in range(n):
        p = m - n + i
        seen = (j <= p) & ((j > p - window) | (j < sinks) if window else True)
        if not seen.any():
            continue
        with np.errstate(invalid="ignore"):
            s = (k[seen] @ q[i]) * scale
            w = np.exp(s - s.max())
            out[i], size[i] = w @ v[seen] / w.sum(), w @ np.abs(v[seen]) / w.sum()
            lse[i] = s.max() + np.log(w.sum())
    return out, lse, size
