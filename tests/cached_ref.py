"""The quantised caches and the cached decode steps in 64 bits, on the CPU, and
bounds on what float32 arithmetic may add.

Bounds.  A score's dot product of D products in float32 is off by at most
D 2^-24 A, A the largest sum of |q k| times the scale; the scale, the prior, the
change to base two and the exponential add a few roundings of values up to the
largest logit: 16 * 2^-24 (|delta| + 8).  A weight is off by that relatively, a
sum over n rows by n 2^-24 more.  Numerator and denominator of the output carry
both, so it is off by at most 2 delta sum(p |v|), with
    delta = 2^-24 (D A + 16 (max |delta| + 8) + n),
and the lse by delta and 8 roundings of its own.  bf16 outputs add half a step,
2^-8 |out|; weights that are rounded to bf16 add 2^-8 of sum(p |v|).
"""
import math

import numpy as np
import torch

GATE_EPS = 1e-4
E4M3 = torch.float8_e4m3fn


def quantise(x):
    """Codes (float64, NaN for what is not finite) and scale bytes of rows [..., D], by the definition."""
    x = x.detach().cpu().double().numpy()
    fin = np.isfinite(x)
    amax = np.where(fin, np.abs(x), 0.0).max(-1)
    e = np.maximum(np.frexp(amax / 448)[1].astype(np.int64) - 3, -126)   # below the least one
    e = np.where(amax > 0, e, -126)
    while (short := amax > np.ldexp(448.0, e)).any():
        e = e + short
    y = np.ldexp(np.where(fin, x, 0.0), -e[..., None])
    exponent = np.maximum(np.frexp(np.abs(y))[1] - 1, -6)       # of the value; subnormals share that of 2^-6
    step = np.ldexp(1.0, exponent - 3)
    codes = np.rint(y / step) * step                            # halves to even
    return np.where(fin, codes, np.nan), (e + 127).astype(np.uint8)


def value_of(codes, byte):
    """float64 values of a cache's rows."""
    c = codes.detach().cpu().view(torch.uint8).view(E4M3).float().double().numpy()
    return np.ldexp(c, byte.detach().cpu().numpy().astype(np.int64)[..., None] - 127)


def f64(x):
    return x.detach().cpu().double().numpy()


class Step:
    """One step: out, lse and their bounds [S, H, D], [S, H] for rows of each sequence given as float64 [H, rows, D], the
    new one last; `own_from`: the position from which on rows lie in the own cache (for the bound of rounded weights)."""

    def __init__(self, q, gate, k, pi, clamp, rows, dtype, rounded_below):
        S, H, D = q.shape
        q, gate = f64(q), f64(gate)
        gate = np.broadcast_to(gate, (S, H))
        self.out, self.out_tol = np.full((S, H, D), np.nan), np.zeros((S, H, D))
        self.lse, self.lse_tol = np.full((S, H), np.nan), np.zeros((S, H))
        scale = 1 / math.sqrt(D)
        for s in range(S):
            if rows[s] is None:
                continue
            kk, vv = rows[s]
            t = kk.shape[1] - 1
            lo = max(0, t - k)
            w = list(range(lo, t + 1)) + ([t - pi] if pi > k and t >= pi else [])
            for h in range(H):
                a = GATE_EPS + (1 - 2 * GATE_EPS) / (1 + math.exp(-gate[s, h]))
                prior = np.array([math.log(a)] * (t + 1 - lo) + [math.log(1 - a)] * (len(w) - (t + 1 - lo)))
                d = kk[h, w] @ q[s, h] * scale + prior
                A = np.nanmax(np.abs(kk[h, w]) @ np.abs(q[s, h])) * scale
                if clamp > 0:
                    d = np.clip(d, -clamp, clamp)
                m = d.max()
                p = np.exp(d - m)
                self.lse[s, h] = m + math.log(p.sum())
                p /= p.sum()
                self.out[s, h] = p @ vv[h, w]
                size = p @ np.abs(vv[h, w])
                delta = 2.0 ** -24 * (D * A + 16 * (np.abs(d).max() + 8) + len(w))
                tol = 2 * delta * size
                if dtype == torch.bfloat16:
                    in_prefix = np.array([lo <= j < min(rounded_below, t - 0) and i <= t - lo for i, j in enumerate(w)])
                    tol = tol + 2.0 ** -8 * (p * in_prefix) @ np.abs(vv[h, w]) + 2.0 ** -8 * np.abs(self.out[s, h])
                else:
                    tol = tol + 2.0 ** -24 * np.abs(self.out[s, h])
                self.out_tol[s, h] = tol
                self.lse_tol[s, h] = delta + 8 * 2.0 ** -24 * abs(self.lse[s, h])

    def check(self, out, lse=None):
        out = f64(out)
        assert np.array_equal(np.isnan(out), np.isnan(self.out))
        worst = np.nanmax(np.abs(out - self.out) - self.out_tol)
        assert worst <= 0, worst
        if lse is not None:
            lse = f64(lse)
            assert np.array_equal(np.isnan(lse), np.isnan(self.lse))
            worst = np.nanmax(np.abs(lse - self.lse) - self.lse_tol)
            assert worst <= 0, worst
