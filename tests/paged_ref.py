"""Rotary positions, paged caches and the decode step over them in 64 bits, on the CPU, and bounds on
what float32 arithmetic may add.

Bounds.  A cosine or sine of the kernels: the angle in turns has a rounding of 64-bit numbers, |turns| 2^-51
(three operations), and one to float32, 2^-25 of at most half a turn; times 2 pi, 2^-22.3 and |turns| 2^-48.  The
function itself adds at most 4 units in the last place of numbers up to 1, 2^-22.  So it is off by at most
    c = 2^-21 + |turns| 2^-48,
and an element a cos - b sin by (c + 2 * 2^-24) (|a| + |b|) (two products, a sum: three roundings, two of each
term), plus its last rounding, half a step.

A score's dot product of D products in float32 is off by at most D 2^-24 A, A the largest sum of |q k| times the
scale; the query's own error (turned, not rounded) adds at most dq sum |k|; the scale, the prior, the change to base
two and the exponential add 16 * 2^-24 (|delta| + 8); a query held as two bf16 numbers adds 2^-16 A.  A weight is
off by that relatively, a sum over n rows by n 2^-24 more, and where weights enter a product as two bf16 numbers by
2^-16.  Numerator and denominator carry both, so the output is off by at most 2 delta sum(p |v|), the lse by delta
and 8 roundings of its own; bf16 outputs add half a step.
"""
import math

import numpy as np
import torch

from tests.cached_ref import E4M3, f64, quantise, value_of

GATE_EPS = 1e-4
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative to the value


def frequencies(pairs, theta=1e4):
    i = torch.arange(pairs, dtype=torch.float64)
    return (theta ** (-i / max(1, pairs))).float()


def turned(x, pos, freq, sections, back=False):
    """Rows x [..., D] (float64) at pos [axes, ...]: turned, and how far float32 may be off before its last rounding."""
    y, tol = x.copy(), np.zeros_like(x)
    half, first = x.shape[-1] // 2, 0
    f = f64(freq)
    for axis, n in enumerate(sections):
        for i in range(first, first + n):
            angle = pos[axis].astype(np.float64) * f[i] * (-1.0 if back else 1.0)
            c, s = np.cos(angle), np.sin(angle)
            a, b = x[..., i], x[..., half + i]
            y[..., i], y[..., half + i] = a * c - b * s, a * s + b * c
            off = 2.0 ** -21 + np.abs(angle) / (2 * math.pi) * 2.0 ** -48 + 2.0 ** -23
            tol[..., i] = tol[..., half + i] = off * (np.abs(a) + np.abs(b))
        first += n
    return y, tol


def rounded_tol(y, tol, dtype):
    """The bound once the value is rounded to dtype (bf16 and float32: half a step of what it may be)."""
    return tol + HALF[dtype] * (np.abs(y) + tol)


class Cache:
    """Pages and a table on the GPU, and the float64 values that they hold."""

    def __init__(self, S, Hk, D, page, max_pages, dtype, quantised, seed, spare=2, extra=0.0):
        g = torch.Generator().manual_seed(seed)
        self.S, self.Hk, self.D, self.page, self.max_pages = S, Hk, D, page, max_pages
        n = S * max_pages + spare
        rows = [torch.randn(n, Hk, page, D, generator=g) * (1 + extra * torch.rand(n, Hk, page, 1, generator=g)) for _ in range(2)]
        self.table = torch.randperm(n, generator=g, dtype=torch.int32)[:S * max_pages].view(S, max_pages).cuda()
        self.k_exp = self.v_exp = None
        if quantised:
            (kc, ke), (vc, ve) = (quantise(x) for x in rows)
            self.k, self.v = (torch.from_numpy(c).float().to(E4M3).cuda() for c in (kc, vc))
            self.k_exp, self.v_exp = (torch.from_numpy(e).cuda() for e in (ke, ve))
        else:
            self.k, self.v = (x.to(dtype).cuda() for x in rows)

    def args(self):
        return dict(k_exp=self.k_exp, v_exp=self.v_exp)

    def tensors(self):
        return [t for t in (self.k, self.v, self.k_exp, self.v_exp) if t is not None]

    def values(self):
        """float64 keys and values [pages, Hk, page, D]."""
        if self.k_exp is None:
            return f64(self.k), f64(self.v)
        return value_of(self.k, self.k_exp), value_of(self.v, self.v_exp)

    def entry(self, s, j):
        """Page of position j of sequence s, or -1."""
        if not 0 <= j < self.page * self.max_pages:
            return -1
        e = int(self.table[s, j // self.page])
        return e if 0 <= e < self.k.shape[0] else -1


class PagedStep:
    """One step over the cache as it is after the step (the new rows in their places): out, lse and their bounds."""

    def __init__(self, cache, lens, q, gate, k, pi, clamp=0.0, freq=None, sections=None, pos=None, two_terms=False):
        S, H, D = q.shape
        G = H // cache.Hk
        dtype = q.dtype
        keys, vals = cache.values()
        qq, gate = f64(q), np.broadcast_to(f64(gate), (S, H))
        lens = [int(x) for x in lens]
        dq = np.zeros_like(qq)
        if freq is not None:
            at = np.array([lens] * len(sections)) if pos is None else np.asarray(pos.cpu()).reshape(len(sections), S)
            qq, dq = turned(qq, np.repeat(at[:, :, None], H, 2), freq, sections)
        self.out, self.out_tol = np.full((S, H, D), np.nan), np.zeros((S, H, D))
        self.lse, self.lse_tol = np.full((S, H), np.nan), np.zeros((S, H))
        scale = 1 / math.sqrt(D)
        for s, t in enumerate(lens):
            if cache.entry(s, t) < 0:
                continue
            w = [(j, 0) for j in range(max(0, t - k), t + 1)] + ([(t - pi, 1)] if pi > k and t >= pi else [])
            w = [(j, c, cache.entry(s, j)) for j, c in w if cache.entry(s, j) >= 0]
            kk = np.stack([keys[e, :, j % cache.page] for j, _, e in w], 1)     # [Hk, n, D]
            vv = np.stack([vals[e, :, j % cache.page] for j, _, e in w], 1)
            partner = np.array([c for _, c, _ in w])
            for h in range(H):
                a = GATE_EPS + (1 - 2 * GATE_EPS) / (1 + math.exp(-gate[s, h]))
                prior = np.where(partner == 1, math.log(1 - a), math.log(a))
                K, V = kk[h // G], vv[h // G]
                d = K @ qq[s, h] * scale + prior
                A = np.max(np.abs(K) @ np.abs(qq[s, h])) * scale
                B = np.max(np.abs(K) @ dq[s, h]) * scale
                if clamp > 0:
                    d = np.clip(d, -clamp, clamp)
                m = d.max()
                p = np.exp(d - m)
                self.lse[s, h] = m + math.log(p.sum())
                p /= p.sum()
                self.out[s, h] = p @ V
                delta = 2.0 ** -24 * (D * A + 16 * (np.abs(d).max() + 8) + len(w)) + B
                if two_terms:
                    delta += 2.0 ** -16 * (A + 1)
                tol = 2 * delta * (p @ np.abs(V))
                self.out_tol[s, h] = rounded_tol(self.out[s, h], tol, dtype)
                self.lse_tol[s, h] = delta + 8 * 2.0 ** -24 * abs(self.lse[s, h])

    def check(self, out, lse=None):
        out = f64(out)
        assert np.array_equal(np.isnan(out), np.isnan(self.out))
        if not np.isnan(out).all():
            worst = np.nanmax(np.abs(out - self.out) - self.out_tol)
            assert worst <= 0, worst
        if lse is not None:
            lse = f64(lse)
            assert np.array_equal(np.isnan(lse), np.isnan(self.lse))
            if not np.isnan(lse).all():
                worst = np.nanmax(np.abs(lse - self.lse) - self.lse_tol)
                assert worst <= 0, worst
