"""Element by element bounds of attention's bf16 outputs, from the 64-bit form, which do not
loosen where an output is the mean of many rows.

With p_j a row's probability and half a step of bf16 2^-8 of a value, P is rounded once, so
that every p_j is off by 2^-8 p_j at most (the sum that divides it is not rounded), and the
result is rounded once.  With A_d = sum_j p_j |v_jd| an element is off by at most
  2^-8 A_d + 2^-8 (|out_d| + 2^-8 A_d) + (n + 64 D) 2^-24 A_d,
the last for fp32: a sum of n products of weights and values, and weights relatively off by
twice a logit's error, which is D 2^-24 of scale sum_i |q_i k_ji| (some 7 for rows ~ N(0, 1)
at D = 128, and below 16).

Rounding errors of many rows are independent.  Relatively to a value they are spread evenly
over +-2^-8 / m for a mantissa m in [1, 2), 2^-8 / sqrt(6) in the root of their mean square:
2^-9.3, less than c = 2^-9.  So where no few rows have most of the weight (sum_j p_j^2 below
1 / 200), the error's root mean square over a unit's heads and columns is within twice
  c sqrt(mean_d(sum_j p_j^2 v_jd^2 + out_d^2)):
at 9,677 rows 9e-5, where a tile of 32 rows of V in the wrong order moves outputs by 1.4e-3."""
from __future__ import annotations

import math

import torch

from paged_helpers import sees

HALF = 2.0 ** -8
C = 2.0 ** -9


class Expected:
    """What queries q [G][D] of the token at row pos over rows k, v [n][D] give in 64 bits:
    out, lse and the errors that they may have."""

    def __init__(self, k, v, q, pos, scale, sinks=0, window=0):
        ok = sees(k.shape[0], pos, sinks, window)
        k, v, q = k[ok].double(), v[ok].double(), q.double()
        x = (q @ k.T) * scale
        self.lse = torch.logsumexp(x, -1)
        p = torch.exp(x - self.lse[:, None])
        self.out = p @ v
        A = p @ v.abs()
        n, D = k.shape
        self.most = HALF * A + HALF * (self.out.abs() + HALF * A) + (n + 64 * D) * 2.0 ** -24 * A
        self.rms = None
        if (p * p).sum(-1).max() < 1 / 200:
            self.rms = 2 * C * math.sqrt(((p * p) @ (v * v) + self.out ** 2).mean().item())

    def check(self, got, what):
        """Raises AssertionError where got [G][D] is not within the bounds."""
        err = (got.double() - self.out).abs()
        over = (err - self.most).max().item()
        assert over <= 0, f"{what}: an element is off by {over:.3e} more than it may be"
        if self.rms is not None:
            r = err.square().mean().sqrt().item()
            assert r <= self.rms, f"{what}: off by {r:.3e} (root mean square), allowed {self.rms:.3e}"
