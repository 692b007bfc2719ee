"""Plain 64-bit form of the rotation by positions (CPU) and its tolerances.

Tolerances.  A position times a frequency is formed in 64 bits and reduced to a turn
r in [-1/2, 1/2] there: off by 3 * 2^-53 of the turns' number.  r is rounded to fp32
(2^-26 at most, 2 pi 2^-26 = 9.4e-8 of an angle), and sine and cosine of it are within
2 ulp (1.2e-7), so each is off by d = 2.2e-7 + 2 pi 3 2^-53 |turns|.  x c - y s then has
two fp32 roundings, 2^-24 of |x| + |y| each: together an element is off by
  (d + 2^-23) (|x| + |y|),
and in bf16 half a step, 2^-8, of the result more."""
from __future__ import annotations

import math

import numpy as np
import torch


def ends(rot, pairs):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)


def turned(x, pos, freq, axes=None, pairs=False):
    """x [NL][B][H][T][D], pos [n_axes][B][T], freq [rot / 2]: the rotated rows in 64 bits and what
    each element may be off by."""
    rot, half = 2 * freq.numel(), 2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0
    of = torch.zeros(freq.numel(), dtype=torch.int64) if axes is None else torch.tensor(list(axes))
    turns = pos.long()[of].permute(1, 2, 0).numpy().astype(np.longdouble) * freq.numpy().astype(np.longdouble)
    turns = turns / (2 * np.longdouble("3.14159265358979323846264338327950288"))
    left = torch.from_numpy(np.asarray(turns - np.rint(turns), dtype=np.float64)) * (2 * math.pi)
    c, s = left.cos()[:, None], left.sin()[:, None]
    d = (2.2e-7 + 6 * math.pi * 2.0 ** -53 * torch.from_numpy(np.abs(turns).astype(np.float64)) + 2.0 ** -23)[:, None]
    y, off = x.double(), torch.zeros(x.shape, dtype=torch.float64)
    a, b = ends(rot, pairs)
    g, o = y[..., a], y[..., b]
    y[..., a], y[..., b] = g * c - o * s, g * s + o * c
    off[..., a] = off[..., b] = d * (g.abs() + o.abs())
    off[..., :rot] += half * (y[..., :rot].abs() + off[..., :rot])
    return y, off


def close_rows(got, ref, off, what):
    if not ref.numel():
        return
    over = (got.double() - ref).abs() - off
    assert not torch.isnan(over).any() and over.max().item() <= 0, f"{what}: off by {over.max().item():.3e} more than it may be"


def frequencies(rot, base=1e4):
    n = rot // 2
    return torch.from_numpy((base ** (-np.arange(n) / n)).astype(np.float32))


def memory_orders(shape, dtype, g):
    """Tensors of this shape [NL][B][H][T][D] in the orders that programs have them in."""
    NL, B, H, T, D = shape

    def randn(*s):
        return torch.randn(s, generator=g).to(dtype)
    yield "as the kernels", randn(*shape)
    yield "heads of a token beside each other", randn(NL, B, T, H, D).transpose(2, 3)
    yield "behind others in a projection", randn(NL, B, T, H + 3, D)[:, :, :, 2:2 + H].transpose(2, 3)
    yield "tokens first", randn(T, B, NL, H, 2, D)[:, :, :, :, 1].permute(2, 1, 3, 0, 4)
