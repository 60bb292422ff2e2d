"""Rows of 8-bit codes, the norm in front of a layer and the product on codes, from their definitions (numpy; shares no code with the
library).  Steps that the definitions round to fp32 are single fp32 operations here too, everything else is in 64 bits."""
import numpy as np
import torch

import act_reference

F = np.float32


def pitch(cols):
    return -(-cols // 16) * 16


def scales(v):
    """(scale, 1 / scale) of fp32 rows; NaN for a row that is not finite."""
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(v).max(1)
    bad = ~np.isfinite(v).all(1)
    s = np.maximum(np.where(bad, F(0), top).astype(F) / F(127), F(2.0 ** -126))
    return np.where(bad, F(np.nan), s).astype(F), (F(1) / s).astype(F)


def encode(v, draws=None):
    """(codes int8 [rows][pitch], scales) of fp32 rows; draws: (seed, epoch, tag), none for the nearest code."""
    v = np.ascontiguousarray(v, dtype=F)
    rows, cols = v.shape
    s, inverse = scales(v)
    with np.errstate(invalid="ignore", over="ignore"):
        t = (v * inverse[:, None]).astype(F)
        if draws is None:
            c = np.rint(t)
        else:
            k = act_reference.draws(rows, -(-cols // 8) * 8, *draws)[:, :cols]
            c = np.clip(np.floor((t + ((k + 0.5) / 65536.0).astype(F)).astype(F)), -127, 127)
    out = np.zeros((rows, pitch(cols)), np.int8)
    out[:, :cols] = np.where(np.isnan(s)[:, None], 0, np.where(np.isfinite(c), c, 0)).astype(np.int8)
    return out, s


def decode(codes, s, cols):
    return (codes[:, :cols].astype(F) * s[:, None]).astype(F)


def norm(x, add, gain, eps):
    """(r, rstd, v) for torch rows x and add (or None); gain fp32 or None."""
    r = x if add is None else (x.float() + add.float()).to(x.dtype)
    r = r.float().numpy()
    with np.errstate(all="ignore"):
        square = (r.astype(np.float64) ** 2).sum(1) / r.shape[1]
        rstd = (1.0 / np.sqrt(square + float(F(eps)))).astype(F)
        v = (r * rstd[:, None]).astype(F)
        if gain is not None:
            v = (v * gain[None]).astype(F)
    return r, rstd, v


def norm_gradients(dy, r, rstd, gain, dsum):
    """(dx, dgain, what their fp32 evaluation may be off by in units of 2^-24) in 64 bits.

    dx: a and n are rounded once or twice, mean(a n) is a sum of fp32 products over at most 8 * 32 values of a thread (512 of a row of
    more than 32,768 values in these tests), 6 steps in the wave and 16 over the waves, then a division; each step is off by 2^-24 of
    what it adds up.  dgain: a product, n's own rounding, and a chain of at most rows / 1024 + 1 rows, 3 waves, 64 workgroups of a
    wave's and 16 waves (100 is more than the last three)."""
    dy, r, rstd = dy.astype(np.float64), r.astype(np.float64), rstd.astype(np.float64)[:, None]
    g = np.ones(r.shape[1]) if gain is None else gain.astype(np.float64)
    n, a = r * rstd, dy * g
    along = (a * n).mean(1, keepdims=True)
    dx = rstd * (a - n * along)
    size = np.abs(dx)
    if dsum is not None:
        dx = dx + dsum
        size = size + np.abs(dsum)
    off_dx = 2 * size + np.abs(rstd) * (4 * np.abs(a) + np.abs(n) * 600 * np.abs(a * n).mean(1, keepdims=True))
    return dx, (dy * n).sum(0), off_dx, (r.shape[0] // 1024 + 100) * np.abs(dy * n).sum(0)


def product(x, w, sx, sw, bias, dtype):
    """Bit for bit: x, w int8 [rows][d_in] arrays."""
    total = (torch.from_numpy(x).double() @ torch.from_numpy(w).double().t()).numpy()      # exact: below 2^53
    with np.errstate(all="ignore"):
        v = total.astype(np.int64).astype(F)
        v = ((v * sx[:, None]).astype(F) * sw[None]).astype(F)
        if bias is not None:
            v = (v + bias[None]).astype(F)
    return torch.from_numpy(v).to(dtype)
