"""Plain implementations of the norm, of the 8- and 4-bit rows and of the policy loss, for the tests: torch on
the CPU, sums in 64 bits, the roundings that the definitions name in 32."""
from __future__ import annotations

import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def normed(x, residual, gain, eps):
    """(y fp32, h) of rows x: h in the residual's type, or x."""
    h = x if residual is None else (x.float() + residual.float()).to(residual.dtype)
    r = (1.0 / (h.double().square().mean(dim=1, keepdim=True) + eps).sqrt()).float()
    return (h.float() * r) * gain.float(), h


def rows8(y):
    """(e4m3 [M, D], scales [ceil(D/128), M]) of fp32 rows."""
    q = torch.empty(y.shape, dtype=torch.float8_e4m3fn)
    scales = []
    for k in range(0, y.shape[1], 128):
        part = y[:, k:k + 128]
        s = torch.nan_to_num(part.abs(), nan=0.0, posinf=math.inf).amax(dim=1) * torch.tensor(1 / 448, dtype=torch.float32)
        s[s == 0] = 1.0
        q[:, k:k + 128] = (part / s[:, None]).to(torch.float8_e4m3fn)
        scales.append(s)
    return q, torch.stack(scales)


def nearest4(u):
    """Codes 0..7 of the nearest grid value of |u|, of two as near the even code."""
    off = np.abs(np.minimum(np.abs(u), 6.0)[..., None] - GRID)
    best = off.min(axis=-1, keepdims=True)
    near = off == best
    first = near.argmax(axis=-1)
    return np.where((near.sum(axis=-1) == 2) & (first % 2 == 1), first + 1, first)


def rows4(y):
    """(codes [M, D], block scales fp32 [M, ceil(D/16)], row scales [M]) of finite fp32 rows."""
    f32 = dict(dtype=torch.float32)
    M, D = y.shape
    row = torch.maximum(y.abs().amax(dim=1) * torch.tensor(1 / 2688, **f32), torch.tensor(2.0 ** -100, **f32))
    blocks = torch.nn.functional.pad(y, (0, -D % 16)).view(M, -1, 16)
    t = blocks.abs().amax(dim=2) / row[:, None] * torch.tensor(1 / 6, **f32)
    s = t.clamp(max=448).to(torch.float8_e4m3fn).float()
    step = s * row[:, None]
    u = (blocks * torch.where(step > 0, 1.0 / step, torch.zeros(()))[:, :, None]).view(M, -1)[:, :D].numpy()
    code = nearest4(u) | (np.signbit(u) * 8)
    return code.astype(np.uint8), s, row


def unpack4(q, scales, row_scales, D):
    """(codes [M, D], block scales [M, ceil(D/16)], what lies behind D) of packed rows."""
    q, scales = q.cpu(), scales.cpu().view(torch.uint8)
    M = q.shape[0]
    code = torch.stack([q & 15, q >> 4], dim=2).flatten(1)
    r, b = torch.arange(M)[:, None], torch.arange(scales.shape[1] * 4)[None, :]
    s = scales[r // 128, b // 4, r % 32, r % 128 // 32, b % 4]
    n = (D + 15) // 16
    return code[:, :D].numpy(), s[:, :n].contiguous().view(torch.float8_e4m3fn).float(), (code[:, D:], s[:, n:])


def values4(q, scales, row_scales, D):
    """Packed rows' values in 64 bits, on their device."""
    M = q.shape[0]
    code = torch.stack([q & 15, q >> 4], dim=2).flatten(1)[:, :D].long()
    grid = torch.tensor(np.concatenate([GRID, -GRID]), device=q.device)
    r = torch.arange(M, device=q.device)[:, None]
    k = torch.arange(0, D, 16, device=q.device)[None, :]
    s = scales.view(torch.uint8)[r // 128, k // 64, r % 32, r % 128 // 32, k % 64 // 16].view(torch.float8_e4m3fn)
    return grid[code] * s.double().repeat_interleave(16, dim=1)[:, :D] * row_scales.double()[:, None]


def policy(x, token, old, A, ref, weight, temperature, low, high, kl, ok):
    """(loss, lp, slope, gradient) of one row in 64 bits: x float64 [V], ok bool [V]."""
    T = temperature if temperature > 0 else 1.0
    T = min(max(T, 2.0 ** -126), 3.4028234663852886e38)
    grad = np.zeros(len(x))
    if not (0 <= token < len(x)) or not ok[token] or x[token] == -math.inf:
        return 0.0, -math.inf, 0.0, grad
    with np.errstate(all="ignore"):
        top = x[ok].max() if not np.isnan(x[ok]).any() else math.nan
        y = (x[ok] - top) / T
        lse = math.log(np.exp(y).sum()) if math.isfinite(top) else math.nan
        p = np.exp(y - lse)
        lp = (x[token] - top) / T - lse
        if lp == -math.inf:
            return 0.0, -math.inf, 0.0, grad
        if weight == 0:
            return 0.0, lp, 0.0, grad
        rho = np.exp(np.float64(lp) - old)
        free, held = rho * A, min(max(rho, 1 - low), 1 + high) * A
        loss = -(held if free > held else free)
        slope = 0.0 if free > held else -free
        if ref is not None and kl > 0:
            d = ref - lp
            loss += kl * (np.expm1(d) - d)
            slope -= kl * np.expm1(d)
        g = -p
        g[np.flatnonzero(ok).searchsorted(token)] += 1.0
        grad[ok] = weight * slope * g / T
    return weight * loss, lp, weight * slope, grad
