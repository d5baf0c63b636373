"""Plain float64 forms of 8-bit blocks, of the head in them and of sampling, written from their formulas, and the error
bounds that their tests take. They work on tensors of any device."""
from __future__ import annotations

import math

import torch

from tests.operators_ref import U32, half_step, stats  # noqa: F401

BLOCK = 128


def e4m3(t):
    """t (float64, |t| <= 448) to the nearest value with 4 significant bits, or multiple of 2^-9 below 2^-6; ties to even."""
    a = t.abs().clamp_min(2.0 ** -6)
    f, _ = torch.frexp(a)   # a = f 2^e, f in [1/2, 1): the quotient is 2^e exactly
    step = a / f / 16.0
    return torch.round(t / step) * step


def quantize(x, per):
    """(values of the codes, scales) of x [rows][d] in float64; NaN where x is not finite."""
    rows, d = x.shape
    x = x.double()
    rb, kb = -(-rows // per), -(-d // BLOCK)
    powers = [2.0 ** e for e in range(-126, 121)]
    codes = torch.empty((rows, d), dtype=torch.float64, device=x.device)
    scales = torch.empty((rb, kb), dtype=torch.float64, device=x.device)
    finite = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x))
    for j in range(kb):
        top = torch.zeros((rb * per, min(BLOCK, d - j * BLOCK)), dtype=torch.float64, device=x.device)
        top[:rows] = finite[:, j * BLOCK:(j + 1) * BLOCK]
        top = top.view(rb, -1).amax(1)
        s = torch.ones_like(top)
        found = top == 0
        for p in powers:
            here = ~found & (top <= 448.0 * p)
            s[here] = p
            found |= here
        scales[:, j] = s
        t = x[:, j * BLOCK:(j + 1) * BLOCK] / s.repeat_interleave(per)[:rows].unsqueeze(1)
        codes[:, j * BLOCK:(j + 1) * BLOCK] = torch.where(t.isfinite(), e4m3(torch.nan_to_num(t, 0.0, 0.0, 0.0)),
                                                          torch.full_like(t, math.nan))
    return codes, scales


def values(codes, scales, per):
    """What codes and scales stand for."""
    rows, d = codes.shape
    s = scales.double().repeat_interleave(BLOCK, 1)[:, :d]
    return codes.double() * (s if per == 1 else s.repeat_interleave(per, 0)[:rows])


def make_head(V, d, seed, device):
    """Codes of every magnitude and sign, scales of any value."""
    g = torch.Generator().manual_seed(seed)
    codes = (torch.randn((V, d), generator=g) * 60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = (0.2 + torch.rand((-(-V // BLOCK), -(-d // BLOCK)), generator=g)) / 60.0 / math.sqrt(d)
    return codes.to(device), scales.to(device)


def product(w, x):
    return torch.matmul(x, w.t().contiguous())


def product_bound(w, x):
    """Bound on a logit's error in float32: a term goes through the additions of its block of 128, the scaling, and the
    additions of the blocks (parts of the sum among them)."""
    terms = torch.matmul(x.abs(), w.abs().t().contiguous())
    return (BLOCK + -(-w.shape[1] // BLOCK) + 4) * U32 * terms
