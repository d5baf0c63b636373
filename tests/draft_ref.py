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


# --------------------------------------------------------------- sampling --

def in_order(z):
    """(logits in order, float64, their indexes): the largest first, equal ones by index; -inf left out."""
    order = torch.argsort(-z.double(), stable=True)
    t = z.double()[order]
    n = int((t > -math.inf).sum())
    return t[:n], order[:n]


def f32(v):
    return float(torch.tensor(v, dtype=torch.float32))


def check_sample(z, r, scale, top_k, top_p, min_p, token, prob, kept, filtered=None, slack=1e-9):
    """One row's outputs against the definition in float64. Where a border lies within `slack` of the whole mass of a
    token's edge, either side of it is right."""
    scale, top_p, min_p = f32(scale), f32(top_p), f32(min_p)
    scale = 1.0 if scale == 0 else scale
    zz = z.double()
    if bool(zz.isnan().any()) or not bool(zz.isfinite().any()) or bool((zz == math.inf).any()) or not 0 < scale <= 2.0 ** 100:
        assert token == -1 and kept == 0 and math.isnan(prob)
        if filtered is not None:
            assert bool((filtered == -math.inf).all())
        return
    t, order = in_order(z)
    x = (t - t[0]) * scale
    e = x.exp()
    n = len(t)
    if top_k > 0:
        n = min(n, top_k)
    c = e.cumsum(0)
    before = c - e
    least, most = n, n
    if top_p < 1:
        T = top_p * float(c[n - 1])
        s = slack * float(c[n - 1])
        least = max(1, int((before[:n] < T - s).sum()))
        most = max(1, int((before[:n] < T + s).sum()))
    if min_p > 0:
        m = int((x >= math.log(min(min_p, 1.0)) - 0.0).sum())
        least, most = min(least, m), min(most, m)
    assert least <= kept <= most, (kept, least, most, n)
    S = float(c[kept - 1])
    at = (order[:kept] == token).nonzero()
    assert at.numel() == 1, "a token that was not kept"
    j = int(at[0, 0])
    s = slack * S
    assert float(before[j]) <= r * S + s and (float(c[j]) >= r * S - s or j == kept - 1), (j, r * S, float(before[j]), float(c[j]))
    assert abs(prob - float(e[j]) / S) <= 2.0 ** -24 * prob + 1e-9
    if filtered is not None:
        want = torch.full_like(z, -math.inf)
        want[order[:kept]] = z[order[:kept]]
        assert torch.equal(filtered, want)
