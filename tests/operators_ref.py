"""Plain float64 forms of the operators beside the commit step, written from their formulas, and the error bounds that
their tests take. They work on tensors of any device."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -23   # one float32 operation, truncating or not, with its operand's rounding


def half_step(dtype: torch.dtype) -> float:
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------ quant --

def make_head(V, d, group, dtype, zeros, seed, device):
    g = torch.Generator().manual_seed(seed)
    ng = -(-d // group)
    codes = torch.randint(0, 256, (V, d // 2), generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand((V, ng), generator=g)) * 0.02).to(dtype)
    z = torch.randint(0, 16, (V, ng), generator=g, dtype=torch.uint8) if zeros else None
    return codes.to(device), scales.to(device), None if z is None else z.to(device)


def dequantize(codes, scales, zeros, group):
    V, d = codes.shape[0], 2 * codes.shape[1]
    q = torch.empty((V, d), dtype=torch.float64, device=codes.device)
    q[:, 0::2] = (codes & 15).double()
    q[:, 1::2] = (codes >> 4).double()
    at = torch.arange(d, device=codes.device) // group
    z = 8.0 if zeros is None else zeros.double()[:, at]
    return (q - z) * scales.double()[:, at]


def quant_logits(w, x):
    return torch.matmul(x.double(), w.t().contiguous())


def quant_bound(w, x, groups):
    """Bound on a logit's error in float32: the products and the scaling round each term, and a term goes through
    the additions of its group, of the groups and of at most 16 waves; bf16 rows lose 2^-28 of their largest."""
    terms = torch.matmul(x.double().abs(), w.abs().t().contiguous())
    flushed = 2.0 ** -28 * x.double().abs().amax(1, keepdim=True) * w.abs().sum(1).unsqueeze(0)
    return (128 + groups + 16 + 4) * U32 * terms + flushed


def stats(y):
    lse = torch.logsumexp(y, 1)
    p = (y - lse.unsqueeze(1)).exp()
    h = -(torch.where(p > 0, p * (y - lse.unsqueeze(1)), torch.zeros_like(p))).sum(1)
    return y.argmax(1), p.amax(1), h


# ----------------------------------------------------------------- verify --

def verify(target, token, u, r, draft=None, lens=None, target_scale=1.0, draft_scale=1.0, greedy=False):
    """One sequence and token after another, as the rule is stated."""
    B, T1, V = target.shape
    out = torch.full((B, T1), -1, dtype=torch.int64)
    n_accept = torch.zeros(B, dtype=torch.int64)
    accept = torch.zeros((B, T1 - 1), dtype=torch.float64)
    f32 = lambda s: float(torch.tensor(s, dtype=torch.float32))   # noqa: E731

    def dist(row, scale):
        z = row.double().cpu() * f32(scale)
        m = z.max()
        e = (z - (m if m != -math.inf else 0.0)).exp()
        return e / e.sum()

    for b in range(B):
        n = T1 - 1 if lens is None else min(max(int(lens[b]), 0), T1 - 1)
        w = None
        for t in range(n + 1):
            row = target[b, t]
            if greedy:
                z = row.double().cpu()
                z = torch.where(z.isnan(), torch.full_like(z, -math.inf), z)
                best = int(z.argmax()) if bool((z > -math.inf).any()) else -1
                w = best
                if t < n:
                    accept[b, t] = float(best >= 0 and int(token[b, t]) == best)
                continue
            if t == n:
                w = dist(row, target_scale)
                break
            x = int(token[b, t])
            p = dist(row, target_scale)
            q = dist(draft[b, t], draft_scale) if draft is not None else None
            valid = 0 <= x < V
            if valid:
                a = float(p[x]) if q is None else float(p[x] / q[x])
                a = min(a, 1.0) if not math.isnan(a) else a
            else:
                a = 0.0
            accept[b, t] = a
            if float(u[b, t]) < a:
                continue
            if q is None:
                rest = p.clone()
                if valid:
                    rest[x] = 0.0
            else:
                rest = (p - q).clamp_min(0.0)
            w = rest if float(rest.sum()) > 0 else p
            n_accept[b] = t
            break
        if greedy:
            k = 0
            while k < n and accept[b, k] == 1.0:
                k += 1
            n_accept[b] = k
            z = target[b, k].double().cpu()
            z = torch.where(z.isnan(), torch.full_like(z, -math.inf), z)
            out[b, k] = int(z.argmax()) if bool((z > -math.inf).any()) else -1
        else:
            if t == n:
                n_accept[b] = n
            # behind the first rejection the acceptance probabilities are reported too
            for s in range(int(n_accept[b]) + 1, n):
                x = int(token[b, s])
                p = dist(target[b, s], target_scale)
                if not 0 <= x < V:
                    continue
                a = float(p[x]) if draft is None else float(p[x] / dist(draft[b, s], draft_scale)[x])
                accept[b, s] = min(a, 1.0) if not math.isnan(a) else a
            total = float(w.sum())
            k = int(n_accept[b])
            if total > 0 and math.isfinite(total):
                c = w.cumsum(0)
                hit = (c > float(r[b]) * float(c[-1])).nonzero()
                out[b, k] = int(hit[0]) if len(hit) else int((w > 0).nonzero()[-1])
        out[b, :int(n_accept[b])] = token[b, :int(n_accept[b])].long().cpu()
    return out, n_accept, accept


# ---------------------------------------------------------------- distill --

def distill(logits, ids, teacher, lse=None, weight=None, up=None, scale=1.0):
    """loss [N], gradient [N][V], and the magnitude of the gradient's terms [N][V], in float64, row by row."""
    N, V = logits.shape
    losses = torch.zeros(N, dtype=torch.float64)
    grads = torch.zeros((N, V), dtype=torch.float64)
    terms = torch.zeros((N, V), dtype=torch.float64)
    for n in range(N):
        w = 1.0 if weight is None else float(weight[n])
        if w == 0.0:
            continue
        keep = [j for j in range(ids.shape[1]) if 0 <= int(ids[n, j]) < V]
        at = ids[n].cpu().long()[keep]
        t = teacher[n].double().cpu()[keep] * scale
        if lse is None:
            if not keep or bool((t == -math.inf).all()):
                continue
            p = (t - t.max()).exp()
            p = p / p.sum()
            rest = 0.0
        else:
            p = (t - float(lse[n])).exp()
            rest = max(0.0, 1.0 - float(p.sum()))
        z = logits[n].double().cpu() * scale
        inside = torch.zeros(V, dtype=torch.bool)
        inside[at] = True
        lz = torch.logsumexp(z, 0)
        lt = torch.logsumexp(z[~inside], 0) if bool((~inside).any()) else torch.tensor(-math.inf, dtype=torch.float64)
        pos = p > 0
        loss = (p[pos] * (p[pos].log() - (z[at][pos] - lz))).sum()
        if rest > 0:
            loss = loss + rest * (math.log(rest) - float(lt - lz))
        P = float(p.sum()) + rest
        q = (z - lz).exp()
        g = P * q
        share = torch.zeros(V, dtype=torch.float64).scatter_add(0, at, p)
        g = g - share
        mag = P * q + share
        if rest > 0:
            tail = torch.where(inside, torch.zeros_like(z), rest * (z - lt).exp())
            g = g - tail
            mag = mag + tail
        c = w * (1.0 if up is None else float(up[n])) * scale
        losses[n] = w * loss
        grads[n] = c * g
        terms[n] = abs(c) * mag
    return losses, grads, terms


def sum_error(V):
    """Relative error of a float32 sum of V positive exponentials, 8 at a time by 256 threads over parts of a row:
    the additions of a thread, the merges, and an exponential of an argument down to -24 (smaller ones weigh less
    than their error)."""
    part = -(-(-(-V // 64)) // 2048) * 2048
    return (part / 256 + 32 + 2 * 24) * U32
