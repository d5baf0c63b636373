"""Workloads of the operators around the commit step: a 4-bit output head, the verification of drafted tokens and
the distillation of a drafter.

Three kinds of case, each through the package's public entry points, with a plain form in elementary torch operations:

  quant    an output head with 4-bit weights and group scales over few rows: logits (``QuantHead.logits``), or the
           softmax statistics that ``gate_commit`` takes (``QuantHead.stats``)
  verify   drafted tokens against a target's logits, from given random numbers (``VerifyDraft``)
  distill  loss against a teacher's top logits: forward and backward (``distill``), or both in one pass
           (``distill_grad``)

The inputs are seeded random stand-ins: W_U ~ N(0, 1/d) rounded to 4 bits; hidden rows whose target token has a logit
around ln V; drafts and targets whose logits are correlated, with a few tokens a row that hold most of the mass.
"""
from __future__ import annotations

import math

import torch

own = False

LLADA = dict(d=4096, V=126464)
DREAM = dict(d=3584, V=152064)
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _quant(name, dtype, M, d, V, group=128, zeros=False, stats=False, out="f32"):
    return dict(name=name, kind="quant", dtype=dtype, M=M, d=d, V=V, group=group, zeros=zeros, stats=stats, out=out)


def _verify(name, dtype, B, T, V, draft=True, ragged=False, greedy=False, scale=1.0):
    return dict(name=name, kind="verify", dtype=dtype, B=B, T=T, V=V, draft=draft, ragged=ragged, greedy=greedy,
                scale=scale)


def _distill(name, dtype, N, V, k, tail=False, masked=1.0, fused=False, scale=1.0):
    return dict(name=name, kind="distill", dtype=dtype, N=N, V=V, k=k, tail=tail, masked=masked, fused=fused,
                scale=scale)


def listed():
    return [
        # one row at a toy head: launch and latency
        _quant("quant_one_toy", "bf16", 1, 256, 4096, group=64),
        # a single token at the LLaDA-8B head
        _quant("quant_one", "bf16", 1, group=128, out="bf16", **LLADA),
        # late decoding, 8 masked positions of 4 layers: the statistics that the gate takes, no logits
        _quant("quant_late_stats", "bf16", 32, group=128, stats=True, **LLADA),
        # a handful of drafted positions at the Dream-7B head, fp16, zero points, small groups
        _quant("quant_dream_f16", "f16", 13, group=64, zeros=True, out="f16", **DREAM),
        # a batch of 64 rows, logits in fp32
        _quant("quant_batch", "bf16", 64, group=128, **LLADA),
        # one user's draft of four tokens
        _verify("verify_one", "bf16", 1, 4, 126464),
        # a batch of ragged drafts of up to eight tokens
        _verify("verify_batch", "bf16", 32, 8, 152064, ragged=True, scale=1.25),
        # drafts without probabilities (a lookup's), fp32 logits, odd vocabulary
        _verify("verify_lookup_f32", "f32", 7, 5, 32003, draft=False),
        # greedy verification of a batch
        _verify("verify_greedy", "f16", 24, 3, 65537, draft=False, ragged=True, greedy=True),
        # the masked positions of one nearly finished canvas, forward and backward
        _distill("distill_few", "bf16", 8, 126464, 32),
        # four canvases of 256 positions, three quarters masked, the teacher's tail as one entry, in one pass
        _distill("distill_canvas", "bf16", 1024, 126464, 64, tail=True, masked=0.75, fused=True),
        # fp32 logits, odd vocabulary and list, temperature 2, forward and backward
        _distill("distill_f32", "f32", 301, 32003, 50, tail=True, scale=0.5),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["quant", "verify", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f16"] if kind == "quant" else ["bf16", "bf16", "f16", "f32"])
    V = int(_log(rng, 4096, 152065))
    if kind == "quant":
        d = int(_log(rng, 256, 4097)) // 8 * 8
        V = min(V, 126464 * 4096 // d)
        return dict(kind=kind, dtype=dtype, M=int(_log(rng, 1, 65)), d=d, V=V, group=rng.choice([32, 64, 128, 128]),
                    zeros=rng.random() < 0.4, stats=rng.random() < 0.35, out=rng.choice(["f32", dtype]))
    if kind == "verify":
        T = int(_log(rng, 1, 13))
        most = 288 * 152064 * (2 if dtype == "f32" else 4) // 4   # logits of the target
        B = max(1, min(int(_log(rng, 1, 65)), most // ((T + 1) * V)))
        return dict(kind=kind, dtype=dtype, B=B, T=T, V=V, draft=rng.random() < 0.7, ragged=rng.random() < 0.5,
                    greedy=rng.random() < 0.2, scale=rng.choice([1.0, 1.0, 0.7, 1.5]))
    most = 1024 * 126464 * (2 if dtype == "f32" else 4) // 4
    N = max(1, min(int(_log(rng, 1, 1025)), most // V))
    return dict(kind=kind, dtype=dtype, N=N, V=V, k=int(_log(rng, 1, 129)), tail=rng.random() < 0.5,
                masked=rng.choice([1.0, 1.0, 0.75, 0.3]), fused=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 0.5]))


# ------------------------------------------------------------------ inputs --

def _lens(case):
    """Drafted tokens of each sequence, 0 to T of them."""
    B, T = case["B"], case["T"]
    return [(5 * b + T) % (T + 1) for b in range(B)] if case["ragged"] else [T] * B


def _quant_inputs(case, seed):
    """codes uint8 [V][d/2], scales [V][groups], zeros uint8 [V][groups] or None, x [M][d]."""
    M, d, V, G = (case[k] for k in ("M", "d", "V", "group"))
    dt = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    ng = -(-d // G)
    codes = torch.empty((V, d // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((V, ng), dtype=dt, device="cuda")
    zeros = torch.empty((V, ng), dtype=torch.uint8, device="cuda") if case["zeros"] else None
    target = torch.randint(0, V, (M,), generator=g, device="cuda")
    rows = torch.empty((M, d), device="cuda")
    for v0 in range(0, V, 16384):
        n = min(16384, V - v0)
        w = torch.zeros((n, ng * G), device="cuda")
        w[:, :d] = torch.randn((n, d), generator=g, device="cuda") / math.sqrt(d)
        w = w.view(n, ng, G)
        if zeros is None:
            s = (w.abs().amax(2) / 7.0).to(dt)
            z = torch.full_like(s, 8.0).float()
        else:
            lo, hi = w.amin(2).clamp_max(0.0), w.amax(2)
            s = ((hi - lo) / 15.0).to(dt)
            z = torch.round(-lo / s.float()).clamp(0, 15)
            zeros[v0:v0 + n] = z.to(torch.uint8)
        q = torch.round(w / s.float().unsqueeze(2) + z.unsqueeze(2)).clamp(0, 15)
        here = (target >= v0) & (target < v0 + n)
        deq = ((q - z.unsqueeze(2)) * s.float().unsqueeze(2)).view(n, ng * G)[:, :d]
        rows = torch.where(here.unsqueeze(1), deq[(target - v0).clamp(0, n - 1)], rows)
        q = q.view(n, ng * G)[:, :d].to(torch.uint8)
        codes[v0:v0 + n] = q[:, 0::2] | (q[:, 1::2] << 4)
        scales[v0:v0 + n] = s
    level = math.log(V) - 3.0 + 9.0 * torch.rand((M,), generator=g, device="cuda")
    x = rows * (level / rows.square().sum(1)).unsqueeze(1) + torch.randn((M, d), generator=g, device="cuda")
    return codes, scales, zeros, x.to(dt)


def _logit_rows(g, rows, V, level=1.5):
    """Rows of logits: a wide floor, and 24 tokens a row of which a few hold most of the mass."""
    z = torch.randn((rows, V), generator=g, device="cuda")
    at = torch.randint(0, V, (rows, 24), generator=g, device="cuda")
    top = math.log(V) + level + 2.0 * torch.randn((rows, 24), generator=g, device="cuda")
    return z.scatter_(1, at, top)


def _verify_inputs(case, seed):
    """target [B][T+1][V], draft [B][T][V] or None, token int32 [B][T], u [B][T], r [B], lens int32 [B]."""
    B, T, V = (case[k] for k in "BTV")
    dt = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.empty((B, T + 1, V), dtype=dt, device="cuda")
    draft = torch.empty((B, T, V), dtype=dt, device="cuda") if case["draft"] else None
    token = torch.empty((B, T), dtype=torch.int32, device="cuda")
    for b in range(B):
        z = _logit_rows(g, T + 1, V)
        target[b] = z
        zd = (z[:T] + 0.6 * torch.randn((T, V), generator=g, device="cuda")).to(dt)
        race = torch.rand((T, V), generator=g, device="cuda").clamp_min(1e-20).log().neg().log().neg()
        # drawn from the draft; greedy drafts are its likeliest token
        token[b] = (zd.float() * case["scale"] + (0.0 if case["greedy"] else 1.0) * race).argmax(1).int()
        if draft is not None:
            draft[b] = zd
    u = torch.rand((B, T), generator=g, device="cuda")
    r = torch.rand((B,), generator=g, device="cuda")
    lens = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    return target, draft, token, u, r, lens


def _distill_inputs(case, seed):
    """logits [N][V], ids int32 [N][k], teacher's logits [N][k] and log-sum-exp [N], weight [N], upstream gradient [N]."""
    N, V, k = (case[x] for x in "NVk")
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.empty((N, V), dtype=DTYPES[case["dtype"]], device="cuda")
    ids = torch.empty((N, k), dtype=torch.int32, device="cuda")
    top = torch.empty((N, k), device="cuda")
    lse = torch.empty((N,), device="cuda")
    for n0 in range(0, N, 64):
        n = min(64, N - n0)
        z = _logit_rows(g, n, V)
        t, i = z.topk(k, dim=1)
        ids[n0:n0 + n], top[n0:n0 + n] = i.int(), t
        lse[n0:n0 + n] = torch.logsumexp(z * case["scale"], 1)
        logits[n0:n0 + n] = z + 0.8 * torch.randn((n, V), generator=g, device="cuda")
    weight = (torch.rand((N,), generator=g, device="cuda") < case["masked"]).float()
    up = (0.5 + torch.rand((N,), generator=g, device="cuda")) / N
    return logits, ids, top, lse, weight, up


def prepare(case, seed):
    if case["kind"] == "quant":
        codes, scales, zeros, x = _quant_inputs(case, seed)
        state = dict(case=case, codes=codes, scales=scales, zeros=zeros, x=x)
        if own:   # the weights laid out once, as a program that serves them keeps them
            from paper_2609_36452_amd import binding as rpd
            state["head"] = rpd.QuantHead(codes, scales, zeros, group=case["group"])
        return state
    if case["kind"] == "verify":
        target, draft, token, u, r, lens = _verify_inputs(case, seed)
        state = dict(case=case, target=target, draft=draft, token=token, u=u, r=r,
                     lens=lens if case["ragged"] else None)
        if own:   # outputs and workspace kept over the iterations
            from paper_2609_36452_amd import binding as rpd
            state["call"] = rpd.VerifyDraft(target, token, u, r, draft_logits=draft, draft_len=state["lens"],
                                            target_scale=case["scale"], draft_scale=case["scale"],
                                            greedy=case["greedy"])
        return state
    logits, ids, top, lse, weight, up = _distill_inputs(case, seed)
    return dict(case=case, logits=logits.requires_grad_(not case["fused"]), ids=ids, top=top,
                lse=lse if case["tail"] else None, weight=weight, up=up)


# -------------------------------------------------------------- plain form --

def _plain_quant(case, codes, scales, zeros, x):
    V, d, G = case["V"], case["d"], case["group"]
    x = x.float()
    y = torch.empty((x.shape[0], V), device=x.device)
    for v0 in range(0, V, 32768):
        c = codes[v0:v0 + 32768]
        q = torch.stack([c & 15, c >> 4], dim=2).view(c.shape[0], d).float()
        s = scales[v0:v0 + 32768].float().repeat_interleave(G, 1)[:, :d]
        z = 8.0 if zeros is None else zeros[v0:v0 + 32768].float().repeat_interleave(G, 1)[:, :d]
        y[:, v0:v0 + 32768] = x @ ((q - z) * s).t()
    if not case["stats"]:
        return y.to(DTYPES[case["out"]])
    m, at = y.max(1)
    t = y - m.unsqueeze(1)
    e = t.exp()
    S = e.sum(1)
    return {"argmax": at.int(), "confidence": 1.0 / S, "entropy": S.log() - (e * t).sum(1) / S}


def _softmax64(row, scale):
    t = row.double() * scale
    e = (t - t.amax(-1, keepdim=True)).exp()
    return e / e.sum(-1, keepdim=True)


def _plain_verify(case, target, draft, token, u, r, lens):
    B, T, V = (case[k] for k in "BTV")
    scale = float(torch.tensor(case["scale"], dtype=torch.float32))
    at = torch.arange(T, device=target.device)
    n_of = torch.full((B,), T, device=target.device) if lens is None else lens.long()
    live = at.unsqueeze(0) < n_of.unsqueeze(1)
    x = token.long()
    batch = torch.arange(B, device=target.device)
    slot = torch.arange(T + 1, device=target.device)
    drafted = torch.cat([token, token.new_zeros((B, 1))], 1)
    if case["greedy"]:
        best = target.float().argmax(2)
        same = (best[:, :T] == x) & live
        n = same.int().cumprod(1).sum(1)
        last = best[batch, n].int()
        accept = same.float()
    else:
        zp = target.float() * scale
        lp = zp[:, :T].gather(2, x.unsqueeze(2)).squeeze(2) - torch.logsumexp(zp[:, :T], 2)
        if draft is not None:
            zq = draft.float() * scale
            lp = lp - (zq.gather(2, x.unsqueeze(2)).squeeze(2) - torch.logsumexp(zq, 2))
        accept = torch.where(live, lp.clamp_max(0.0).exp(), torch.zeros_like(lp))
        n = ((u < accept) & live).int().cumprod(1).sum(1)
        p = _softmax64(target[batch, n], scale)
        w = p
        if T > 0:
            turned = (n < n_of).unsqueeze(1)
            row = n.clamp_max(T - 1)
            if draft is not None:
                rest = (p - _softmax64(draft[batch, row], scale)).clamp_min(0.0)
            else:
                rest = p.scatter(1, x[batch, row].unsqueeze(1), 0.0)
            w = torch.where(turned & (rest.sum(1, keepdim=True) > 0), rest, p)
        c = w.cumsum(1)
        last = (c <= (r.double() * c[:, -1]).unsqueeze(1)).sum(1).int()
    token_out = torch.where(slot.unsqueeze(0) < n.unsqueeze(1), drafted, torch.full_like(drafted, -1))
    token_out = torch.where(slot.unsqueeze(0) == n.unsqueeze(1), last.unsqueeze(1), token_out)
    return {"token": token_out, "n_accept": n.int(), "accept": accept}


def _plain_distill(case, logits, ids, top, lse, weight, up):
    V, scale = case["V"], case["scale"]
    at = ids.long()
    t = top * scale
    if lse is None:
        e = (t - t.amax(1, keepdim=True)).exp()
        p = e / e.sum(1, keepdim=True)
        rest = torch.zeros_like(p[:, 0])
    else:
        p64 = (t.double() - lse.double().unsqueeze(1)).exp()
        rest = (1.0 - p64.sum(1)).clamp_min(0.0).float()
        p = p64.float()
    z = logits.detach().float() * scale
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    listed_mass = e.gather(1, at)
    outside = e.scatter(1, at, 0.0).sum(1)
    S = outside + listed_mass.sum(1)
    log_q = z.gather(1, at) - S.log().unsqueeze(1)
    loss = (p * (p.log() - log_q)).sum(1)
    share = p.sum(1)
    tail = torch.zeros_like(S)
    if lse is not None:
        loss = loss + torch.where(rest > 0, rest * (rest.log() - (outside / S).log()), torch.zeros_like(rest))
        share = share + rest
        tail = torch.where(rest > 0, rest / outside, torch.zeros_like(rest))
    g = (weight * up * scale).unsqueeze(1)
    inside = g * ((share / S).unsqueeze(1) * listed_mass - p)
    grad = (e * (g * (share / S - tail).unsqueeze(1))).scatter(1, at, inside)
    return loss * weight, grad.to(logits.dtype)


def run(state):
    case = state["case"]
    if case["kind"] == "quant":
        if not own:
            return _plain_quant(case, state["codes"], state["scales"], state["zeros"], state["x"])
        if case["stats"]:
            return state["head"].stats(state["x"])
        return state["head"].logits(state["x"], out_dtype=DTYPES[case["out"]])
    if case["kind"] == "verify":
        if not own:
            return _plain_verify(case, *(state[k] for k in ("target", "draft", "token", "u", "r", "lens")))
        return state["call"]()
    a = {k: state[k] for k in ("logits", "ids", "top", "lse", "weight", "up")}
    if not own:
        return _plain_distill(case, **a)
    from paper_2609_36452_amd import binding as rpd
    if case["fused"]:
        return rpd.distill_grad(a["logits"], a["ids"], a["top"], teacher_lse=a["lse"], weight=a["weight"],
                                grad_loss=a["up"], logit_scale=case["scale"])
    loss = rpd.distill(a["logits"], a["ids"], a["top"], teacher_lse=a["lse"], weight=a["weight"],
                       logit_scale=case["scale"])
    grad, = torch.autograd.grad(loss, a["logits"], a["up"])
    return loss.detach(), grad


# ----------------------------------------------------------------- what it takes --

def work(case):
    if case["kind"] == "quant":
        M, d, V = case["M"], case["d"], case["V"]
        groups = -(-d // case["group"])
        out = 12 * M if case["stats"] else M * V * (4 if case["out"] == "f32" else 2)
        return {"bytes": V * d // 2 + V * groups * (3 if case["zeros"] else 2) + 2 * M * d + out,
                "flops": 2 * M * V * d}
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "verify":
        B, T, V = (case[k] for k in "BTV")
        rows = sum((2 if case["draft"] and not case["greedy"] else 1) * n + 1 for n in _lens(case))
        return {"bytes": rows * V * size + B * (16 * T + 12), "flops": rows * V * (1 if case["greedy"] else 4)}
    N, V, k = (case[x] for x in "NVk")
    rows = math.ceil(N * case["masked"])   # rows of weight 0 are written, not read
    return {"bytes": (rows + N) * V * size + N * (8 * k + 16), "flops": rows * V * 6}


# ------------------------------------------------------------------- exact --

def _exact_quant(case, seed):
    codes, scales, zeros, x = _quant_inputs(case, seed)
    V, d, G = case["V"], case["d"], case["group"]
    y = torch.empty((case["M"], V), dtype=torch.float64, device="cuda")
    for v0 in range(0, V, 8192):
        v1 = min(V, v0 + 8192)
        w = torch.empty((v1 - v0, d), dtype=torch.float64, device="cuda")
        w[:, 0::2] = (codes[v0:v1] % 16).double()
        w[:, 1::2] = (codes[v0:v1] // 16).double()
        for i in range(scales.shape[1]):
            part = w[:, i * G:(i + 1) * G]
            part -= 8.0 if zeros is None else zeros[v0:v1, i:i + 1].double()
            part *= scales[v0:v1, i:i + 1].double()
        y[:, v0:v1] = torch.matmul(x.double(), w.t().contiguous())
    if not case["stats"]:
        return y
    lse = torch.logsumexp(y, 1)
    q = (y - lse.unsqueeze(1)).exp()
    return {"argmax": None, "confidence": q.amax(1), "entropy": lse - (q * y).sum(1)}


def _exact_verify(case, seed):
    target, draft, token, _, _, _ = _verify_inputs(case, seed)
    if case["greedy"]:
        return None   # whole numbers and truth values only
    B, T = case["B"], case["T"]
    accept = torch.zeros((B, T), dtype=torch.float64, device="cuda")
    scale = float(torch.tensor(case["scale"], dtype=torch.float32))
    for b, n in enumerate(_lens(case)):
        for t in range(n):
            x = int(token[b, t])
            ratio = (target[b, t].double() * scale).softmax(0)[x]
            if draft is not None:
                ratio = ratio / (draft[b, t].double() * scale).softmax(0)[x]
            accept[b, t] = ratio.clamp(max=1.0)
    return {"token": None, "n_accept": None, "accept": accept}


def _exact_distill(case, seed):
    logits, ids, top, lse, weight, up = _distill_inputs(case, seed)
    losses, grads = [], []
    for n0 in range(0, case["N"], 64):
        part = slice(n0, min(case["N"], n0 + 64))
        at, s = ids[part].long(), case["scale"]
        p = (top[part] * s).double()
        p = (p - lse[part].double().unsqueeze(1)).exp() if case["tail"] else p.softmax(1)
        log_q = (logits[part].double() * s).log_softmax(1)
        q = log_q.exp()
        loss = (p * (p.log() - log_q.gather(1, at))).sum(1)
        spread = q * p.sum(1, keepdim=True)
        if case["tail"]:
            rest = (1.0 - p.sum(1)).clamp(min=0.0)
            free = q.scatter(1, at, 0.0)
            tail = free.sum(1)
            loss = loss + torch.xlogy(rest, rest) - torch.xlogy(rest, tail)
            spread = spread + q * rest.unsqueeze(1) - free * (rest / tail).unsqueeze(1)
        g = (weight[part] * up[part]).double() * s
        grads.append((spread - torch.zeros_like(q).scatter_add(1, at, p)) * g.unsqueeze(1))
        losses.append(loss * weight[part].double())
    return torch.cat(losses), torch.cat(grads)


def exact(case, seed):
    return {"quant": _exact_quant, "verify": _exact_verify, "distill": _exact_distill}[case["kind"]](case, seed)
