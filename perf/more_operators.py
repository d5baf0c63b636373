"""Workloads of drafting with an 8-bit output head: quantization to 8-bit floating point with a scale for each block
of 128, the output head in that form (also as the frozen head behind a drafter that is trained), and sampling from the
logits.

Three kinds of case, each through the package's public entry points, with a plain form in elementary torch operations:

  blocks  rows (hidden states) or a weight matrix to e4m3 codes, one power-of-two scale for 128 columns of a row or
          for 128 x 128 of a matrix (``fp8_quantize``)
  head    an output head in e4m3 with a float32 scale for each block of 128 x 128: logits (``Fp8Head.logits``), the
          softmax statistics that ``gate_commit`` takes (``Fp8Head.stats``), or logits and the gradient of the rows
          (``Fp8Head.logits`` and ``Fp8Head.input_grad``). Rows and upstream gradients are quantized within the call
  sample  tokens drawn from given random numbers with temperature, top-k, top-p and min-p, for a whole batch or with
          parameters of each row (``sample``), where asked with the logits that the filters leave, for ``verify_draft``

The inputs are seeded random stand-ins: W_U ~ N(0, 1/d), hidden rows whose target token has a logit around ln V, and
rows of logits with a wide floor and a few tokens that hold most of the mass.
"""
from __future__ import annotations

import math

import torch

own = False

LLADA = dict(d=4096, V=126464)
DREAM = dict(d=3584, V=152064)
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 128
LARGEST = 448.0   # of e4m3


def _blocks(name, dtype, rows, d, per=1):
    return dict(name=name, kind="blocks", dtype=dtype, rows=rows, d=d, per=per)


def _head(name, dtype, M, d, V, what="logits", out=None):
    return dict(name=name, kind="head", dtype=dtype, M=M, d=d, V=V, what=what, out=out or dtype)


def _sample(name, dtype, N, V, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=False, filtered=False):
    return dict(name=name, kind="sample", dtype=dtype, N=N, V=V, scale=scale, top_k=top_k, top_p=top_p, min_p=min_p,
                per_row=per_row, filtered=filtered)


def listed():
    return [
        # a few hidden rows on their way into a head: launch and latency
        _blocks("blocks_few_f16", "f16", 13, 3584),
        # the LLaDA-8B head, once, from bf16 weights
        _blocks("blocks_head", "bf16", 126464, 4096, per=128),
        # one row at a toy head: launch and latency
        _head("head_one_toy", "bf16", 1, 256, 4096),
        # a single token at the LLaDA-8B head
        _head("head_one", "bf16", 1, **LLADA),
        # late decoding, 8 masked positions of 4 layers: the statistics that the gate takes, no logits
        _head("head_late_stats", "bf16", 32, what="stats", **LLADA),
        # an odd number of drafted positions at the Dream-7B head, fp16
        _head("head_dream_f16", "f16", 101, **DREAM),
        # a whole canvas of 256 positions, 4 layers of each: statistics
        _head("head_canvas_stats", "bf16", 1024, what="stats", **LLADA),
        # a drafter's training step through the frozen head: logits, then the gradient of the rows
        _head("head_train", "bf16", 256, what="train", **LLADA),
        # one user's next token: short list, then nucleus
        _sample("sample_one", "bf16", 1, 126464, scale=1.25, top_k=40, top_p=0.95),
        # fp32 logits, odd vocabulary, tokens of a fiftieth of the likeliest one's probability and more
        _sample("sample_min_p_f32", "f32", 7, 32003, min_p=0.02),
        # a served batch, each row with parameters of its own; the filtered logits go on to the verification
        _sample("sample_batch", "f16", 32, 152064, per_row=True, filtered=True),
        # every position of a canvas, nucleus of 0.9
        _sample("sample_canvas", "bf16", 256, 126464, scale=1.0, top_p=0.9),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["blocks", "head", "head", "sample", "sample"])
    if kind == "blocks":
        per = rng.choice([1, 1, 128])
        d = int(_log(rng, 100, 4097))
        rows = int(_log(rng, 1, 8193) if per == 1 else _log(rng, 100, 126465))
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), rows=rows, d=d, per=per)
    V = int(_log(rng, 4096, 152065))
    if kind == "head":
        d = int(_log(rng, 200, 4097))
        if rng.random() < 0.5:
            d = max(128, d // 128 * 128)
        V = min(V, 126464 * 4096 // d)
        what = rng.choice(["logits", "logits", "stats", "train"])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        return dict(kind=kind, dtype=dtype, M=int(_log(rng, 1, 257 if what == "train" else 1025)), d=d, V=V, what=what,
                    out=dtype if what == "train" else rng.choice([dtype, dtype, "f32"]))
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    N = max(1, min(int(_log(rng, 1, 257)), 256 * 126464 // V // (2 if dtype == "f32" else 1)))
    return dict(kind=kind, dtype=dtype, N=N, V=V, scale=rng.choice([1.0, 1.0, 0.7, 1.4]),
                top_k=rng.choice([0, 0, int(_log(rng, 1, 2000))]), top_p=rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                min_p=rng.choice([0.0, 0.0, _log(rng, 0.001, 0.3)]), per_row=rng.random() < 0.3,
                filtered=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs --

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _blocks_inputs(case, seed):
    """x [rows][d]: weights ~ N(0, 1/d), or hidden rows whose columns differ in size."""
    g = _generator(seed)
    x = torch.randn((case["rows"], case["d"]), generator=g, device="cuda")
    if case["per"] == 1:
        x = x * (1.5 * torch.randn((case["d"],), generator=g, device="cuda")).exp()
    else:
        x = x / math.sqrt(case["d"])
    return x.to(DTYPES[case["dtype"]])


def _logit_rows(g, rows, V, level=1.5):
    """Rows of logits: a wide floor, and 24 tokens a row of which a few hold most of the mass."""
    z = torch.randn((rows, V), generator=g, device="cuda")
    part = V // 24   # one in each part of the row: no index twice, so that equal seeds give equal rows
    at = part * torch.arange(24, device="cuda") + torch.randint(0, part, (rows, 24), generator=g, device="cuda")
    top = math.log(V) + level + 2.0 * torch.randn((rows, 24), generator=g, device="cuda")
    return z.scatter_(1, at, top)


def _head_inputs(case, seed):
    """codes e4m3 [V][d], scales float32 [V/128][d/128], x [M][d], upstream gradient [M][V] or None."""
    M, d, V = (case[k] for k in ("M", "d", "V"))
    dt = DTYPES[case["dtype"]]
    g = _generator(seed)
    vb, kb = -(-V // BLOCK), -(-d // BLOCK)
    w = torch.zeros((vb * BLOCK, kb * BLOCK), device="cuda")
    w[:V, :d] = torch.randn((V, d), generator=g, device="cuda") / math.sqrt(d)
    w = w.view(vb, BLOCK, kb, BLOCK)
    scales = w.abs().amax((1, 3)) / LARGEST   # of any value, as checkpoints hold them
    s = scales.view(vb, 1, kb, 1)
    codes = (w / s).to(torch.float8_e4m3fn)
    target = torch.randint(0, V, (M,), generator=g, device="cuda")
    rows = (codes.float() * s).view(vb * BLOCK, kb * BLOCK)[target, :d]
    codes = codes.view(vb * BLOCK, kb * BLOCK)[:V, :d].contiguous()
    level = math.log(V) - 3.0 + 9.0 * torch.rand((M,), generator=g, device="cuda")
    x = rows * (level / rows.square().sum(1)).unsqueeze(1) + torch.randn((M, d), generator=g, device="cuda")
    up = None
    if case["what"] == "train":   # of a softmax loss against one token a row
        up = _logit_rows(g, M, V).softmax(1)
        up[torch.arange(M, device="cuda"), target] -= 1.0
        up = (up * ((1024.0 if dt == torch.float16 else 1.0) / M)).to(dt)   # fp16 takes a loss scale
    return codes, scales, x.to(dt), up


def _sample_inputs(case, seed):
    """logits [N][V], r [N], and scale, top_k, top_p, min_p: numbers, or tensors [N]."""
    N, V = case["N"], case["V"]
    g = _generator(seed)
    logits = _logit_rows(g, N, V).to(DTYPES[case["dtype"]])
    r = torch.rand((N,), generator=g, device="cuda")
    if not case["per_row"]:
        return logits, r, case["scale"], case["top_k"], case["top_p"], case["min_p"]
    u = torch.rand((4, N), generator=g, device="cuda")
    on = torch.rand((3, N), generator=g, device="cuda") < 0.6   # a filter that a row does not ask for is off
    scale = 0.6 + 0.9 * u[0]
    top_k = torch.where(on[0], (u[1] * math.log(1000.0)).exp(), torch.zeros_like(r)).int()
    top_p = torch.where(on[1], 0.5 + 0.49 * u[2], torch.ones_like(r))
    min_p = torch.where(on[2], 0.1 * u[3], torch.zeros_like(r))
    return logits, r, scale, top_k, top_p, min_p


def prepare(case, seed):
    if case["kind"] == "blocks":
        return dict(case=case, x=_blocks_inputs(case, seed))
    if case["kind"] == "head":
        codes, scales, x, up = _head_inputs(case, seed)
        state = dict(case=case, codes=codes, scales=scales, x=x, up=up)
        if own:   # the weights laid out once, as a program that serves them keeps them
            from paper_2609_36452_amd import binding as rpd
            state["head"] = rpd.Fp8Head(codes, scales, train=case["what"] == "train")
        return state
    names = ("logits", "r", "scale", "top_k", "top_p", "min_p")
    return dict(case=case, **dict(zip(names, _sample_inputs(case, seed))))


# -------------------------------------------------------------- plain form --

def _plain_quantize(x, per):
    """codes and scales: the smallest power of two with which the block's largest magnitude is at most 448."""
    rows, d = x.shape
    rb, kb = -(-rows // per), -(-d // BLOCK)
    t = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - d, 0, rb * per - rows)).view(rb, per, kb, BLOCK)
    top = t.abs().amax((1, 3))
    f, e = torch.frexp(top)
    e = torch.where(f <= 0.875, e - 9, e - 8).clamp(-126, 120)
    s = torch.where(top > 0, ((e + 127) << 23).view(torch.float32), torch.ones_like(top))   # 2^e by its bits
    codes = (t / s.view(rb, 1, kb, 1)).to(torch.float8_e4m3fn)
    return codes.view(rb * per, kb * BLOCK)[:rows, :d].contiguous(), s


def _values(codes, scales, per):
    """What codes and scales stand for, float32."""
    rows, d = codes.shape
    s = scales.repeat_interleave(BLOCK, 1)[:, :d]
    return codes.float() * (s if per == 1 else s.repeat_interleave(per, 0)[:rows])


def _plain_head(case, codes, scales, x, up):
    w = _values(codes, scales, BLOCK)
    y = _values(*_plain_quantize(x, 1), 1) @ w.t()
    if case["what"] == "stats":
        m, at = y.max(1)
        t = y - m.unsqueeze(1)
        e = t.exp()
        S = e.sum(1)
        return {"argmax": at.int(), "confidence": 1.0 / S, "entropy": S.log() - (e * t).sum(1) / S}
    y = y.to(DTYPES[case["out"]])
    if case["what"] == "logits":
        return y
    return y, (_values(*_plain_quantize(up, 1), 1) @ w).to(x.dtype)


def _column(v, like):
    """A parameter of each row, float64."""
    v = v.double() if torch.is_tensor(v) else torch.full_like(like, float(torch.tensor(v, dtype=torch.float32)), dtype=torch.float64)
    return v.unsqueeze(1)


def _plain_sample(case, logits, r, scale, top_k, top_p, min_p):
    N, V = case["N"], case["V"]
    z, at = logits.float().sort(dim=1, descending=True, stable=True)   # equal logits: the lowest index first
    x = (z.double() - z[:, :1].double()) * _column(scale, r)
    e = x.exp()
    before = e.cumsum(1) - e
    rank = torch.arange(V, device=z.device).unsqueeze(0)
    k, p, least = _column(top_k, r), _column(top_p, r), _column(min_p, r)
    kept = (k <= 0) | (rank < k)
    listed_mass = torch.where(kept, e, torch.zeros_like(e)).sum(1, keepdim=True)
    kept &= (p >= 1) | (before < p * listed_mass) | (rank == 0)
    kept &= (least <= 0) | (x >= least.log())
    e = torch.where(kept, e, torch.zeros_like(e))
    c = e.cumsum(1)
    n = kept.sum(1, keepdim=True)
    j = (c <= r.double().unsqueeze(1) * c[:, -1:]).sum(1, keepdim=True).minimum(n - 1)
    out = {"token": at.gather(1, j).squeeze(1).int(), "prob": (e.gather(1, j) / c[:, -1:]).squeeze(1).float(),
           "kept": n.squeeze(1).int()}
    if case["filtered"]:
        whole = torch.zeros_like(kept).scatter(1, at, kept)
        out["logits"] = torch.where(whole, logits, torch.full_like(logits, -math.inf))
    return out


def run(state):
    case = state["case"]
    if not own:
        a = {k: v for k, v in state.items() if k != "case"}
        if case["kind"] == "blocks":
            return _plain_quantize(a["x"], case["per"])
        return (_plain_head if case["kind"] == "head" else _plain_sample)(case, **a)
    from paper_2609_36452_amd import binding as rpd
    if case["kind"] == "blocks":
        return rpd.fp8_quantize(state["x"], block_rows=case["per"])
    if case["kind"] == "head":
        if case["what"] == "stats":
            return state["head"].stats(state["x"])
        y = state["head"].logits(state["x"], out_dtype=DTYPES[case["out"]])
        return y if case["what"] == "logits" else (y, state["head"].input_grad(state["up"]))
    return rpd.sample(state["logits"], state["r"], logit_scale=state["scale"], top_k=state["top_k"],
                      top_p=state["top_p"], min_p=state["min_p"], filtered=case["filtered"])


# ----------------------------------------------------------------- what it takes --

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "blocks":
        rows, d = case["rows"], case["d"]
        return {"bytes": rows * d * (size + 1) + 4 * -(-rows // case["per"]) * -(-d // BLOCK), "flops": 2 * rows * d}
    if case["kind"] == "head":
        M, d, V = (case[k] for k in ("M", "d", "V"))
        weights = V * d + 4 * -(-V // BLOCK) * -(-d // BLOCK)
        out = 12 * M if case["what"] == "stats" else M * V * (4 if case["out"] == "f32" else 2)
        train = case["what"] == "train"   # the gradient reads the weights and M V, and writes M d
        return {"bytes": weights + M * d * size + out + ((weights + M * V * size + M * d * size) if train else 0),
                "flops": (4 if train else 2) * M * V * d}
    N, V = case["N"], case["V"]
    return {"bytes": N * V * size * (2 if case["filtered"] else 1) + 16 * N, "flops": 4 * N * V}


# ------------------------------------------------------------------- exact --

def _exact_codes(x, per):
    """(values of the codes, scales) of x [rows][d] in float64, block by block of columns."""
    rows, d = x.shape
    codes = torch.empty((rows, d), dtype=torch.float64, device=x.device)
    scales = torch.empty((-(-rows // per), -(-d // BLOCK)), dtype=torch.float64, device=x.device)
    of = torch.arange(rows, device=x.device) // per
    power_of_two = torch.tensor([2.0 ** e for e in range(-126, 121)], dtype=torch.float64, device=x.device)
    for i in range(scales.shape[1]):
        t = x[:, i * BLOCK:(i + 1) * BLOCK].double()
        top = torch.zeros(scales.shape[0], dtype=torch.float64, device=x.device)
        top = top.scatter_reduce(0, of, t.abs().amax(1), "amax")
        power = power_of_two[torch.searchsorted(LARGEST * power_of_two, top)]   # the first with 448 of it enough
        power = torch.where(top > 0, power, torch.ones_like(power))
        scales[:, i] = power
        t = t / power[of].unsqueeze(1)
        f, _ = torch.frexp(t.abs().clamp_min(2.0 ** -6))
        step = t.abs().clamp_min(2.0 ** -6) / f / 16.0   # three bits behind the leading one
        codes[:, i * BLOCK:(i + 1) * BLOCK] = torch.round(t / step) * step
    return codes, scales


def _exact_rows(x):
    codes, scales = _exact_codes(x, 1)
    for i in range(scales.shape[1]):
        codes[:, i * BLOCK:(i + 1) * BLOCK] *= scales[:, i:i + 1]
    return codes


def _exact_head(case, seed):
    codes, scales, x, up = _head_inputs(case, seed)
    V, d = case["V"], case["d"]
    xq = _exact_rows(x)
    gq = None if up is None else _exact_rows(up)
    y = torch.empty((case["M"], V), dtype=torch.float64, device="cuda")
    grad = torch.zeros((case["M"], d), dtype=torch.float64, device="cuda")
    column = torch.arange(d, device="cuda") // BLOCK
    for v0 in range(0, V, 64 * BLOCK):
        v1 = min(V, v0 + 64 * BLOCK)
        row = torch.arange(v0, v1, device="cuda") // BLOCK
        w = codes[v0:v1].double() * scales.double()[row][:, column]
        y[:, v0:v1] = torch.matmul(xq, w.t().contiguous())
        if gq is not None:
            grad += torch.matmul(gq[:, v0:v1].contiguous(), w)
    if case["what"] == "stats":
        lse = torch.logsumexp(y, 1)
        q = (y - lse.unsqueeze(1)).exp()
        return {"argmax": None, "confidence": q.amax(1), "entropy": lse - (q * y).sum(1)}
    return y if gq is None else (y, grad)


def _exact_sample(case, seed):
    logits, r, scale, top_k, top_p, min_p = _sample_inputs(case, seed)
    prob = torch.empty((case["N"],), dtype=torch.float64, device="cuda")
    param = [[float(t) for t in (v.double().tolist() if torch.is_tensor(v) else [v] * case["N"])]
             for v in (scale, top_k, top_p, min_p)]
    for b in range(case["N"]):
        s, k, p, least = (v[b] for v in param)
        s, p, least = (float(torch.tensor(v, dtype=torch.float32)) for v in (s, p, least))
        t = logits[b].double()
        t = t[torch.argsort(-t, stable=True)] * s
        if k > 0:
            t = t[:int(k)]
        q = (t - torch.logsumexp(t, 0)).exp()
        n = q.numel()
        if p < 1:
            n = max(1, int((q.cumsum(0) - q < p).sum()))
        if least > 0:
            n = min(n, int((q >= least * q[0]).sum()))
        q = q[:n] / q[:n].sum()
        j = min(n - 1, int(torch.searchsorted(q.cumsum(0), r[b].double(), right=True)))
        prob[b] = q[j]
    return {"token": None, "prob": prob, "kept": None, "logits": None} if case["filtered"] else \
        {"token": None, "prob": prob, "kept": None}


def exact(case, seed):
    if case["kind"] == "blocks":
        return _exact_codes(_blocks_inputs(case, seed), case["per"])
    return (_exact_head if case["kind"] == "head" else _exact_sample)(case, seed)
