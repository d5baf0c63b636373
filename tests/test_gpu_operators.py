"""The 4-bit output head, the verification of drafted tokens and the distillation loss against plain float64 forms."""
import math

import numpy as np
import pytest
import torch

from paper_2609_36452_amd import binding as rpd
from tests import operators_ref as R
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


# ------------------------------------------------------------------ quant --

def _x(M, d, dtype, seed, level=1.0):
    g = torch.Generator().manual_seed(seed)
    return (level * torch.randn((M, d), generator=g)).to(dtype).to(DEV)


def _check_logits(y, w, x, groups):
    ref = R.quant_logits(w, x)
    tol = R.quant_bound(w, x, groups) + R.half_step(y.dtype) * ref.abs() * 1.01
    if y.dtype == HF:
        tol = tol + 2.0 ** -25   # half a subnormal step
    bad = (y.double() - ref).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float((y.double() - ref).abs().max()))


QUANT = [  # M, d, V, group, dtype, zeros
    (1, 256, 4096, 64, BF, False), (1, 8, 1, 32, BF, True), (2, 136, 17, 128, HF, False), (3, 40, 15, 32, BF, True),
    (16, 2048, 1000, 128, BF, False), (17, 2056, 333, 64, HF, True), (31, 4096, 515, 128, BF, False),
    (32, 4096, 2500, 32, HF, True), (33, 3584, 1111, 128, BF, True), (64, 4104, 257, 64, BF, False),
    (5, 8192, 300, 128, HF, False), (20, 9000, 130, 128, BF, True), (100, 1024, 777, 64, BF, False),
    (7, 17000, 40, 32, BF, False), (1, 128, 40001, 128, BF, False), (12, 384, 9000, 128, HF, True),
]


@pytest.mark.parametrize("M,d,V,group,dtype,zeros", QUANT)
def test_quant_logits(M, d, V, group, dtype, zeros):
    note(f"  quant logits M={M} d={d} V={V} group={group} {dtype} zeros={zeros}")
    codes, scales, z = R.make_head(V, d, group, dtype, zeros, M + d, DEV)
    head = rpd.QuantHead(codes, scales, z, group=group)
    x = _x(M, d, dtype, V)
    w = R.dequantize(codes, scales, z, group)
    ng = scales.shape[1]
    _check_logits(head.logits(x, out_dtype=F32), w, x, ng)
    _check_logits(head.logits(x), w, x, ng)


@pytest.mark.parametrize("M,d,V,group,dtype,zeros", QUANT)
def test_quant_stats(M, d, V, group, dtype, zeros):
    note(f"  quant stats M={M} d={d} V={V} group={group} {dtype} zeros={zeros}")
    codes, scales, z = R.make_head(V, d, group, dtype, zeros, M + d, DEV)
    head = rpd.QuantHead(codes, scales, z, group=group)
    x = _x(M, d, dtype, V, level=0.7)
    scale = 1.0 if M % 2 else 0.5
    o = head.stats(x, logit_scale=scale)
    w = R.dequantize(codes, scales, z, group)
    y = R.quant_logits(w, x) * scale
    delta = (R.quant_bound(w, x, scales.shape[1]) * scale + R.U32 * y.abs()).amax(1)
    at, c, h = R.stats(y)
    got = o["argmax"].long()
    assert bool(((got >= 0) & (got < V)).all())
    chosen = y.gather(1, got.unsqueeze(1)).squeeze(1)
    assert bool((chosen >= y.amax(1) - 2 * delta).all())
    # a sum of positive terms, in chains of the tiles of a slot, 16 columns and at most 2048 slots
    chain = (V / 16 / 8 + 16 + 40 + 2 * 24) * R.U32 if V < 16 * 256 else (V / 16 / 256 + 16 + 40 + 2 * 24) * R.U32
    rel = torch.expm1(2 * delta) + 2 * chain
    assert bool(((o["confidence"].double() - c).abs() <= rel * c).all())
    assert bool(((o["entropy"].double() - h).abs() <= 2 * rel * (h + math.log(max(V, 2)) + 1)).all())


def test_quant_equal_rows_take_the_lowest_index():
    codes, scales, _ = R.make_head(3000, 4096, 128, BF, False, 3, DEV)
    x = _x(32, 4096, BF, 4)
    head = rpd.QuantHead(codes, scales)
    best = head.stats(x)["argmax"].long()
    # the winners' rows again at the end and in front of everything
    codes2 = torch.cat([codes[best], codes, codes[best]])
    scales2 = torch.cat([scales[best], scales, scales[best]])
    got = rpd.QuantHead(codes2, scales2).stats(x)["argmax"].long()
    y = R.quant_logits(R.dequantize(codes2, scales2, None, 128), x)
    first = (y == y.amax(1, keepdim=True)).int().argmax(1)
    assert torch.equal(got, first)


def test_quant_rows_keep_to_themselves():
    """NaN, infinities and a huge row beside ordinary ones; rows of unaligned stride."""
    codes, scales, z = R.make_head(700, 264, 64, BF, True, 5, DEV)
    head = rpd.QuantHead(codes, scales, z, group=64)
    wide = _x(9, 271, BF, 6)
    x = wide[:, 3:267]
    plain = head.logits(x, out_dtype=F32)
    _check_logits(plain, R.dequantize(codes, scales, z, 64), x, scales.shape[1])
    x[2, 5] = math.nan
    x[4, 7] = math.inf
    x[6] *= 2.0 ** 100
    x[7] *= 2.0 ** -100
    y = head.logits(x, out_dtype=F32)
    assert bool(y[2].isnan().all()) and not bool(y[4].isfinite().any())
    for m in (0, 1, 3, 5, 8):
        assert torch.equal(y[m], plain[m])
    assert torch.equal(y[6], plain[6] * 2.0 ** 100) and torch.equal(y[7], plain[7] * 2.0 ** -100)


@pytest.mark.parametrize("M", [9, 24])
def test_quant_statistics_of_broken_rows(M):
    codes, scales, _ = R.make_head(700, 264, 64, BF, False, 7, DEV)
    head = rpd.QuantHead(codes, scales, group=64)
    x = _x(M, 264, BF, 10)
    plain = head.stats(x)
    x[2, 5] = math.nan
    x[4, 7] = math.inf
    got = head.stats(x)
    assert int(got["argmax"][2]) == -1
    assert all(bool(got[k][m].isnan()) for k, m in (("confidence", 2), ("entropy", 2), ("entropy", 4)))
    keep = [m for m in range(M) if m not in (2, 4)]
    for k in plain:
        assert torch.equal(got[k][keep], plain[k][keep])


def test_quant_out_of_wider_rows_and_nothing_beside_them():
    codes, scales, _ = R.make_head(333, 128, 32, HF, False, 8, DEV)
    head = rpd.QuantHead(codes, scales, group=32)
    x = _x(6, 128, HF, 9)
    buf = torch.full((6, 400), 7.0, dtype=F32, device=DEV)
    head.logits(x, out=buf[:, 20:353])
    assert torch.equal(buf[:, 20:353], head.logits(x, out_dtype=F32))
    assert bool((buf[:, :20] == 7).all()) and bool((buf[:, 353:] == 7).all())
    assert head.logits(x[:0]).shape == (0, 333)
    assert head.stats(x[:0])["argmax"].shape == (0,)
    assert torch.equal(head.logits(x[2]), head.logits(x)[2])
    assert torch.equal(head.logits(x.view(2, 3, 128)).view(6, 333), head.logits(x))


# ----------------------------------------------------------------- verify --

def _rows(g, shape, V, dtype, level=3.0):
    return (level * torch.randn((*shape, V), generator=g)).to(dtype)


def _verify_case(B, T, V, dtype, draft, ragged, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    target = _rows(g, (B, T + 1), V, dtype)
    q = (target[:, :T].float() + torch.randn((B, T, V), generator=g)).to(dtype) if draft else None
    base = q if draft else target[:, :T]
    race = -torch.log(-torch.log(torch.rand((B, T, V), generator=g).clamp_min(1e-20)))
    token = (base.float() * scale + race).argmax(2).int() if T else torch.zeros((B, 0), dtype=torch.int32)
    u = torch.rand((B, T), generator=g)
    r = torch.rand((B,), generator=g)
    lens = torch.randint(-1, T + 2, (B,), generator=g, dtype=torch.int32) if ragged else None
    return target, token, u, r, q, lens


def _check_verify(o, ref, V):
    token, n, accept = ref
    assert torch.equal(o["n_accept"].cpu().long(), n)
    assert torch.equal(o["token"].cpu().long(), token)
    got = o["accept"].cpu().double()
    assert torch.equal(got.isnan(), accept.isnan())
    tol = 2 * R.sum_error(V) * accept + 2.0 ** -23
    ok = ((got - accept).abs() <= tol) | accept.isnan()
    assert bool(ok.all()), float((got - accept).abs().nan_to_num(0).max())


VERIFY = [  # B, T, V, dtype, draft, ragged, scale
    (1, 4, 126464, BF, True, False, 1.0), (3, 1, 1, F32, True, False, 1.0), (5, 3, 7, HF, True, True, 1.0),
    (4, 2, 255, BF, False, False, 0.7), (6, 5, 2049, F32, True, True, 1.5), (2, 0, 4099, BF, True, False, 1.0),
    (40, 7, 997, BF, False, True, 1.0), (9, 12, 5003, HF, True, True, 1.0), (3, 3, 152064, F32, True, False, 0.25),
    (2, 2, 300001, BF, True, False, 1.0), (33, 2, 131, HF, False, False, 2.0),
]


@pytest.mark.parametrize("B,T,V,dtype,draft,ragged,scale", VERIFY)
def test_verify_draft(B, T, V, dtype, draft, ragged, scale):
    note(f"  verify B={B} T={T} V={V} {dtype} draft={draft} ragged={ragged} scale={scale}")
    c = _verify_case(B, T, V, dtype, draft, ragged, B + T + V, scale)
    d = [None if t is None else t.to(DEV) for t in c]
    o = rpd.verify_draft(*d[:4], draft_logits=d[4], draft_len=d[5], target_scale=scale, draft_scale=scale)
    _check_verify(o, R.verify(*c[:4], draft=c[4], lens=c[5], target_scale=scale, draft_scale=scale), V)


@pytest.mark.parametrize("B,T,V,dtype,draft,ragged,scale", VERIFY)
def test_verify_greedy(B, T, V, dtype, draft, ragged, scale):
    note(f"  verify greedy B={B} T={T} V={V} {dtype} ragged={ragged}")
    target, token, _, _, _, lens = _verify_case(B, T, V, dtype, draft, ragged, B + V, scale)
    if T:   # most drafted tokens right; and equal largest entries
        token = torch.where(torch.rand((B, T), generator=torch.Generator().manual_seed(1)) < 0.7,
                            target[:, :T].float().argmax(2).int(), token)
    target[0, 0, :] = 1.0
    o = rpd.verify_draft(target.to(DEV), token.to(DEV), greedy=True, draft_len=None if lens is None else lens.to(DEV))
    _check_verify(o, R.verify(target, token, None, None, lens=lens, greedy=True), V)


def test_verify_scales_that_round():
    """Scaled maxima that are no float32 numbers, over rows of many merges: as exact as scale 1."""
    for scale in (0.7, 1.3):
        c = _verify_case(6, 4, 60001, F32, True, False, 41, scale)
        d = [None if t is None else t.to(DEV) for t in c]
        o = rpd.verify_draft(*d[:4], draft_logits=d[4], target_scale=scale, draft_scale=scale)
        ref = R.verify(*c[:4], draft=c[4], target_scale=scale, draft_scale=scale)
        _check_verify(o, ref, 60001)
        err = (o["accept"].cpu().double() - ref[2]).abs() / ref[2].clamp_min(1e-30)
        # a float32 sum whose terms and chains (12 additions a thread, 8 merges, 30 parts) each round: their errors
        # have either sign, so twice the root of their number, and the exponentials' of arguments down to -16
        assert float(err.max()) <= 2 * (2 * math.sqrt(50) + 16) * 2.0 ** -24


def test_verify_many_rows():
    """Enough logits for float32 statistics (with float64 sums of the sampled rows)."""
    c = _verify_case(48, 7, 32003, BF, True, True, 51, 0.7)
    d = [None if t is None else t.to(DEV) for t in c]
    o = rpd.verify_draft(*d[:4], draft_logits=d[4], draft_len=d[5], target_scale=0.7, draft_scale=0.7)
    _check_verify(o, R.verify(*c[:4], draft=c[4], lens=c[5], target_scale=0.7, draft_scale=0.7), 32003)
    o = rpd.verify_draft(*d[:4], draft_len=d[5], target_scale=0.7)
    _check_verify(o, R.verify(*c[:4], lens=c[5], target_scale=0.7), 32003)


@pytest.mark.parametrize("copies", [1, 900])   # 900: as many rows as take float32 statistics
def test_verify_masked_and_broken_rows(copies):
    V = 3001
    g = torch.Generator().manual_seed(2)
    B, T = 9, 2
    target, draft = _rows(g, (B, T + 1), V, F32), _rows(g, (B, T), V, F32)
    token = torch.zeros((B, T), dtype=torch.int32)
    u, r = torch.full((B, T), 0.5), torch.rand((B,), generator=g)
    lo = torch.finfo(F32).min
    target[0, 0, 1:] = -math.inf                        # only token 0 is left: accepted for certain
    target[1, 0] = -math.inf                            # nothing left
    target[2, 0, 5] = math.nan
    draft[3, 0, 0] = -math.inf                          # drafted though its probability is 0
    target[4, 0, 0] = -math.inf                         # the target excludes the drafted token
    target[5, 0], draft[5, 0] = lo, lo                  # a mask of the lowest value everywhere: flat
    target[6, 0, :], draft[6, 0, :] = -math.inf, -math.inf
    target[6, 0, 7], draft[6, 0, 9] = 0.0, 0.0          # disjoint
    token[7] = torch.tensor([V, -1], dtype=torch.int32)  # outside the vocabulary
    draft[8, 0, 3] = math.inf
    many = lambda t: t.to(DEV).repeat(copies, *[1] * (t.dim() - 1))   # noqa: E731

    def check(o, ref):
        for i in range(0, 9 * copies, 9):
            _check_verify({k: v[i:i + 9] for k, v in o.items()}, ref, V)
    a = [many(t) for t in (target, token, u, r)]
    check(rpd.verify_draft(*a, draft_logits=many(draft)), R.verify(target, token, u, r, draft=draft))
    check(rpd.verify_draft(*a), R.verify(target, token, u, r))
    check(rpd.verify_draft(*a[:2], greedy=True), R.verify(target, token, None, None, greedy=True))


def test_verify_rows_behind_the_draft_are_not_read():
    c = list(_verify_case(6, 4, 1003, BF, True, False, 77))
    lens = torch.tensor([0, 1, 2, 3, 4, 2], dtype=torch.int32)
    for b, n in enumerate(lens.tolist()):
        c[0][b, n + 1:] = math.nan
        c[4][b, n:] = math.nan
    ref = R.verify(*c[:4], draft=c[4], lens=lens)
    d = [t.to(DEV) for t in c[:5]]
    o = rpd.verify_draft(*d[:4], draft_logits=d[4], draft_len=lens.to(DEV))
    _check_verify(o, ref, 1003)
    assert bool(o["accept"].isfinite().all())


def test_verify_draws_follow_the_target():
    """Over equally spaced r the drawn tokens come out as often as the residual says."""
    V, B = 64, 4096
    g = torch.Generator().manual_seed(5)
    t1, q1 = _rows(g, (2,), V, F32, 1.5), _rows(g, (1,), V, F32, 1.5)
    target = t1.expand(B, 2, V).to(DEV)      # one row for every sequence: batch stride 0
    draft = q1.expand(B, 1, V).to(DEV)
    token = torch.full((B, 1), 3, dtype=torch.int32, device=DEV)
    r = ((torch.arange(B) + 0.5) / B).to(DEV)
    o = rpd.verify_draft(target, token, torch.full((B, 1), 0.99999, device=DEV), r, draft_logits=draft)
    p, q = t1[0].double().softmax(0), q1[0].double().softmax(0)
    a = min(1.0, float(p[3] / q[3]))
    w = (p - q).clamp_min(0) if a < 0.99999 else t1[1].double().softmax(0)
    want = w / w.sum()
    got = torch.bincount(o["token"][:, 0 if a < 0.99999 else 1].cpu().long(), minlength=V).double() / B
    assert float((got - want).abs().max()) <= 1.0 / B + 1e-9   # equally spaced points: at most one off


def test_verify_strided_logits():
    """Draft and target rows as a serving program keeps them: one padded buffer, sequences in another order."""
    c = _verify_case(4, 3, 501, HF, True, False, 9)
    buf = torch.zeros((4, 4, 512), dtype=HF, device=DEV)
    buf[:, :, 5:506] = c[0].to(DEV)
    qbuf = torch.zeros((3, 4, 640), dtype=HF, device=DEV)
    qbuf[:, :, 1:502] = c[4].to(DEV).transpose(0, 1)
    d = [t.to(DEV) for t in c[:4]]
    o = rpd.verify_draft(buf[:, :, 5:506], d[1], d[2], d[3], draft_logits=qbuf[:, :, 1:502].transpose(0, 1))
    _check_verify(o, R.verify(*c[:4], draft=c[4]), 501)


# ---------------------------------------------------------------- distill --

def _distill_case(N, V, k, dtype, tail, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    z = 2.0 * torch.randn((N, V), generator=g)
    logits = (z + torch.randn((N, V), generator=g)).to(dtype)
    kk = min(k, V)
    top, ids = z.topk(kk, dim=1)
    if kk < k:   # padded
        ids = torch.cat([ids, torch.full((N, k - kk), -1)], 1)
        top = torch.cat([top, torch.zeros((N, k - kk))], 1)
    lse = torch.logsumexp(z.double() * scale, 1).float() if tail else None
    up = torch.randn((N,), generator=g)
    weight = (torch.rand((N,), generator=g) < 0.8).float() * (0.5 + torch.rand((N,), generator=g))
    return logits, ids.int(), top, lse, weight, up


def _check_distill(loss, grad, ref, V, scale=1.0):
    rl, rg, terms = ref
    e = R.sum_error(V)
    tol = 2 * e * (1 + rl.abs())
    d = (loss.detach().cpu().double() - rl).abs()
    assert bool((d <= tol).all()), (float(d.max()), float(rl.abs().max()))
    if grad is None:
        return
    g = grad.cpu().double()
    tol = 2 * e * terms + R.half_step(grad.dtype) * 1.01 * (rg.abs() + 2 * e * terms) + 1e-30
    if grad.dtype == HF:
        tol = tol + 2.0 ** -25
    if grad.dtype == BF:
        tol = tol + 2.0 ** -134
    d = (g - rg).abs()
    assert bool((d <= tol).all()), (int((d > tol).sum()), float((d - tol).max()))


DISTILL = [  # N, V, k, dtype, tail, scale
    (8, 12647, 32, BF, False, 1.0), (1, 1, 1, F32, False, 1.0), (2, 1, 3, BF, True, 1.0), (3, 7, 4, HF, True, 0.5),
    (5, 2047, 1, F32, True, 1.0), (5, 2049, 64, BF, True, 2.0), (17, 4999, 100, HF, False, 1.0),
    (300, 777, 256, F32, True, 0.5), (4, 126464, 64, BF, True, 1.0), (2, 200003, 50, F32, False, 0.7),
    (3, 262147, 33, HF, True, 1.0), (600, 513, 16, BF, True, 1.0),
]


@pytest.mark.parametrize("N,V,k,dtype,tail,scale", DISTILL)
def test_distill(N, V, k, dtype, tail, scale):
    note(f"  distill N={N} V={V} k={k} {dtype} tail={tail} scale={scale}")
    scale = float(np.float32(scale))
    c = _distill_case(N, V, k, dtype, tail, N + V + k, scale)
    ref = R.distill(*c, scale=scale)
    logits, ids, top, lse, weight, up = [None if t is None else t.to(DEV) for t in c]
    logits.requires_grad_(True)
    loss = rpd.distill(logits, ids, top, teacher_lse=lse, weight=weight, logit_scale=scale)
    grad, = torch.autograd.grad(loss, logits, up)
    _check_distill(loss, grad, ref, V, scale)
    loss2, grad2 = rpd.distill_grad(logits, ids, top, teacher_lse=lse, weight=weight, grad_loss=up, logit_scale=scale)
    _check_distill(loss2, grad2, ref, V, scale)


def test_distill_lists_padded_repeated_and_empty():
    V = 3001
    logits, ids, top, lse, _, up = _distill_case(6, V, 12, F32, True, 3)
    ids[0, 5:] = -1
    ids[1, 3] = ids[1, 7] = ids[1, 9]           # one token three times
    ids[2, :] = -1                              # no list
    ids[3, 4] = V                               # outside
    top[4, 2] = -math.inf                       # probability 0
    ids[5, :] = ids[5, 0]
    top = top - 1.5                             # a larger rest
    for tail in (None, lse):
        ref = R.distill(logits, ids, top, tail, None, up)
        a = [t.to(DEV) for t in (logits, ids, top)]
        loss, grad = rpd.distill_grad(*a, teacher_lse=None if tail is None else tail.to(DEV), grad_loss=up.to(DEV))
        _check_distill(loss, grad, ref, V)
    assert float(loss[2]) == 0.0 or lse is not None


def test_distill_rows_of_weight_zero_are_not_read():
    logits, ids, top, lse, _, up = _distill_case(9, 5000, 20, BF, True, 4)
    weight = torch.tensor([1., 0., 1., 0., 0., 2., 1., 0., .5])
    ref = R.distill(logits, ids, top, lse, weight, up)
    logits[weight == 0] = math.nan
    lse[weight == 0] = math.nan
    top[weight == 0] = math.nan
    up[weight == 0] = math.nan
    a = [t.to(DEV) for t in (logits, ids, top, lse, weight, up)]
    loss, grad = rpd.distill_grad(*a)
    _check_distill(loss, grad, ref, 5000)
    assert not bool(grad[1].any()) and float(loss[1]) == 0.0


def test_distill_sure_students_and_masked_entries():
    """A student hundreds of nats above its tail; -inf and the type's lowest value in the row; a list over everything."""
    V = 4000
    logits, ids, top, lse, _, up = _distill_case(6, V, 8, F32, True, 6)
    logits[0, int(ids[0, 0])] = 400.0
    logits[1, 1234] = 300.0
    outside = torch.ones(V, dtype=torch.bool)
    outside[ids[2].long()] = False
    logits[2, outside.nonzero()[10:, 0]] = -math.inf
    logits[3, outside.nonzero()[10:, 0]] = torch.finfo(F32).min
    ref = R.distill(logits, ids, top, lse, None, up)
    a = [t.to(DEV) for t in (logits, ids, top, lse)]
    loss, grad = rpd.distill_grad(*a, grad_loss=up.to(DEV))
    _check_distill(loss, grad, ref, V)
    # the list's token masked out: the loss is infinite, the gradient is not
    logits[4, ids[4, 1].long()] = -math.inf
    loss, grad = rpd.distill_grad(logits.to(DEV), *a[1:], grad_loss=up.to(DEV))
    assert math.isinf(float(loss[4])) and bool(grad[4].isfinite().all())
    logits[5, 17] = math.nan
    loss, grad = rpd.distill_grad(logits.to(DEV), *a[1:], grad_loss=up.to(DEV))
    assert math.isnan(float(loss[5])) and bool(loss[:4].isfinite().all())


def test_distill_gradient_by_differences():
    V, h = 600, 1.0 / 16
    logits, ids, top, lse, _, _ = _distill_case(1, V, 6, F32, True, 8)
    at = [int(ids[0, 0]), int(ids[0, 3]), 5, 599, int(logits[0].argmax())]
    a = [t.to(DEV) for t in (ids, top, lse)]
    _, grad = rpd.distill_grad(logits.to(DEV), *a)
    rows = logits.repeat(2 * len(at), 1)
    for i, v in enumerate(at):
        rows[2 * i, v] += h
        rows[2 * i + 1, v] -= h
    n = rows.shape[0]
    loss = rpd.distill(rows.to(DEV), a[0].repeat(n, 1), a[1].repeat(n, 1), teacher_lse=a[2].repeat(n)).cpu().double()
    noise = 2 * R.sum_error(V) * (1 + float(loss.abs().max()))
    for i, v in enumerate(at):
        diff = float(loss[2 * i] - loss[2 * i + 1]) / (2 * h)
        # the third derivative of the log-sum-exps is at most 2 (one over everything, one over the tail)
        assert abs(diff - float(grad[0, v])) <= noise / h + 2 * h * h / 6 + 1e-6


def test_distill_autograd_broadcast_upstream_and_leading_dimensions():
    logits, ids, top, lse, weight, _ = _distill_case(12, 999, 10, BF, True, 11)
    a = [t.to(DEV).view(3, 4, *t.shape[1:]) for t in (logits, ids, top, lse, weight)]
    x = a[0].clone().requires_grad_(True)
    rpd.distill(x, a[1], a[2], teacher_lse=a[3], weight=a[4]).mean().backward()
    loss, g = rpd.distill_grad(*a[:3], teacher_lse=a[3], weight=a[4], grad_loss=torch.full((3, 4), 1 / 12, device=DEV))
    assert loss.shape == (3, 4) and torch.equal(x.grad, g)
    wide = torch.zeros((12, 1010), dtype=BF, device=DEV)
    wide[:, 7:1006] = logits.to(DEV)
    view = wide[:, 7:1006]
    loss2, g2 = rpd.distill_grad(view, *[t.view(12, *t.shape[2:]) for t in a[1:3]], teacher_lse=a[3].view(12),
                                 weight=a[4].view(12), grad_loss=torch.full((12,), 1 / 12, device=DEV))
    assert torch.equal(loss2.view(3, 4), loss) and torch.equal(g2.view(3, 4, 999), g)
    empty, eg = rpd.distill_grad(view[:0], *[t.view(12, *t.shape[2:])[:0] for t in a[1:3]])
    assert empty.shape == (0,) and eg.shape == (0, 999)


# ------------------------------------------------------- streams, graphs, together --

def test_operators_on_a_stream_and_in_graphs():
    """Each operator captured and replayed on new inputs, with eager work between, equals its eager results."""
    codes, scales, _ = R.make_head(2000, 512, 128, BF, False, 12, DEV)
    head = rpd.QuantHead(codes, scales)
    x = _x(8, 512, BF, 13)
    c = _verify_case(4, 3, 2000, BF, True, False, 14)
    target, token, u, r, q = [t.to(DEV) for t in c[:5]]
    logits, ids, top, lse, weight, up = [t.to(DEV) for t in _distill_case(8, 2000, 16, BF, True, 15)]
    verify = rpd.VerifyDraft(target, token, u, r, draft_logits=q)
    torch.cuda.synchronize()

    def step():
        s = head.stats(x)
        o = verify()
        loss, grad = rpd.distill_grad(logits, ids, top, teacher_lse=lse, weight=weight, grad_loss=up)
        return [head.logits(x), *s.values(), *o.values(), loss, grad]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        eager = [t.clone() for t in step()]
    side.synchronize()
    for a, b in zip(step(), eager):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(_x(8, 512, BF, 20 + i))
        u.copy_(torch.rand((4, 3), generator=torch.Generator().manual_seed(i)))
        logits.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in held]
        for a, b in zip(step(), again):
            assert torch.equal(a, b)


def test_operators_together():
    """A drafter's head trained a step against the target's top logits, served in 4 bits: its statistics decide
    commitments, its logits propose tokens, and the target verifies them."""
    K, B, L, d, V = 2, 1, 24, 256, 3000
    g = torch.Generator().manual_seed(30)
    codes, scales, _ = R.make_head(V, d, 64, BF, False, 31, DEV)
    head = rpd.QuantHead(codes, scales, group=64)
    w = R.dequantize(codes, scales, None, 64)
    hidden = torch.randn((K, B, L, d), generator=g).to(BF).to(DEV)
    mask = (torch.rand((B, L), generator=g) < 0.7).to(torch.uint8).to(DEV)
    # statistics of the 4-bit head into the commitment, against the same rows through the float64 head
    s = head.stats(hidden, logit_scale=0.3)
    out = rpd.gate_commit(mask, s["argmax"], s["confidence"], s["entropy"], rpd.Params.llada())
    y = R.quant_logits(w, hidden.view(-1, d)) * float(np.float32(0.3))
    at, c, h = R.stats(y)
    want = rpd.gate_commit(mask, at.int().view(K, B, L), c.float().view(K, B, L), h.float().view(K, B, L),
                           rpd.Params.llada())
    assert torch.equal(out["commit"], want["commit"]) and torch.equal(out["token"], want["token"])
    # drafted tokens of four positions, verified by another model's logits
    T = 4
    q = head.logits(hidden[-1, :, :T])
    target = torch.cat([q, q[:, :1]], 1) + 0.5 * torch.randn((B, T + 1, V), generator=g).to(BF).to(DEV)
    token = out["token"][:, :T].contiguous()
    token = torch.where(token < 0, q.float().argmax(2).int(), token)
    u, r = torch.rand((B, T), generator=g), torch.rand((B,), generator=g)
    o = rpd.verify_draft(target, token, u.to(DEV), r.to(DEV), draft_logits=q)
    _check_verify(o, R.verify(target.cpu(), token.cpu(), u, r, draft=q.cpu()), V)
    # and the drafter's logits distilled towards the target's
    top, ids = target[:, :T].float().topk(32, dim=2)
    lse = torch.logsumexp(target[:, :T].float(), 2)
    x = q.clone().requires_grad_(True)
    loss = rpd.distill(x, ids.int(), top, teacher_lse=lse, weight=mask[:, :T].float())
    loss.sum().backward()
    ref = R.distill(q[0].cpu(), ids[0].int().cpu(), top[0].cpu(), lse[0].cpu(), mask[0, :T].float().cpu())
    _check_distill(loss[0], x.grad[0], ref, V)


# ------------------------------------------------------------ long rows, far apart --

def test_verify_parts_longer_than_a_workgroup_holds():
    V = 1200007
    c = _verify_case(1, 1, V, F32, True, False, 61)
    d = [t.to(DEV) for t in c[:5]]
    o = rpd.verify_draft(*d[:4], draft_logits=d[4])
    _check_verify(o, R.verify(*c[:4], draft=c[4]), V)
    o = rpd.verify_draft(*d[:2], greedy=True)
    _check_verify(o, R.verify(*c[:2], None, None, greedy=True), V)


def test_verify_many_short_sequences():
    c = _verify_case(5000, 1, 7, HF, True, True, 62)
    d = [t.to(DEV) for t in c]
    o = rpd.verify_draft(*d[:4], draft_logits=d[4], draft_len=d[5])
    _check_verify(o, R.verify(*c[:4], draft=c[4], lens=c[5]), 7)


@pytest.mark.parametrize("V,dtype", [(1 << 20, BF), (700001, F32)])
def test_distill_parts_longer_than_a_workgroup_holds(V, dtype):
    c = _distill_case(2, V, 256, dtype, True, 63)
    ref = R.distill(*c)
    logits, ids, top, lse, weight, up = [t.to(DEV) for t in c]
    loss, grad = rpd.distill_grad(logits, ids, top, teacher_lse=lse, weight=weight, grad_loss=up)
    _check_distill(loss, grad, ref, V)


def _apart(rows):
    """The same rows more than 2^31 elements apart."""
    n, step = rows.shape[-1], (1 << 31) + 8
    far = torch.empty(((rows.shape[0] - 1) * step + n,), dtype=rows.dtype, device=DEV)
    view = far.as_strided(rows.shape, (step, 1))
    view.copy_(rows)
    return view


def test_rows_further_apart_than_32_bits():
    codes, scales, _ = R.make_head(1003, 256, 64, BF, False, 64, DEV)
    head = rpd.QuantHead(codes, scales, group=64)
    x = _x(3, 256, BF, 65)
    near = head.logits(x)
    out = _apart(torch.zeros_like(near))
    head.logits(_apart(x), out=out)
    assert torch.equal(out, near)
    del out
    c = _verify_case(1, 2, 1003, BF, True, False, 66)
    target, token, u, r, q = [t.to(DEV) for t in c[:5]]
    want = rpd.verify_draft(target, token, u, r, draft_logits=q)
    got = rpd.verify_draft(_apart(target[0])[None], token, u, r, draft_logits=_apart(q[0])[None])
    for k in want:
        assert torch.equal(got[k], want[k])
    logits, ids, top, lse, weight, up = [t.to(DEV) for t in _distill_case(3, 1003, 16, BF, True, 67)]
    a = (ids, top, lse, None, up)
    for got, want in zip(rpd.distill_grad(_apart(logits), *a), rpd.distill_grad(logits, *a)):
        assert torch.equal(got, want)


# ---------------------------------------------------------------- calls of no rows --

def test_no_rows():
    codes, scales, _ = R.make_head(100, 64, 32, HF, False, 68, DEV)
    head = rpd.QuantHead(codes, scales, group=32)
    x = torch.empty((2, 0, 64), dtype=HF, device=DEV)
    assert head.logits(x).shape == (2, 0, 100)
    assert all(v.shape == (2, 0) for v in head.stats(x).values())
    logits = torch.empty((0, 50), dtype=F32, device=DEV, requires_grad=True)
    loss = rpd.distill(logits, torch.empty((0, 4), dtype=torch.int32, device=DEV), torch.empty((0, 4), device=DEV))
    grad, = torch.autograd.grad(loss.sum(), logits)
    assert loss.shape == (0,) and grad.shape == (0, 50)


# ------------------------------------------------------------------------ autograd --

def test_distill_backward_from_saved_tensors_that_moved():
    """A strided view saved on the host comes back dense, at another address."""
    wide = _rows(torch.Generator().manual_seed(69), (6,), 1500, BF).to(DEV)
    _, ids, top, lse, weight, up = [t.to(DEV) for t in _distill_case(6, 999, 10, BF, True, 70)]
    _, want = rpd.distill_grad(wide[:, :999], ids, top, lse, weight, up)
    x = wide[:, :999].detach().requires_grad_(True)
    with torch.autograd.graph.save_on_cpu():
        loss = rpd.distill(x, ids, top, lse, weight)
    grad, = torch.autograd.grad(loss, x, up)
    assert torch.equal(grad, want)


def test_distill_forward_and_backward_in_a_graph():
    """Captured with gradients by autograd; every replay on new logits equals the eager call, which runs between."""
    _, ids, top, lse, weight, up = [t.to(DEV) for t in _distill_case(7, 2500, 12, F32, True, 71)]
    x = torch.zeros((7, 2500), device=DEV, requires_grad=True)

    def step():
        loss = rpd.distill(x, ids, top, teacher_lse=lse, weight=weight)
        return loss.detach(), torch.autograd.grad(loss, x, up)[0]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # what the first backward pass sets up is not captured
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        with torch.no_grad():
            x.copy_(_rows(torch.Generator().manual_seed(seed), (7,), 2500, F32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for a, b in zip(got, rpd.distill_grad(x, ids, top, lse, weight, up)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls that overlap on two streams, each with objects or workspaces of its own, over one packed head."""
    codes, scales, _ = R.make_head(30011, 1024, 128, BF, False, 72, DEV)
    head = rpd.QuantHead(codes, scales)
    xs = [_x(24, 1024, BF, 73 + i) for i in range(2)]
    cases = [[t.to(DEV) for t in _verify_case(6, 3, 30011, BF, True, False, 75 + i)[:5]] for i in range(2)]
    calls = [rpd.VerifyDraft(*c[:4], draft_logits=c[4]) for c in cases]

    def work(i):
        o = calls[i]()
        return [head.logits(xs[i]), *head.stats(xs[i]).values(), *[t.clone() for t in o.values()]]

    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(work(i))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[i]))
