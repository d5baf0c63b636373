"""The operators beside the commit step where their values or sizes go to the ends of what a call may hold, against plain
float64 forms."""
import math

import pytest
import torch

from paper_2609_36452_amd import binding as rpd
from tests import operators_ref as R
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def _f32(scale):
    return float(torch.tensor(scale, dtype=F32))


def _dev(*tensors):
    return [None if t is None else t.to(DEV) for t in tensors]


# ---------------------------------------------------------------- distill --

def _distill(logits, ids, top, lse=None, up=None, scale=1.0):
    """loss [N], gradient [N][V] and the magnitude of its terms in float64; differences of logits before their scale, so
    that rows far from 0 keep them."""
    N, V = logits.shape
    up = torch.ones(N) if up is None else up
    losses, grads, terms = torch.zeros(N).double(), torch.zeros((N, V)).double(), torch.zeros((N, V)).double()
    for n in range(N):
        at = ids[n].long()[(ids[n] >= 0) & (ids[n] < V)]
        t = top[n].double()[(ids[n] >= 0) & (ids[n] < V)]
        p = ((t - t.max()) * scale).softmax(0) if lse is None else (t * scale - float(lse[n])).exp()
        inside = torch.zeros(V, dtype=torch.bool).index_fill_(0, at, True)
        rest = 0.0 if lse is None or bool(inside.all()) else max(0.0, 1.0 - float(p.sum()))
        z = logits[n].double()
        ln_S = ((z - z.max()) * scale).exp().sum().log()
        log_q = (z - z.max()) * scale - ln_S
        some = p > 0
        loss = (p[some] * (p[some].log() - log_q[at][some])).sum()
        share = torch.zeros(V, dtype=torch.float64).scatter_add(0, at, p)
        tail = torch.zeros(V, dtype=torch.float64)
        if rest > 0:
            o = z[~inside]
            ln_T = ((o - o.max()) * scale).exp().sum().log()
            loss = loss + rest * (math.log(rest) - ((o.max() - z.max()) * scale + ln_T - ln_S))
            tail = torch.where(inside, tail, rest * ((z - o.max()) * scale - ln_T).exp())
        q = (float(p.sum()) + rest) * log_q.exp()
        c = float(up[n]) * scale
        losses[n], grads[n], terms[n] = loss, c * (q - share - tail), abs(c) * (q + share + tail)
    return losses, grads, terms


def _check_loss_and_grad(loss, grad, ref, V):
    """As far from the float64 form as float32 sums allow; infinite where that is above float32's range."""
    rl, rg, terms = ref
    e = 2 * R.sum_error(V)
    loss, rl = loss.detach().cpu().double(), rl.float().double()
    assert torch.equal(loss.isinf(), rl.isinf()) and bool(((loss == rl) | ((loss - rl).abs() <= e * (1 + rl.abs()))).all()), \
        (loss, rl)
    g = grad.cpu().double()
    step = R.half_step(grad.dtype) * 1.01 * (rg.abs() + e * terms) + torch.finfo(grad.dtype).smallest_normal
    assert bool(((g - rg).abs() <= e * terms + step).all()), float((g - rg).abs().nan_to_num(math.inf).max())


def _masked_students(V, dtype, value, tail, scale, seed):
    """Rows of logits with `value` in places, a teacher's list of 12 tokens in each; what stays is ordinary."""
    g = torch.Generator().manual_seed(seed)
    N, k = 6, 12
    z = 2.0 * torch.randn((N, V), generator=g)
    z[:, 1024:1032] -= 40.0                          # eight neighbours and the second half, never listed
    z[:, V // 2:] -= 40.0
    top, ids = z.topk(k, dim=1)
    logits = (z + torch.randn((N, V), generator=g)).to(dtype)
    outside = torch.ones((N, V), dtype=torch.bool).scatter_(1, ids, False)
    logits[0, 1024:1032] = value
    logits[1, V // 2:] = value
    logits[2, outside[2].nonzero()[10:, 0]] = value  # an allow-list
    logits[3, outside[3]] = value                    # nothing but the list
    logits[4] = value                                # flat
    logits[5, V - 8:] = value                        # padding behind the vocabulary
    lse = torch.logsumexp(z.double() * scale, 1).float() if tail else None
    return logits, ids.int(), top, lse, 0.5 + torch.rand((N,), generator=g)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("scale", [0.7, 1.0, 1.25, 2.0])
@pytest.mark.parametrize("dtype,value", [(BF, "lowest"), (F32, "lowest"), (F32, -1e10), (BF, -1e30)])
def test_distill_masks_of_any_value(dtype, value, scale, tail):
    note(f"  distill masked {dtype} {value} scale={scale} tail={tail}")
    V, scale = 8192, _f32(scale)
    value = torch.finfo(dtype).min if value == "lowest" else value
    logits, ids, top, lse, up = _masked_students(V, dtype, value, tail, scale, 80)
    ref = _distill(logits, ids, top, lse, up, scale)
    a = _dev(logits, ids, top, lse, up)
    loss, grad = rpd.distill_grad(*a[:3], teacher_lse=a[3], grad_loss=a[4], logit_scale=scale)
    _check_loss_and_grad(loss, grad, ref, V)
    x = a[0].clone().requires_grad_(True)
    loss = rpd.distill(x, *a[1:3], teacher_lse=a[3], logit_scale=scale)
    _check_loss_and_grad(loss, torch.autograd.grad(loss, x, a[4])[0], ref, V)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_masks_in_long_parts(dtype):
    """So many rows that a part is as long as a thread can hold."""
    V, copies, scale = 32768, 200, 1.25
    logits, ids, top, lse, up = _masked_students(V, dtype, torch.finfo(dtype).min, True, scale, 81)
    ref = _distill(logits, ids, top, lse, up, scale)
    a = [t.to(DEV).repeat(copies, *[1] * (t.dim() - 1)) for t in (logits, ids, top, lse, up)]
    loss, grad = rpd.distill_grad(*a[:3], teacher_lse=a[3], grad_loss=a[4], logit_scale=scale)
    _check_loss_and_grad(loss[:6], grad[:6], ref, V)
    assert torch.equal(loss.view(copies, 6), loss[:6].expand(copies, 6))
    assert bool((grad.view(copies, 6, V) == grad[:6]).all())


@pytest.mark.parametrize("scale", [3e8, 1e30])
def test_distill_scales_that_leave_one_token(scale):
    V, scale = 3000, _f32(scale)
    g = torch.Generator().manual_seed(82)
    logits = 2.0 * torch.randn((3, V), generator=g)
    ids = torch.tensor([[5, 9], [7, -1], [int(logits[2].argmax()), 4]], dtype=torch.int32)
    top = torch.tensor([[1.0, 1.0], [2.0, 0.0], [3.0, 1.0]])
    ref = _distill(logits, ids, top, scale=scale)
    loss, grad = rpd.distill_grad(*_dev(logits, ids, top), logit_scale=scale)
    _check_loss_and_grad(loss, grad, ref, V)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_teachers_of_lowest_values(dtype):
    """A teacher that masks what it lists: flat over the list, or its one other token."""
    V, scale = 2500, 2.0
    g = torch.Generator().manual_seed(83)
    logits = torch.randn((2, V), generator=g)
    ids = torch.tensor([[3, 700, 2400], [8, 9, 10]], dtype=torch.int32)
    top = torch.full((2, 3), torch.finfo(dtype).min, dtype=dtype)
    top[1, 1] = 1.0
    ref = _distill(logits, ids, top, scale=scale)
    loss, grad = rpd.distill_grad(*_dev(logits, ids, top), logit_scale=scale)
    _check_loss_and_grad(loss, grad, ref, V)


@pytest.mark.parametrize("V,k", [(1, 1), (50, 50), (50, 64), (256, 256)])
def test_distill_lists_of_the_whole_vocabulary(V, k):
    """No token is outside the list, whatever the teacher's rounded sum leaves for one."""
    g = torch.Generator().manual_seed(88 + V)
    N = 40
    z = 2.0 * torch.randn((N, V), generator=g)
    ids = torch.full((N, k), -1, dtype=torch.int32)
    ids[:, :V] = torch.stack([torch.randperm(V, generator=g) for _ in range(N)]).int()
    top = torch.zeros((N, k))
    top[:, :V] = z.gather(1, ids[:, :V].long())
    logits = z + torch.randn((N, V), generator=g)
    lse = torch.logsumexp(z, 1)
    lse[::2] += 1e-3                         # in these rows the list's mass is below 1 for certain
    loss, grad = rpd.distill_grad(*_dev(logits, ids, top), teacher_lse=lse.to(DEV))
    _check_loss_and_grad(loss, grad, _distill(logits, ids, top, lse), V)


# ----------------------------------------------------------------- verify --

def _check_verify(o, ref, V):
    token, n, accept = ref
    got = o["accept"].cpu().double()
    assert torch.equal(got.isnan(), accept.isnan()), (got, accept)
    assert bool((((got - accept).abs() <= 2 * R.sum_error(V) * accept + 2.0 ** -23) | accept.isnan()).all()), (got, accept)
    assert torch.equal(o["n_accept"].cpu().long(), n) and torch.equal(o["token"].cpu().long(), token)


@pytest.mark.parametrize("copies", [1, 14, 40])   # float64 statistics, float32 ones, and those of longer parts
@pytest.mark.parametrize("scales", [(1.5, 0.7), (0.9, 1.25)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_verify_masks_of_any_value(dtype, scales, copies):
    note(f"  verify masked {dtype} scales={scales} copies={copies}")
    V, B, T = 20011, 9, 2
    g = torch.Generator().manual_seed(84)
    target = 3.0 * torch.randn((B, T + 1, V), generator=g)
    draft = target[:, :T] + torch.randn((B, T, V), generator=g)
    lo = torch.finfo(dtype).min
    some = torch.randperm(V, generator=g)[20:]
    target[0, :, some] = lo                          # an allow-list
    draft[0, :, some] = lo
    target[1, :, 8192:16384] = lo                    # whole parts
    draft[2, :, 8192:16384] = lo
    target[3, :, 16384:], draft[3, :, 16384:] = lo, lo
    target[4], draft[4] = lo, lo                     # flat
    target[5, :, 2048:8192] = -1e10
    target[6, :, 2048:8192], draft[6, :, :9000] = -1e30, -1e30
    token = draft.argmax(2).int()
    target[7, 0, int(token[7, 0])] = lo              # the drafted token masked out
    draft[8, 0, 5] = lo                              # drafted though masked out
    token[8, 0] = 5
    token[4] = 11
    target, draft = target.to(dtype), draft.to(dtype)
    u, r = torch.rand((B, T), generator=g), torch.rand((B,), generator=g)
    ts, ds = scales
    many = [t.to(DEV).repeat(copies, *[1] * (t.dim() - 1)) for t in (target, token, u, r, draft)]
    for q in (draft, None):
        ref = R.verify(target, token, u, r, draft=q, target_scale=ts, draft_scale=ds)
        o = rpd.verify_draft(*many[:4], draft_logits=None if q is None else many[4], target_scale=ts, draft_scale=ds)
        for i in (0, B * (copies - 1)):
            _check_verify({k: v[i:i + B] for k, v in o.items()}, ref, V)
        for v in o.values():
            assert torch.equal(v.view(copies, -1), v[:B].view(1, -1).expand(copies, -1))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_parts_of_two_rounds(dtype):
    """Rows of a length and number whose parts are longer than a workgroup's threads hold at once."""
    V, copies, scale = 300001, 30, 1.25
    logits, ids, top, lse, up = _masked_students(V, dtype, torch.finfo(dtype).min, True, scale, 89)
    ref = _distill(logits, ids, top, lse, up, scale)
    a = [t.to(DEV).repeat(copies, *[1] * (t.dim() - 1)) for t in (logits, ids, top, lse, up)]
    loss, grad = rpd.distill_grad(*a[:3], teacher_lse=a[3], grad_loss=a[4], logit_scale=scale)
    _check_loss_and_grad(loss[:6], grad[:6], ref, V)
    assert torch.equal(loss.view(copies, 6), loss[:6].expand(copies, 6))
    assert bool((grad.view(copies, 6, V) == grad[:6]).all())


@pytest.mark.parametrize("greedy", [False, True])
def test_verify_parts_of_two_rounds(greedy):
    """Rows of a length and number whose parts are longer than a workgroup's threads hold at once."""
    V, B, T, copies = 300001, 3, 2, 24
    g = torch.Generator().manual_seed(95)
    target = (3.0 * torch.randn((B, T + 1, V), generator=g)).to(BF)
    draft = (target[:, :T].float() + torch.randn((B, T, V), generator=g)).to(BF)
    target[1, :, 12288:40000] = torch.finfo(BF).min
    target[2, 0, 200000] = target[2, 0].max()            # equal largest entries
    token = (target[:, :T] if greedy else draft).float().argmax(2).int()
    u, r = torch.rand((B, T), generator=g), torch.rand((B,), generator=g)
    ref = R.verify(target, token, u, r, draft=draft, target_scale=1.5, draft_scale=0.7, greedy=greedy)
    many = [t.to(DEV).repeat(copies, *[1] * (t.dim() - 1)) for t in (target, token, u, r, draft)]
    o = rpd.verify_draft(*many[:4], draft_logits=many[4], target_scale=1.5, draft_scale=0.7, greedy=greedy)
    for i in (0, B * (copies - 1)):
        _check_verify({k: v[i:i + B] for k, v in o.items()}, ref, V)
    for v in o.values():
        assert torch.equal(v.view(copies, -1), v[:B].view(1, -1).expand(copies, -1))


@pytest.mark.parametrize("copies", [1, 25])   # float64 and float32 statistics
def test_verify_scales_of_their_own(copies):
    """Target and draft at different temperatures: neither scale taken for the other's."""
    V, B, T = 40009, 4, 3
    g = torch.Generator().manual_seed(85)
    target = (3.0 * torch.randn((B, T + 1, V), generator=g)).to(HF)
    draft = (target[:, :T].float() + torch.randn((B, T, V), generator=g)).to(HF)
    token = draft.float().argmax(2).int()
    u, r = torch.rand((B, T), generator=g), torch.rand((B,), generator=g)
    ref = R.verify(target, token, u, r, draft=draft, target_scale=0.6, draft_scale=1.4)
    many = [t.to(DEV).repeat(copies, *[1] * (t.dim() - 1)) for t in (target, token, u, r, draft)]
    o = rpd.verify_draft(*many[:4], draft_logits=many[4], target_scale=0.6, draft_scale=1.4)
    for i in range(0, B * copies, B):
        _check_verify({k: v[i:i + B] for k, v in o.items()}, ref, V)


@pytest.mark.parametrize("teacher_dtype", [BF, HF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_teachers_of_each_type(dtype, teacher_dtype):
    V, k, scale = 3001, 40, 0.5
    g = torch.Generator().manual_seed(86)
    z = 2.0 * torch.randn((5, V), generator=g)
    top, ids = z.topk(k, dim=1)
    top, ids, logits = top.to(teacher_dtype), ids.int(), (z + torch.randn((5, V), generator=g)).to(dtype)
    ids[1, 7] = ids[1, 2]
    up = torch.rand((5,), generator=g)
    for lse in (None, torch.logsumexp(z.double() * scale, 1).float()):
        ref = _distill(logits, ids, top, lse, up, scale)
        a = _dev(logits, ids, top, lse, up)
        loss, grad = rpd.distill_grad(*a[:3], teacher_lse=a[3], grad_loss=a[4], logit_scale=scale)
        _check_loss_and_grad(loss, grad, ref, V)


def test_distill_empty_lists_have_no_loss():
    logits = torch.randn((3, 2100), generator=torch.Generator().manual_seed(87))
    ids = torch.tensor([[-1, -1], [5, 6], [2100, -7]], dtype=torch.int32)
    top = torch.zeros((3, 2))
    top[1] = -math.inf                       # listed, of probability 0
    loss, grad = rpd.distill_grad(*_dev(logits, ids, top))
    assert loss.tolist() == [0.0, 0.0, 0.0] and not bool(grad.any())


# ------------------------------------------------------------------ quant --

def _bound(w, x, groups, lost):
    """A logit's error: every term is rounded with its product and scale and goes through the additions of its group,
    of the groups and of at most 16 waves; an element of x may be off by `lost` of its row's largest."""
    terms = torch.matmul(x.double().abs(), w.abs().t().contiguous())
    off = lost * x.double().abs().amax(1, keepdim=True) * w.abs().sum(1).unsqueeze(0)
    return (128 + groups + 16 + 4) * R.U32 * terms + off


def _check_logits(y, w, x, groups, lost=0.0):
    ref = R.quant_logits(w, x)
    err = (y.double() - ref).abs()
    assert bool((err <= _bound(w, x, groups, lost)).all()), float(err.max())
    # the roundings of a logit's additions have either sign: over many logits they add up as their number's root does,
    # and none is of more than the logits themselves
    norm = err.norm(dim=1) / ref.norm(dim=1)
    off = lost * x.double().abs().amax(1) * w.abs().sum(1).norm() / ref.norm(dim=1)
    assert bool((norm <= math.sqrt(128 + groups + 20) * R.U32 + off).all()), norm


def _small(V, d, group, dtype, zeros, seed):
    codes, scales, z = R.make_head(V, d, group, dtype, zeros, seed, DEV)
    return rpd.QuantHead(codes, scales, z, group=group), R.dequantize(codes, scales, z, group), scales.shape[1]


@pytest.mark.parametrize("M", [3, 16, 24])   # rows converted by their readers, or laid out before
@pytest.mark.parametrize("level", [-22, -18, -14])
def test_quant_fp16_rows_of_small_elements(level, M):
    """fp16 rows among the type's subnormal numbers are as exact as any."""
    head, w, groups = _small(2003, 1024, 128, HF, True, 90)
    x = torch.randn((M, 1024), generator=torch.Generator().manual_seed(91)) * 2.0 ** level
    x[1, 5] = 1.0                            # one row of small elements beside a large one
    x = x.to(HF).to(DEV)
    _check_logits(head.logits(x, out_dtype=F32), w, x, groups)
    big = (x.float() * 2.0 ** 10).to(HF)     # far from them; the first row's elements are the same numbers scaled
    assert torch.equal((x.float() * 2.0 ** 10)[0], big[0].float())
    assert torch.equal(head.logits(x[:1], out_dtype=F32) * 2.0 ** 10, head.logits(big[:1], out_dtype=F32))


@pytest.mark.parametrize("M", [2, 20])
def test_quant_bf16_rows_of_a_wide_range(M):
    """An element of 2^20 whose weights are all 0 beside elements 2^28 to 2^36 times smaller: what they lose is 2^-39 of
    the largest, as the contract says, and nothing else."""
    V, d = 1500, 512
    codes, scales, _ = R.make_head(V, d, 128, BF, False, 92, DEV)
    codes[:, 100] = codes[:, 100] & 0xf0 | 8           # column 200
    head, w = rpd.QuantHead(codes, scales), R.dequantize(codes, scales, None, 128)
    assert not bool(w[:, 200].any())
    g = torch.Generator().manual_seed(93)
    x = 2.0 ** (20 - 28 - 8 * torch.rand((M, d), generator=g)) * (1.0 - 2.0 * torch.randint(0, 2, (M, d), generator=g))
    x[:, 200] = 2.0 ** 20
    x = x.to(BF).to(DEV)
    y, ref = head.logits(x, out_dtype=F32).double(), R.quant_logits(w, x)
    rest = x.clone()
    rest[:, 200] = 0                                   # the large element's terms are 0
    off = 2.0 ** -39 * 2.0 ** 20 * w.abs().sum(1).unsqueeze(0)
    assert bool(((y - ref).abs() <= _bound(w, rest, 4, 0.0) + off).all()), float((y - ref).abs().max())


STREAMS = [  # M, d, V, group, dtype, zeros: several tiles of the vocabulary to a workgroup
    (1, 4096, 20011, 128, BF, False), (13, 3584, 20011, 64, HF, True), (16, 4096, 9001, 32, BF, True),
    (32, 4096, 20003, 128, BF, False), (64, 4096, 9001, 128, BF, False), (27, 2048, 17001, 64, HF, True),
    (9, 2048, 24007, 128, BF, False), (5, 512, 70001, 32, HF, False), (100, 1024, 9001, 64, BF, True),
    (3, 9000, 9001, 128, BF, True), (20, 9000, 5003, 64, HF, False), (2, 7168, 13001, 128, BF, False),
]


@pytest.mark.parametrize("M,d,V,group,dtype,zeros", STREAMS)
def test_quant_streams_many_tiles(M, d, V, group, dtype, zeros):
    note(f"  quant streams M={M} d={d} V={V} group={group} {dtype} zeros={zeros}")
    head, w, groups = _small(V, d, group, dtype, zeros, V + d)
    x = torch.randn((M, d), generator=torch.Generator().manual_seed(V)).to(dtype).to(DEV)
    lost = 2.0 ** -39 if dtype == BF else 0.0
    _check_logits(head.logits(x, out_dtype=F32), w, x, groups, lost)
    o = head.stats(x, logit_scale=0.5)
    y = R.quant_logits(w, x) * 0.5
    delta = (_bound(w, x, groups, lost) * 0.5 + R.U32 * y.abs()).amax(1)
    at, c, h = R.stats(y)
    got = o["argmax"].long()
    assert bool(((got >= 0) & (got < V)).all())
    assert bool((y.gather(1, got.unsqueeze(1)).squeeze(1) >= y.amax(1) - 2 * delta).all())
    # a sum of positive terms: the tiles of a workgroup, 16 columns, the workgroups, and exponentials of down to -24
    chain = (V / 16 / 256 + 16 + 40 + 2 * 24) * R.U32
    rel = torch.expm1(2 * delta) + 2 * chain
    assert bool(((o["confidence"].double() - c).abs() <= rel * c).all())
    assert bool(((o["entropy"].double() - h).abs() <= 2 * rel * (h + math.log(V) + 1)).all())


@pytest.mark.parametrize("M", [1, 20])
def test_quant_statistics_of_an_infinite_logit(M):
    """A logit above float32's range, alone in its row: e^(inf - inf) is no number, in whichever tile it falls."""
    V, d = 5000, 256
    codes = torch.full((V, d // 2), 0x88, dtype=torch.uint8)
    scales = torch.ones((V, 2), dtype=BF)
    for at in (0, 4321):
        c = codes.clone()
        c[at, 3] = 0x8f                     # weight 7 at column 6, where every other token has 0
        head = rpd.QuantHead(c.to(DEV), scales.to(DEV))
        x = torch.randn((M, d), generator=torch.Generator().manual_seed(94)).to(BF).to(DEV)
        plain = head.stats(x)
        x[0, 6] = 3e38
        got = head.stats(x)
        assert bool(head.logits(x, out_dtype=F32)[0, at].isinf()) and int(got["argmax"][0]) == at
        assert bool(got["confidence"][0].isnan()) and bool(got["entropy"][0].isnan())
        for k in plain:
            assert torch.equal(got[k][1:], plain[k][1:])
