"""What the operators beside the commit step refuse, on the host, before anything is enqueued; and the float64 forms
that their GPU tests compare with."""
import ctypes
import math

import pytest
import torch

from paper_2609_36452_amd import binding as rpd
from tests import operators_ref as R

P = 4096   # non-NULL, never dereferenced


def _head(**kw):
    a = dict(V=1000, d=256, group=64, dtype=rpd.DTYPE_BF16, has_zeros=0)
    a.update(kw)
    return rpd.RpdQuantHead(*[a[n] for n in ("V", "d", "group", "dtype", "has_zeros")])


@pytest.mark.parametrize("kw,status", [
    (dict(V=0), 2), (dict(V=1 << 28), 2), (dict(d=0), 2), (dict(d=12), 2), (dict(d=(1 << 20) + 8), 2),
    (dict(V=1 << 22, d=(1 << 14) + 8), 2), (dict(group=16), 5), (dict(group=0), 5), (dict(group=256), 5),
    (dict(dtype=rpd.DTYPE_F32), 5), (dict(dtype=9), 5), (dict(has_zeros=2), 3)])
def test_quant_head_refusals(kw, status):
    h = _head(**kw)
    L = rpd.lib()
    assert L.rpd_quant_packed_size(ctypes.byref(h)) == 0
    assert L.rpd_quant_workspace_size(ctypes.byref(h), 4, 1) == 0
    assert L.rpd_quant_pack(ctypes.byref(h), P, P, None, P, 1 << 40, None) == status
    assert L.rpd_quant_project(ctypes.byref(h), P, 1, P, 1 << 21, P, 1 << 29, h.dtype, None, None, None, 1.0, None, 0,
                               None) == status
    assert rpd.last_error()


def test_quant_sizes():
    L = rpd.lib()
    # 63 tiles of 16 rows, 2 chunks of 128 columns, 1 KB of codes each; 4 groups a row
    codes, entries = 63 * 2 * 1024, 63 * 16 * 4
    r = lambda n: (n + 255) // 256 * 256   # noqa: E731
    assert L.rpd_quant_packed_size(ctypes.byref(_head())) == codes + r(2 * entries)
    assert L.rpd_quant_packed_size(ctypes.byref(_head(has_zeros=1))) == codes + r(2 * entries) + r(entries)
    assert L.rpd_quant_workspace_size(ctypes.byref(_head()), 3, 0) == 0
    assert L.rpd_quant_workspace_size(ctypes.byref(_head()), 3, 1) == r(3 * 64 * 16)   # 63 tiles in 64 slots
    # more than 16 rows are laid out first: 2 tiles of 16 rows, their groups' sums and exponents
    assert L.rpd_quant_workspace_size(ctypes.byref(_head()), 17, 0) == 2 * 2 * 4096 + r(2 * 64)
    assert L.rpd_quant_packed_size(None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(packed=None), 1), (dict(zeros=P), 1), (dict(scales=P + 1), 5),
    (dict(packed=P + 16), 5), (dict(nbytes=1000), 4)])
def test_quant_pack_refusals(kw, status):
    a = dict(codes=P, scales=P, zeros=None, packed=P, nbytes=1 << 30)
    a.update(kw)
    s = rpd.lib().rpd_quant_pack(ctypes.byref(_head()), a["codes"], a["scales"], a["zeros"], a["packed"], a["nbytes"], None)
    assert s == status
    assert rpd.lib().rpd_quant_pack(None, P, P, None, P, 1 << 30, None) == 1
    assert rpd.lib().rpd_quant_pack(ctypes.byref(_head(has_zeros=1)), P, P, None, P, 1 << 30, None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), 2), (dict(M=(1 << 20) + 1), 2), (dict(xs=255), 2), (dict(os=999), 2), (dict(ot=rpd.DTYPE_F16), 5),
    (dict(ot=7), 5), (dict(scale=-1.0), 3), (dict(scale=math.nan), 3), (dict(scale=math.inf), 3), (dict(packed=None), 1),
    (dict(x=None), 1), (dict(out=None), 1), (dict(am=P), 1), (dict(out=None, am=P, cf=P), 1),
    (dict(out=None, am=P, cf=P, en=P, ws=None), 1), (dict(out=None, am=P, cf=P, en=P, ws=P + 8), 5),
    (dict(out=None, am=P, cf=P, en=P, nbytes=16), 4), (dict(packed=P + 2), 5), (dict(x=P + 1), 5), (dict(out=P + 1), 5),
    (dict(out=None, am=P + 2, cf=P, en=P), 5)])
def test_quant_project_refusals(kw, status):
    a = dict(packed=P, M=4, x=P, xs=256, out=P, os=1000, ot=rpd.DTYPE_BF16, am=None, cf=None, en=None, scale=1.0, ws=P,
             nbytes=1 << 30)
    a.update(kw)
    s = rpd.lib().rpd_quant_project(ctypes.byref(_head()), a["packed"], a["M"], a["x"], a["xs"], a["out"], a["os"],
                                    a["ot"], a["am"], a["cf"], a["en"], a["scale"], a["ws"], a["nbytes"], None)
    assert s == status and rpd.last_error()


def test_empty_calls_do_nothing():
    L = rpd.lib()
    assert L.rpd_quant_project(ctypes.byref(_head()), None, 0, None, 256, None, 0, 0, None, None, None, 1.0, None, 0,
                               None) == 0
    p = _distill(N=0, logits=None, id=None, teacher=None, state=None, loss=None)
    assert L.rpd_distill_loss(ctypes.byref(p), None, 0, None) == 0
    assert L.rpd_distill_workspace_size(ctypes.byref(p)) == 0


def _verify(**kw):
    a = dict(B=2, T=3, V=100, dtype=0, target=P, tb=400, tr=100, draft=P, db=300, dr=100, token=P, len=P, u=P, r=P,
             ts=1.0, ds=1.0, flags=0, out=P, n=P, accept=P)
    a.update(kw)
    return rpd.RpdVerify(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 2), (dict(T=-1), 2), (dict(V=0), 2), (dict(V=(1 << 28) + 1), 2), (dict(B=1 << 20, T=1), 2),
    (dict(tb=-1), 2), (dict(dr=-1), 2), (dict(dtype=3), 5), (dict(flags=2), 3), (dict(ts=math.nan), 3),
    (dict(ds=-0.5), 3), (dict(ds=math.inf), 3), (dict(target=None), 1), (dict(token=None), 1), (dict(u=None), 1),
    (dict(r=None), 1), (dict(out=None), 1), (dict(n=None), 1), (dict(accept=None), 1), (dict(target=P + 1), 5),
    (dict(token=P + 2), 5), (dict(dtype=1, draft=P + 2), 5), (dict(B=1 << 10, T=1000, V=1 << 28), 2)])
def test_verify_refusals(kw, status):
    p = _verify(**kw)
    assert rpd.lib().rpd_verify_draft(ctypes.byref(p), P, 1 << 50, None) == status
    assert rpd.last_error()


def test_verify_workspace_refusals():
    L = rpd.lib()
    p = _verify()
    n = L.rpd_verify_workspace_size(ctypes.byref(p))
    assert n > 0
    assert L.rpd_verify_draft(ctypes.byref(p), None, n, None) == 1
    assert L.rpd_verify_draft(ctypes.byref(p), P + 128, n, None) == 5
    assert L.rpd_verify_draft(ctypes.byref(p), P, n - 1, None) == 4
    assert L.rpd_verify_draft(None, P, n, None) == 1


def test_verify_workspace_of_many_sequences():
    """A launch holds fewer than 2^24 workgroups: the parts of a row grow with the sequences."""
    L = rpd.lib()

    def size(B):
        return L.rpd_verify_workspace_size(ctypes.byref(_verify(B=B, T=0, V=32000, draft=None)))

    # per sequence: 4 parts' statistics of 16 bytes, a pick of 32, and float64 sums of 2 rows and their totals in 16
    # parts, or 8 where 16 of them are too many
    assert size(1 << 19) == (1 << 19) * (4 * 16 + 32 + 2 * 16 * 16)
    assert size(1 << 20) == (1 << 20) * (4 * 16 + 32 + 2 * 8 * 16)


def _distill(**kw):
    a = dict(N=4, V=100, k=8, dtype=0, teacher_dtype=1, logits=P, logits_stride=100, id=P, teacher=P, teacher_lse=P,
             weight=P, grad_loss=P, logit_scale=1.0, loss=P, state=P, grad=2 * P, grad_stride=100)
    a.update(kw)
    return rpd.RpdDistill(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), 2), (dict(N=(1 << 24) + 1), 2), (dict(V=0), 2), (dict(V=(1 << 20) + 1), 2), (dict(k=0), 2),
    (dict(k=257), 2), (dict(dtype=4), 5), (dict(teacher_dtype=-1), 5), (dict(logit_scale=math.nan), 3),
    (dict(logit_scale=-2.0), 3), (dict(logits_stride=99), 2), (dict(grad_stride=99), 2), (dict(logits=None), 1),
    (dict(id=None), 1), (dict(teacher=None), 1), (dict(state=None), 1), (dict(id=P + 2), 5), (dict(logits=P + 1), 5),
    (dict(weight=P + 1), 5), (dict(grad=P), 3), (dict(N=1 << 24), 2),
    (dict(N=(1 << 24) - 1, V=1 << 20, logits_stride=1 << 20, grad_stride=1 << 20), 2)])
def test_distill_refusals(kw, status):
    L = rpd.lib()
    p = _distill(**kw)
    assert L.rpd_distill_loss(ctypes.byref(p), P, 1 << 50, None) == status
    assert rpd.last_error()
    assert L.rpd_distill_grad(ctypes.byref(p), None) == status


def test_distill_workspace_refusals():
    L = rpd.lib()
    p = _distill()
    n = L.rpd_distill_workspace_size(ctypes.byref(p))
    assert L.rpd_distill_loss(ctypes.byref(p), None, n, None) == 1
    assert L.rpd_distill_loss(ctypes.byref(p), P + 8, n, None) == 5
    assert L.rpd_distill_loss(ctypes.byref(p), P, n - 1, None) == 4
    assert L.rpd_distill_loss(ctypes.byref(_distill(loss=None)), P, n, None) == 1
    assert L.rpd_distill_grad(ctypes.byref(_distill(grad=None)), None) == 1


def test_binding_refuses_host_tensors():
    codes, scales, _ = R.make_head(32, 64, 32, torch.bfloat16, False, 1, "cpu")
    with pytest.raises(ValueError):
        rpd.QuantHead(codes, scales, group=32)
    z = torch.zeros((2, 3, 10))
    with pytest.raises(ValueError):
        rpd.verify_draft(z, torch.zeros((2, 2), dtype=torch.int32), torch.zeros((2, 2)), torch.zeros(2))
    with pytest.raises(ValueError):
        rpd.distill(z[0], torch.zeros((3, 1), dtype=torch.int32), torch.zeros((3, 1)))


def test_float64_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    z = torch.randn((1, 40), generator=g, dtype=torch.float64)
    ids = torch.tensor([[3, 7, 7, -1, 12]], dtype=torch.int32)
    t = torch.randn((1, 5), generator=g, dtype=torch.float64)
    for lse in (None, torch.tensor([3.0])):
        _, grad, _ = R.distill(z, ids, t, lse, scale=0.5)
        for v in (0, 3, 7, 12, 39):
            h, a, b = 1e-4, z.clone(), z.clone()
            a[0, v] += h
            b[0, v] -= h
            diff = (R.distill(a, ids, t, lse, scale=0.5)[0] - R.distill(b, ids, t, lse, scale=0.5)[0]) / (2 * h)
            assert abs(float(diff[0]) - float(grad[0, v])) < 1e-7


def test_float64_draws_are_the_residual():
    V = 16
    g = torch.Generator().manual_seed(4)
    target, draft = torch.randn((1, 2, V), generator=g), torch.randn((1, 1, V), generator=g)
    p, q = target[0, 0].double().softmax(0), draft[0, 0].double().softmax(0)
    x = int((q - p).argmax())
    w = (p - q).clamp_min(0)
    w = w / w.sum()
    for i in range(50):
        r = torch.tensor([(i + 0.5) / 50])
        token, n, a = R.verify(target, torch.tensor([[x]], dtype=torch.int32), torch.tensor([[0.99999]]), r, draft=draft)
        assert int(n[0]) == 0 and abs(float(a[0, 0]) - float(p[x] / q[x])) < 1e-12
        v = int(token[0, 0])
        assert float(w[:v].sum()) <= float(r) + 1e-7 < float(w[:v + 1].sum()) + 1e-6
