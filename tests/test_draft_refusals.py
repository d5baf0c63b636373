"""What 8-bit blocks, the head in them and sampling refuse, on the host, before anything is enqueued; and the float64
forms that their GPU tests compare with."""
import ctypes
import math

import pytest
import torch

from paper_2609_36452_amd import binding as rpd
from tests import draft_ref as R

P = 1 << 20   # non-NULL, never dereferenced


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 2), (dict(rows=(1 << 28) + 1), 2), (dict(d=0), 2), (dict(d=(1 << 28) + 1), 2), (dict(dtype=3), 5),
    (dict(dtype=-1), 5), (dict(per=0), 3), (dict(per=64), 3), (dict(xs=199), 2), (dict(cs=199), 2),
    (dict(rows=1 << 28, d=1 << 10, xs=1 << 10, cs=1 << 10), 2), (dict(x=None), 1), (dict(codes=None), 1),
    (dict(scales=None), 1), (dict(x=P + 1), 5), (dict(dtype=rpd.DTYPE_F32, x=P + 2), 5), (dict(scales=2 * P + 2), 5),
    (dict(codes=P), 3), (dict(codes=P + 1999), 3), (dict(scales=P + 1996), 3), (dict(codes=2 * P + 8, scales=2 * P), 3),
    (dict(codes=P - 999), 3)])
def test_quantize_refusals(kw, status):
    a = dict(rows=5, d=200, dtype=rpd.DTYPE_BF16, x=P, xs=200, per=1, codes=3 * P, cs=200, scales=2 * P)
    a.update(kw)
    s = rpd.lib().rpd_fp8_quantize(a["rows"], a["d"], a["dtype"], a["x"], a["xs"], a["per"], a["codes"], a["cs"],
                                   a["scales"], None)
    assert s == status and rpd.last_error()


def test_rows_between_each_other_are_apart():
    """Rows of one stride may lie between each other: such calls pass the check (and end at another one, before anything
    is enqueued)."""
    L = rpd.lib()
    # a row of 40 of x, then 30 logits, in rows of 70 elements of 2 bytes; a workspace too small ends the call
    project = lambda out, os: L.rpd_fp8_project(30, 40, P, 40, P, 70, 0, out, os, 0, None, None, None, 1.0, P, 16, None)   # noqa: E731
    assert project(P + 80, 70) == 4 and project(P + 78, 70) == 3 and project(P - 60, 70) == 4
    assert project(P + 80, 71) == 3 and project(P + 70 * 2 * 40, 71) == 4


def test_quantize_nothing():
    assert rpd.lib().rpd_fp8_quantize(0, 200, 0, None, 200, 1, None, 200, None, None) == 0


@pytest.mark.parametrize("V,d", [(0, 128), (128, 0), ((1 << 20) + 1, 8), (8, (1 << 20) + 1), (1 << 18, (1 << 17) + 1)])
def test_head_refusals(V, d):
    L = rpd.lib()
    assert L.rpd_fp8_packed_size(V, d) == 0 and L.rpd_fp8_workspace_size(V, d, 4, 0) == 0
    assert L.rpd_fp8_pack(V, d, P, P, 0, P, 1 << 40, None) == 2
    assert L.rpd_fp8_project(V, d, P, 1, P, 1 << 21, 0, P, 1 << 21, 0, None, None, None, 1.0, P, 1 << 40, None) == 2


def test_head_sizes():
    L = rpd.lib()
    r = lambda n: (n + 255) // 256 * 256   # noqa: E731
    # 63 tiles of 16 rows, 2 chunks of 128 columns, 2 KB each; 8 x 2 scales
    assert L.rpd_fp8_packed_size(1000, 200) == 63 * 2 * 2048 + r(8 * 2 * 4)
    # more than 16 rows as bf16 operands, blocks of 16 x 128; a state for each of 4 tiles
    assert L.rpd_fp8_workspace_size(1000, 200, 33, 0) == 3 * 2 * 4096
    assert L.rpd_fp8_workspace_size(1000, 200, 33, 1) == 3 * 2 * 4096 + r(33 * 4 * 16)
    assert L.rpd_fp8_workspace_size(1000, 200, 17, 0) == 2 * 2 * 4096
    assert L.rpd_fp8_workspace_size(1000, 200, 16, 0) == 0 and L.rpd_fp8_workspace_size(1000, 200, 16, 1) == r(16 * 64)
    # a long sum in parts of 4 chunks or more: 20 chunks, 5 parts; the statistics of those need no states
    assert L.rpd_fp8_workspace_size(1000, 20 * 128, 1, 0) == r(5 * 63 * 64)
    assert L.rpd_fp8_workspace_size(1000, 20 * 128, 40, 1) == 3 * 20 * 4096 + r(5 * 40 * 63 * 64)
    assert L.rpd_fp8_workspace_size(1000, 200, 0, 0) == 0 and L.rpd_fp8_workspace_size(1000, 200, (1 << 20) + 1, 0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(packed=None), 1), (dict(scales=P + 2), 5), (dict(packed=P + 16), 5),
    (dict(nbytes=1000), 4), (dict(tr=2), 3), (dict(codes=2 * P), 3), (dict(scales=2 * P), 3),
    (dict(codes=2 * P - 199999), 3), (dict(codes=2 * P + 63 * 2 * 2048), 3), (dict(scales=2 * P - 60, tr=1), 3)])
def test_pack_refusals(kw, status):
    a = dict(codes=P, scales=P, packed=2 * P, nbytes=1 << 30, tr=0)
    a.update(kw)
    assert rpd.lib().rpd_fp8_pack(1000, 200, a["codes"], a["scales"], a["tr"], a["packed"], a["nbytes"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), 2), (dict(M=(1 << 20) + 1), 2), (dict(xt=5), 5), (dict(xs=199), 2), (dict(os=999), 2), (dict(ot=7), 5),
    (dict(scale=-1.0), 3), (dict(scale=math.nan), 3), (dict(scale=math.inf), 3), (dict(packed=None), 1), (dict(x=None), 1),
    (dict(out=None), 1), (dict(am=P), 1), (dict(out=None, am=P, cf=P), 1), (dict(packed=P + 2), 5), (dict(x=P + 1), 5),
    (dict(out=P + 1), 5), (dict(ot=rpd.DTYPE_F32, out=P + 2), 5), (dict(out=P), 3), (dict(out=P + 15998), 3),
    (dict(out=P - 79998), 3), (dict(xt=rpd.DTYPE_F32, out=P + 31998), 3), (dict(out=None, am=P + 2, cf=P, en=P), 5),
    (dict(ws=None), 1), (dict(ws=P + 8), 5), (dict(nbytes=16), 4)])
def test_project_refusals(kw, status):
    a = dict(packed=P, M=40, x=P, xs=200, xt=rpd.DTYPE_BF16, out=2 * P, os=1000, ot=rpd.DTYPE_BF16, am=None, cf=None, en=None,
             scale=1.0, ws=P, nbytes=1 << 30)
    a.update(kw)
    s = rpd.lib().rpd_fp8_project(1000, 200, a["packed"], a["M"], a["x"], a["xs"], a["xt"], a["out"], a["os"], a["ot"],
                                  a["am"], a["cf"], a["en"], a["scale"], a["ws"], a["nbytes"], None)
    assert s == status and rpd.last_error()


@pytest.mark.parametrize("V,d,M,logits", [
    (126464, 4096, 135000, False), (126464, 4096, 136000, False), (126464, 4096, 1 << 20, False), (126464, 4096, 136000, True),
    (152064, 3584, 1 << 20, True), (1 << 18, 128, 1 << 20, False), (1 << 18, 128, 1 << 20, True), (5, 1 << 16, 1 << 20, False),
    (5, 1 << 16, 1 << 20, True)])
def test_project_takes_many_rows(V, d, M, logits):
    """Rows up to the bounds of rpd.h, among them those whose logits would be more than 2^34, pass the checks of shape:
    such calls end at the workspace, before anything is enqueued."""
    L = rpd.lib()
    need = L.rpd_fp8_workspace_size(V, d, M, int(not logits))
    assert need > 0
    out = (P << 22, V, 0, None, None, None) if logits else (None, 0, 0, P, P, P)
    assert L.rpd_fp8_project(V, d, P, M, P, d, 0, *out, 1.0, P, need - 1, None) == 4


@pytest.mark.parametrize("V,d,M", [((1 << 18) + 1, 128, 1 << 20), (1 << 20, 128, (1 << 18) + 1), (5, (1 << 16) + 1, 1 << 20),
                                   (5, 1 << 20, (1 << 16) + 1)])
def test_project_refuses_more_rows_than_launches_hold(V, d, M):
    L = rpd.lib()
    assert L.rpd_fp8_workspace_size(V, d, M, 0) == 0 and L.rpd_fp8_workspace_size(V, d, M, 1) == 0
    assert L.rpd_fp8_project(V, d, P, M, P, d, 0, P << 22, V, 0, None, None, None, 1.0, P, 1 << 50, None) == 2
    assert L.rpd_fp8_project(V, d, P, M, P, d, 0, None, 0, 0, P, P, P, 1.0, P, 1 << 50, None) == 2
    assert "M*V" in rpd.last_error()


def test_python_refusals():
    """Host tensors, before the library is asked."""
    codes, scales = R.make_head(10, 20, 1, "cpu")
    with pytest.raises(ValueError):
        rpd.Fp8Head(codes, scales)
    with pytest.raises(ValueError):
        rpd.fp8_quantize(torch.zeros((2, 2)))


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("train", [False, True])
def test_dual_tensors_are_refused(train, grad):
    """Forward mode has no rule to go by: its tangent is not dropped in silence."""
    head = object.__new__(rpd.Fp8Head)
    head.V, head.d, head.train = 10, 20, train
    x = torch.ones((2, 20), requires_grad=grad)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(NotImplementedError, match="forward-mode"):
            head.logits(torch.autograd.forward_ad.make_dual(x, torch.ones((2, 20))))
        with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
            head.logits(torch.autograd.forward_ad.make_dual(x, torch.ones((2, 20))), out=torch.empty((2, 10)))


# ------------------------------------------------------- the float64 forms --

def test_reference_codes_are_torch_casts():
    g = torch.Generator().manual_seed(1)
    x = torch.randn((130, 300), generator=g) * (3.0 * torch.randn((300,), generator=g)).exp()
    for per in (1, 128):
        codes, scales = R.quantize(x, per)
        s = scales.repeat_interleave(128, 1)[:, :300].repeat_interleave(per, 0)[:130]
        assert torch.equal((x.double() / s).float().to(torch.float8_e4m3fn).double(), codes)
        assert bool((codes.abs() <= 448).all()) and bool((torch.frexp(scales)[0] == 0.5).all())
        # with half the scale the largest would not fit
        top = torch.nn.functional.pad(x.abs(), (0, 84, 0, -130 % per)).double().view(-(-130 // per), per, 3, 128).amax((1, 3))
        assert bool((top <= 448 * scales).all()) and bool((top > 224 * scales).all())


# --------------------------------------------------------------- sampling --

def _sample(**kw):
    a = dict(N=4, V=1000, dtype=rpd.DTYPE_BF16, logits=P, ls=1000, r=2 * P, scale=1.0, k=0, p=1.0, least=0.0, scales=None,
             ks=None, ps=None, leasts=None, token=3 * P, prob=3 * P, kept=3 * P, filtered=None, fs=0)
    a.update(kw)
    return rpd.RpdSample(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), 2), (dict(N=1 << 22), 2), (dict(V=0), 2), (dict(V=(1 << 20) + 1, ls=1 << 21), 2), (dict(dtype=4), 5),
    (dict(ls=999), 2), (dict(filtered=4 * P, fs=999), 2), (dict(scale=-1.0), 3), (dict(scale=math.nan), 3),
    (dict(scale=math.inf), 3), (dict(scale=1.3e30), 3), (dict(k=-1), 3), (dict(p=0.0), 3), (dict(p=-0.5), 3), (dict(p=math.nan), 3),
    (dict(least=-0.1), 3), (dict(least=1.1), 3), (dict(least=math.nan), 3), (dict(logits=None), 1), (dict(r=None), 1),
    (dict(token=None), 1), (dict(logits=P + 1), 5), (dict(dtype=rpd.DTYPE_F32, logits=P + 2), 5), (dict(r=P + 2), 5),
    (dict(token=P + 1), 5), (dict(prob=P + 2), 5), (dict(kept=P + 2), 5), (dict(scales=P + 2), 5), (dict(ks=P + 2), 5),
    (dict(ps=P + 2), 5), (dict(leasts=P + 2), 5), (dict(filtered=4 * P + 1, fs=1000), 5), (dict(filtered=P, fs=1000), 3),
    (dict(filtered=P + 7998, fs=1000), 3), (dict(filtered=P - 7998, fs=1000), 3)])
def test_sample_refusals(kw, status):
    assert rpd.lib().rpd_sample_tokens(ctypes.byref(_sample(**kw)), P, 1 << 40, None) == status
    assert rpd.last_error()


@pytest.mark.parametrize("top_k", [-1, 2.5, -2**32 + 5])
def test_sample_whole_top_k(top_k):
    with pytest.raises(ValueError, match="top_k"):
        rpd.sample(torch.zeros((2, 8)), torch.zeros((2,)), top_k=top_k)


def test_sample_needs_no_workspace():
    for kw in (dict(), dict(N=1 << 20, V=1 << 20, ls=1 << 20), dict(V=0)):
        assert rpd.lib().rpd_sample_workspace_size(ctypes.byref(_sample(**kw))) == 0


def test_sample_nothing():
    assert rpd.lib().rpd_sample_tokens(ctypes.byref(_sample(N=0, logits=None)), None, 0, None) == 0
    assert rpd.lib().rpd_sample_tokens(None, None, 0, None) == 1


def test_reference_sample():
    """The definition on a row that is known by hand: masses 4, 2, 1, 1 by halves."""
    z = torch.log(torch.tensor([1.0, 4.0, 1.0, 2.0], dtype=torch.float64))
    ok = dict(scale=1.0, top_k=0, top_p=1.0, min_p=0.0)
    R.check_sample(z, 0.49, **ok, token=1, prob=0.5, kept=4)
    R.check_sample(z, 0.51, **ok, token=3, prob=0.25, kept=4)
    R.check_sample(z, 0.76, **ok, token=0, prob=0.125, kept=4)
    R.check_sample(z, 0.9, **{**ok, "top_k": 2}, token=3, prob=1 / 3, kept=2)
    R.check_sample(z, 0.2, **{**ok, "top_p": 0.4}, token=1, prob=1.0, kept=1)
    R.check_sample(z, 0.9, **{**ok, "min_p": 0.4}, token=3, prob=1 / 3, kept=2)
    for wrong in (dict(token=3, prob=0.25, kept=4), dict(token=1, prob=0.4, kept=4), dict(token=1, prob=0.5, kept=3)):
        with pytest.raises(AssertionError):
            R.check_sample(z, 0.49, **ok, **wrong)
