"""What 8-bit blocks, the head in them and sampling refuse, on the host, before anything is enqueued; and the float64
forms that their GPU tests compare with."""
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


def test_quantize_nothing():
    assert rpd.lib().rpd_fp8_quantize(0, 200, 0, None, 200, 1, None, 200, None, None) == 0


@pytest.mark.parametrize("V,d", [(0, 128), (128, 0), ((1 << 20) + 1, 8), (8, (1 << 20) + 1), (1 << 19, (1 << 17) + 1)])
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
    # rows as bf16 operands, blocks of 16 x 128; a state for each of 4 tiles
    assert L.rpd_fp8_workspace_size(1000, 200, 17, 0) == 2 * 2 * 4096
    assert L.rpd_fp8_workspace_size(1000, 200, 17, 1) == 2 * 2 * 4096 + r(17 * 4 * 16)
    # a long sum in parts of 4 chunks or more: 20 chunks, 5 parts
    assert L.rpd_fp8_workspace_size(1000, 20 * 128, 1, 0) == 20 * 4096 + r(5 * 63 * 64)
    assert L.rpd_fp8_workspace_size(1000, 200, 0, 0) == 0 and L.rpd_fp8_workspace_size(1000, 200, (1 << 20) + 1, 0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(packed=None), 1), (dict(scales=P + 2), 5), (dict(packed=P + 16), 5),
    (dict(nbytes=1000), 4), (dict(tr=2), 3)])
def test_pack_refusals(kw, status):
    a = dict(codes=P, scales=P, packed=P, nbytes=1 << 30, tr=0)
    a.update(kw)
    assert rpd.lib().rpd_fp8_pack(1000, 200, a["codes"], a["scales"], a["tr"], a["packed"], a["nbytes"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), 2), (dict(M=(1 << 20) + 1), 2), (dict(xt=5), 5), (dict(xs=199), 2), (dict(os=999), 2), (dict(ot=7), 5),
    (dict(scale=-1.0), 3), (dict(scale=math.nan), 3), (dict(scale=math.inf), 3), (dict(packed=None), 1), (dict(x=None), 1),
    (dict(out=None), 1), (dict(am=P), 1), (dict(out=None, am=P, cf=P), 1), (dict(packed=P + 2), 5), (dict(x=P + 1), 5),
    (dict(out=P + 1), 5), (dict(ot=rpd.DTYPE_F32, out=P + 2), 5), (dict(out=None, am=P + 2, cf=P, en=P), 5),
    (dict(ws=None), 1), (dict(ws=P + 8), 5), (dict(nbytes=16), 4)])
def test_project_refusals(kw, status):
    a = dict(packed=P, M=4, x=P, xs=200, xt=rpd.DTYPE_BF16, out=P, os=1000, ot=rpd.DTYPE_BF16, am=None, cf=None, en=None,
             scale=1.0, ws=P, nbytes=1 << 30)
    a.update(kw)
    s = rpd.lib().rpd_fp8_project(1000, 200, a["packed"], a["M"], a["x"], a["xs"], a["xt"], a["out"], a["os"], a["ot"],
                                  a["am"], a["cf"], a["en"], a["scale"], a["ws"], a["nbytes"], None)
    assert s == status and rpd.last_error()


def test_python_refusals():
    """Host tensors, before the library is asked."""
    codes, scales = R.make_head(10, 20, 1, "cpu")
    with pytest.raises(ValueError):
        rpd.Fp8Head(codes, scales)
    with pytest.raises(ValueError):
        rpd.fp8_quantize(torch.zeros((2, 2)))


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
