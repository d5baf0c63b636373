"""Quantization to 8-bit blocks and the output head in them against plain float64 forms."""
import ctypes
import math

import pytest
import torch

from paper_2609_36452_amd import binding as rpd
from tests import draft_ref as R
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF, F32, E4 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
DTYPES = [BF, HF, F32]


def _x(M, d, dtype, seed, level=1.0):
    g = torch.Generator().manual_seed(seed)
    return (level * torch.randn((M, d), generator=g)).to(dtype).to(DEV)


def _check_codes(x, per):
    codes, scales = rpd.fp8_quantize(x, block_rows=per)
    want, ws = R.quantize(x.reshape(-1, x.shape[-1]), per)
    assert codes.shape == x.shape and codes.dtype == E4 and scales.dtype == F32
    assert torch.equal(scales.reshape(ws.shape).double(), ws)
    got = codes.float().double().reshape(want.shape)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(), want.nan_to_num())
    return codes, scales


# ---------------------------------------------------------- quantization --

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 128), (3, 129), (17, 200), (16, 127), (5, 4096), (300, 1000), (130, 7)])
@pytest.mark.parametrize("per", [1, 128])
def test_quantize(rows, d, dtype, per):
    note(f"  fp8 quantize {rows} x {d} {dtype} per {per}")
    g = torch.Generator().manual_seed(rows + d)
    x = (torch.randn((rows, d), generator=g) * (2.0 * torch.randn((d,), generator=g)).exp()).to(dtype).to(DEV)
    _check_codes(x, per)


def test_quantize_every_bf16_value():
    """Every bf16 magnitude up to 448 beside a 448, which keeps the scale 1: all roundings, subnormals and ties."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF)
    v = v[v.float().abs() <= 448.0]
    n = -(-v.numel() // 127)
    x = torch.zeros((n, 128), dtype=BF)
    x[:, 0] = 448.0
    x[:, 1:] = torch.nn.functional.pad(v, (0, n * 127 - v.numel())).view(n, 127)
    codes, scales = _check_codes(x.to(DEV), 1)
    assert bool((scales == 1).all())
    assert torch.equal(codes.float().signbit(), x.to(DEV).signbit())   # a negative zero among them


def test_quantize_scales_at_their_borders():
    """Maxima at, and one step past, 448 times a power of two; the smallest and largest floats; blocks of zeros."""
    tops = []
    for e in (-149, -140, -127, -126, -120, -60, -1, 0, 1, 60, 119, 120):
        for f in (448.0, 449.0, 447.0, 256.0, 1.0):
            t = torch.tensor(f * 2.0 ** e, dtype=torch.float64).float()
            if bool(t.isfinite()):
                tops += [t, torch.nextafter(t, torch.tensor(math.inf)), torch.nextafter(t, torch.tensor(0.0))]
    tops += [torch.tensor(v) for v in (0.0, -0.0, 3.4028234e38, 1e-45)]
    tops = torch.stack([t for t in tops if bool(t.isfinite())])
    x = torch.zeros((tops.numel(), 130))
    x[:, 7] = -tops
    x[:, 9] = tops * 0.37
    x[:, 129] = tops
    _check_codes(x.to(DEV), 1)
    assert bool((rpd.fp8_quantize(torch.zeros((2, 5), device=DEV))[1] == 1).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("per", [1, 128])
def test_quantize_what_is_not_finite(dtype, per):
    x = _x(140, 300, dtype, 4)
    x[3, 5], x[7, 260], x[9, 0] = math.nan, math.inf, -math.inf
    x[11, 128:256] = math.nan
    codes, _ = _check_codes(x, per)
    assert int(codes.float().isnan().sum()) == 3 + 128


def test_quantize_strided_rows_and_leading_dimensions():
    wide = _x(24, 300, BF, 5)
    for x in (wide[:, 3:204], wide[::3, 1:130], wide.view(2, 3, 4, 300)[..., :129], wide[:1, :5], wide[5]):
        a, s = rpd.fp8_quantize(x)
        b, t = rpd.fp8_quantize(x.contiguous())
        assert a.shape == x.shape and torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(s, t)
    assert rpd.fp8_quantize(wide[:0])[0].shape == (0, 300) and rpd.fp8_quantize(wide[:0])[1].shape == (0, 3)
    m = wide[:, 9:150]
    for a, b in zip(rpd.fp8_quantize(m, block_rows=128), rpd.fp8_quantize(m.contiguous(), block_rows=128)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("per", [1, 128])
def test_quantize_writes_its_rows_only(per):
    x = _x(37, 133, BF, 6)
    codes = torch.full((37, 160), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.empty((37 if per == 1 else 1, 2), device=DEV)
    assert rpd.lib().rpd_fp8_quantize(37, 133, rpd.DTYPE_BF16, x.data_ptr(), 133, per, codes.data_ptr() + 3, 160,
                                      scales.data_ptr(), None) == 0
    torch.cuda.synchronize()
    want, _ = rpd.fp8_quantize(x, block_rows=per)
    assert torch.equal(codes[:, 3:136], want.view(torch.uint8))
    assert bool((codes[:, :3] == 0x55).all()) and bool((codes[:, 136:] == 0x55).all())


# ------------------------------------------------------------------- head --

HEAD = [  # M, d, V, dtype
    (1, 256, 4096, BF), (1, 1, 1, BF), (2, 7, 17, HF), (15, 128, 15, F32), (16, 129, 16, BF), (17, 200, 63, HF),
    (31, 384, 64, BF), (33, 127, 65, F32), (48, 1000, 255, BF), (64, 512, 256, HF), (65, 256, 257, BF),
    (100, 300, 1000, F32), (130, 4096, 515, BF), (5, 4096, 2500, HF), (3, 10000, 300, BF), (256, 640, 130, BF),
    (80, 130, 4097, BF), (96, 2048, 777, HF),
]


def _values_of(x):
    return R.values(*R.quantize(x.reshape(-1, x.shape[-1]), 1), 1)


def _check(y, w, x):
    ref = R.product(w, x)
    tol = R.product_bound(w, x) + R.half_step(y.dtype) * ref.abs() * 1.01
    if y.dtype == HF:
        tol = tol + 2.0 ** -25   # half a subnormal step
    bad = (y.double() - ref).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float((y.double() - ref).abs().max()))


@pytest.mark.parametrize("M,d,V,dtype", HEAD)
def test_head_logits(M, d, V, dtype):
    note(f"  fp8 logits M={M} d={d} V={V} {dtype}")
    codes, scales = R.make_head(V, d, M + d, DEV)
    head = rpd.Fp8Head(codes, scales)
    x = _x(M, d, dtype, V)
    w, xq = R.values(codes.float(), scales, 128), _values_of(x)
    for out in (F32, BF, HF):
        _check(head.logits(x, out_dtype=out), w, xq)
    assert head.logits(x).dtype == dtype
    # bytes in place of the type
    again = rpd.Fp8Head(codes.view(torch.uint8), scales)
    assert torch.equal(again.logits(x), head.logits(x))


@pytest.mark.parametrize("M,d,V,dtype", HEAD)
def test_head_stats(M, d, V, dtype):
    note(f"  fp8 stats M={M} d={d} V={V} {dtype}")
    codes, scales = R.make_head(V, d, M + d, DEV)
    x = _x(M, d, dtype, V, level=0.7)
    scale = 1.0 if M % 2 else 0.5
    o = rpd.Fp8Head(codes, scales).stats(x, logit_scale=scale)
    w, xq = R.values(codes.float(), scales, 128), _values_of(x)
    y = R.product(w, xq) * scale
    delta = (R.product_bound(w, xq) * scale + R.U32 * y.abs()).amax(1)
    at, c, h = R.stats(y)
    got = o["argmax"].long()
    assert bool(((got >= 0) & (got < V)).all())
    chosen = y.gather(1, got.unsqueeze(1)).squeeze(1)
    assert bool((chosen >= y.amax(1) - 2 * delta).all())
    # a sum of positive terms, in chains of 16 entries, 2 + 2 merges of a tile, and of the tiles: at most 16 of a lane
    # and 6 merges (V <= 2^20); each merge, and the exponential, a few roundings
    chain = (16 + 4 * (4 + 16 + 6) + 8) * R.U32
    rel = torch.expm1(2 * delta) + 2 * chain
    assert bool(((o["confidence"].double() - c).abs() <= rel * c).all())
    assert bool(((o["entropy"].double() - h).abs() <= 2 * rel * (h + math.log(max(V, 2)) + 1)).all())


@pytest.mark.parametrize("M,d,V,dtype", HEAD)
def test_head_input_grad(M, d, V, dtype):
    note(f"  fp8 gradient M={M} d={d} V={V} {dtype}")
    codes, scales = R.make_head(V, d, M + d, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    g = _x(M, V, dtype, d)
    wt = R.values(codes.float(), scales, 128).t().contiguous()
    gq = _values_of(g)
    _check(head.input_grad(g, out_dtype=F32), wt, gq)
    _check(head.input_grad(g), wt, gq)


@pytest.mark.parametrize("V,M", [(131073 + 400, 64), (140000, 101), (135500, 49), (131100, 128), (70001, 256)])
def test_head_last_round_of_tiles(V, M):
    """Heads whose last tiles are cut into pieces of fewer rows."""
    note(f"  fp8 last round V={V} M={M}")
    d = 200
    codes, scales = R.make_head(V, d, M, DEV)
    head = rpd.Fp8Head(codes, scales)
    x = _x(M, d, BF, V)
    w, xq = R.values(codes.float(), scales, 128), _values_of(x)
    y = head.logits(x, out_dtype=F32)
    _check(y, w, xq)
    o = head.stats(x)
    assert torch.equal(o["argmax"].long(), y.argmax(1))
    _, c, h = R.stats(y.double())
    assert bool(((o["confidence"].double() - c).abs() <= 1e-4 * c).all())
    assert bool(((o["entropy"].double() - h).abs() <= 1e-4 * (h + 1)).all())


def test_head_gradient_of_long_rows():
    """The gradient's sum over a vocabulary is cut into parts, joined in order: twice the same."""
    codes, scales = R.make_head(20011, 333, 3, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    g = _x(70, 20011, BF, 4)
    a = head.input_grad(g, out_dtype=F32)
    _check(a, R.values(codes.float(), scales, 128).t().contiguous(), _values_of(g))
    for _ in range(3):
        assert torch.equal(a, head.input_grad(g, out_dtype=F32))


def test_head_gradient_by_autograd_and_by_differences():
    """Through ``logits`` by autograd, of rows with leading dimensions and of a broadcast upstream gradient; and by
    differences of rows of small integers, which 4 significant bits hold exactly."""
    codes, scales = R.make_head(77, 130, 5, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    g = torch.Generator().manual_seed(6)
    x = torch.randint(-7, 8, (2, 3, 130), generator=g).float().to(DEV)
    x[..., 0], x[..., 128] = 14.0, 14.0   # the blocks' scales stay what they are
    x.requires_grad_(True)
    y = head.logits(x)
    up = torch.randint(-3, 4, (77,), generator=g).float().to(DEV)
    grad, = torch.autograd.grad(y, x, up.expand(2, 3, 77))
    assert torch.equal(grad, head.input_grad(up.expand(2, 3, 77).contiguous()))
    w = R.values(codes.float(), scales, 128)
    bound = R.product_bound(w, _values_of(x.detach())).reshape(2, 3, 77)
    for k in (1, 64, 127, 129):
        near = [x.detach().clone() for _ in range(2)]
        near[0][..., k] += 1.0
        near[1][..., k] -= 1.0
        a, b = (head.logits(t) for t in near)
        diff = ((a - b).double() * up.double()).sum(-1) / 2.0
        tol = ((bound + R.product_bound(w, _values_of(near[0])).reshape(2, 3, 77)) * up.double().abs()).sum(-1)
        assert bool(((diff - grad[..., k].double()).abs() <= tol + 1e-9).all())
    # not recorded where no gradient is asked for; refused where there is no transposed head
    with torch.no_grad():
        assert not head.logits(x).requires_grad
    assert not head.logits(x.detach()).requires_grad
    with pytest.raises(ValueError):
        rpd.Fp8Head(codes, scales).logits(x)
    with pytest.raises(ValueError):
        head.logits(x, out=torch.empty((2, 3, 77), device=DEV))
    with pytest.raises(ValueError):
        rpd.Fp8Head(codes, scales).input_grad(y.detach())


def test_head_of_a_weight_matrix():
    """``from_weight``: quantized weights, and a head of few rows: the same numbers as by hand."""
    w = _x(300, 200, BF, 7, level=0.1)
    x = _x(4, 200, BF, 8)
    codes, scales = rpd.fp8_quantize(w, block_rows=128)
    a, b = rpd.Fp8Head.from_weight(w).logits(x), rpd.Fp8Head(codes, scales).logits(x)
    assert torch.equal(a, b)
    # every weight is off by half a step at most: 2^-4 of its size or 2^-10 of its scale
    near = R.values(codes.float(), scales, 128)
    s = scales.double().repeat_interleave(128, 0)[:300].repeat_interleave(128, 1)[:, :200]
    assert bool(((near - w.double()).abs() <= torch.maximum(w.double().abs() * 2.0 ** -4, s * 2.0 ** -10)).all())


def test_head_equal_rows_take_the_lowest_index():
    codes, scales = R.make_head(1280, 640, 9, DEV)
    scales[:] = scales[:1]   # rows of any block are then equal where their codes are
    x = _x(40, 640, BF, 10)
    best = rpd.Fp8Head(codes, scales).stats(x)["argmax"].long()
    more = torch.cat([codes[best].view(torch.uint8), codes.view(torch.uint8), codes[best].view(torch.uint8)])
    wide = scales[:1].expand(-(-more.shape[0] // 128), -1).contiguous()
    got = rpd.Fp8Head(more, wide).stats(x)["argmax"].long()
    y = R.product(R.values(more.view(E4).float(), wide, 128), _values_of(x))
    assert torch.equal(got, (y == y.amax(1, keepdim=True)).int().argmax(1))


def test_head_rows_keep_to_themselves():
    """NaN, infinities, zeros and rows of other sizes beside ordinary ones; rows of unaligned stride; broken rows of
    the head."""
    codes, scales = R.make_head(300, 264, 11, DEV)
    head = rpd.Fp8Head(codes, scales)
    wide = _x(37, 271, BF, 12)
    x = wide[:, 3:267]
    plain = head.logits(x, out_dtype=F32)
    _check(plain, R.values(codes.float(), scales, 128), _values_of(x))
    x[2, 5], x[4, 263], x[20, 130] = math.nan, math.inf, -math.inf
    x[6] *= 2.0 ** 90
    x[7] *= 2.0 ** -90
    x[8] = 0.0
    y = head.logits(x, out_dtype=F32)
    assert bool(y[[2, 4, 20]].isnan().all()) and not bool(y[8].any())
    rest = [m for m in range(37) if m not in (2, 4, 6, 7, 8, 20)]
    assert torch.equal(y[rest], plain[rest])
    assert torch.equal(y[6], plain[6] * 2.0 ** 90) and torch.equal(y[7], plain[7] * 2.0 ** -90)
    o = head.stats(x)
    assert o["argmax"][[2, 4, 20]].tolist() == [-1] * 3 and bool(o["entropy"][[2, 4, 20]].isnan().all())
    assert int(o["argmax"][8]) == 0 and abs(float(o["entropy"][8]) - math.log(300)) < 1e-5
    bytes_ = codes.view(torch.uint8).clone()
    bytes_[17, 100] = 0x7f   # NaN
    y = rpd.Fp8Head(bytes_, scales).logits(wide[10:12, 3:267], out_dtype=F32)
    assert bool(y[:, 17].isnan().all()) and int(y.isnan().sum()) == 2
    assert torch.equal(y[:, 18:], plain[10:12, 18:])


def test_head_out_of_wider_rows_and_nothing_beside_them():
    codes, scales = R.make_head(301, 140, 13, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    x = _x(19, 140, BF, 14)
    for dtype in DTYPES:
        wide = torch.full((19, 333), 7.0, dtype=dtype, device=DEV)
        got = head.logits(x, out=wide[:, 5:306])
        assert got.data_ptr() == wide[:, 5:].data_ptr() and torch.equal(got, head.logits(x, out_dtype=dtype))
        assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 306:] == 7).all())
        wide = torch.full((19, 150), 7.0, dtype=dtype, device=DEV)
        g = head.logits(x)
        got = head.input_grad(g, out=wide[:, 3:143])
        assert torch.equal(got, head.input_grad(g, out_dtype=dtype))
        assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 143:] == 7).all())


def test_head_no_rows_and_shapes():
    codes, scales = R.make_head(100, 64, 15, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    x = torch.empty((2, 0, 64), dtype=HF, device=DEV)
    assert head.logits(x).shape == (2, 0, 100) and head.input_grad(head.logits(x)).shape == (2, 0, 64)
    assert all(v.shape == (2, 0) for v in head.stats(x).values())
    one = _x(1, 64, HF, 16)[0]
    assert torch.equal(head.logits(one), head.logits(one[None])[0])
    for bad in (torch.empty((3, 63), dtype=HF, device=DEV), torch.empty((3, 64), dtype=torch.float64, device=DEV),
                torch.empty((3, 64), dtype=HF), torch.empty((3, 128), dtype=HF, device=DEV)[:, ::2]):
        with pytest.raises((ValueError, TypeError)):
            head.logits(bad)


def test_head_rows_further_apart_than_32_bits():
    """Rows of x, and of the logits, more than 2^32 bytes apart; a head of more than 2^31 bytes."""
    codes, scales = R.make_head(70, 200, 17, DEV)
    head = rpd.Fp8Head(codes, scales)
    x = _x(2, 200, BF, 18)
    store = torch.empty((1 << 31) + 4096, dtype=BF, device=DEV)
    far = store.as_strided((2, 200), (1 << 31, 1))
    far.copy_(x)
    out = store[1024:].as_strided((2, 70), (1 << 31, 1))
    want = head.logits(x)
    assert torch.equal(head.logits(far, out=out), want)
    a, b = rpd.fp8_quantize(far), rpd.fp8_quantize(x)
    assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1])
    del store, far, out, a, b
    V, d = 600000, 4096
    codes = torch.randint(0, 0x78, (V, 1), dtype=torch.uint8, device=DEV).expand(V, d).contiguous()
    codes[-300:] = torch.randint(0, 0x78, (300, d), dtype=torch.uint8, device=DEV)
    scales = torch.full((-(-V // 128), d // 128), 2.0 ** -10, device=DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    x = _x(3, d, BF, 19)
    y = head.logits(x, out_dtype=F32)
    for part in (slice(0, 300), slice(524200, 524400), slice(V - 300, V)):
        _check(y[:, part], R.values(codes[part].view(E4).float(), scales[:3], 128), _values_of(x))
    g = torch.zeros((2, V), dtype=BF, device=DEV)
    g[0, 5], g[0, V - 7], g[1, 524288] = 1.0, -2.0, 3.0
    got = head.input_grad(g, out_dtype=F32)
    rows = codes.view(E4)[[5, V - 7, 524288]].float() * 2.0 ** -10
    assert torch.equal(got, torch.stack([rows[0] - 2.0 * rows[1], 3.0 * rows[2]]))


def test_head_on_a_stream_and_in_graphs():
    """Replays with new rows equal the eager calls, which run between them."""
    codes, scales = R.make_head(5000, 384, 20, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    x, g = _x(20, 384, BF, 21), _x(20, 5000, BF, 22)

    def work(**kw):
        q = rpd.fp8_quantize(x, **kw)
        return [head.logits(x, **kw), *head.stats(x, **kw).values(), head.input_grad(g, **kw), q[0].view(torch.uint8), q[1]]

    want = work()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = work(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for seed in range(4):
        x.copy_(_x(20, 384, BF, 30 + seed))
        g.copy_(_x(20, 5000, BF, 40 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(got, work()))


def test_head_forward_and_backward_in_a_graph():
    codes, scales = R.make_head(900, 256, 23, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    x = torch.zeros((9, 256), dtype=BF, device=DEV, requires_grad=True)
    up = _x(9, 900, BF, 24)

    def step():
        y = head.logits(x)
        return y.detach(), torch.autograd.grad(y, x, up)[0]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # what the first backward pass sets up is not captured
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(4):
        with torch.no_grad():
            x.copy_(_x(9, 256, BF, 50 + seed))
        up.copy_(_x(9, 900, BF, 60 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert torch.equal(got[0], head.logits(x.detach())) and torch.equal(got[1], head.input_grad(up))


def test_head_statistics_for_the_gate():
    """[K][B][L][d] rows: what ``gate_commit`` makes of them equals what it makes of the logits' own statistics."""
    K, B, L, d, V = 3, 2, 16, 256, 700
    codes, scales = R.make_head(V, d, 25, DEV)
    head = rpd.Fp8Head(codes, scales)
    x = _x(K * B * L, d, BF, 26).view(K, B, L, d)
    mask = torch.ones((B, L), dtype=torch.uint8, device=DEV)
    s = head.stats(x)
    o = rpd.gate_commit(mask, s["argmax"], s["confidence"], s["entropy"], rpd.Params(theta_h=0.05, theta_c=0.01, theta_s=1.0))
    _, c, _ = R.stats(head.logits(x[-1].reshape(B * L, d), out_dtype=F32).double())
    torch.cuda.synchronize()
    assert int(o["n_commit"].min()) >= 1
    c = c.view(B, L)
    assert bool(((o["confidence"].double() - c).abs() <= 1e-4 * c).all())


def test_two_streams_at_once_over_one_head():
    codes, scales = R.make_head(30011, 512, 27, DEV)
    head = rpd.Fp8Head(codes, scales, train=True)
    xs, gs = [_x(24 + 30 * i, 512, BF, 28 + i) for i in range(2)], [_x(24, 30011, BF, 30 + i) for i in range(2)]
    work = lambda i: [head.logits(xs[i]), *head.stats(xs[i]).values(), head.input_grad(gs[i])]   # noqa: E731
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


def test_head_more_than_2_to_the_34_logits():
    """Logits and statistics of many rows are those of the same rows in small calls."""
    d, V, M = 128, 126464, 136000
    codes, scales = R.make_head(V, d, 41, DEV)
    head = rpd.Fp8Head(codes, scales)
    x = _x(M, d, BF, 42)
    o, y = head.stats(x), head.logits(x)
    assert y.numel() > 1 << 34
    w = R.values(codes.float(), scales, 128)
    for at in (0, 68013, M - 130):
        part = slice(at, at + 130)
        small = head.stats(x[part])
        assert all(torch.equal(o[k][part], small[k]) for k in o)
        assert torch.equal(y[part], head.logits(x[part]))
        _check(y[part][-5:], w, _values_of(x[part][-5:]))
    del y
    torch.cuda.empty_cache()   # 34 GB
