"""4-bit blocks and their product on the GPU against float64 (fp4_ref), at the sizes,
strides, types and values where they can go wrong."""
import math

import pytest
import torch

import fp4_ref as F
from gpu_common import device

pytestmark = pytest.mark.gpu

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.fixture(scope="module")
def R():
    from paper_2609_34608_amd import runtime
    return runtime


def _rand(dev, seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn(*shape, generator=g)).to(dev)


def _rows(x, pad, offset=0, fill=0xA5):
    """x [M, n] bytes with rows `pad` further apart, starting `offset` bytes into a buffer of
    `fill`; the view and the buffer."""
    M, n = x.shape
    buf = torch.full((offset + M * (n + pad),), fill, dtype=U8, device=x.device)
    view = buf[offset:].view(M, n + pad)[:, :n]
    view.copy_(x)
    return view, buf


# ------------------------------------------------------------- blocks
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 32), (3, 31), (5, 33), (2, 64), (7, 71), (64, 256), (33, 1216), (1, 6144),
                                 (130, 1211)])
def test_quantize_and_back(dev, R, M, K, dtype):
    x = (_rand(dev, 1, M, K) * torch.exp2(_rand(dev, 2, M, K) * 3)).to(dtype)
    q, s = R.quantize_fp4(x)
    wq, ws = F.quantize(x)
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
    assert q.stride(0) % 16 == 0 or M == 1
    for kind in (F32, BF16):
        F.same(R.dequantize_fp4(q, s, columns=K, dtype=kind), F.values(wq, ws)[:, :K])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_border(dev, R, dtype):
    """Values on the borders between two codes, one step beside them, and above the largest,
    at scales from the smallest to the largest."""
    mags = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0], dtype=F.F64)
    rows = []
    for e in (-127, -126, -125, -100, -10, 0, 3, 100, 124, 125):
        s = 2.0 ** e
        eps = torch.finfo(dtype).eps
        for shift in (0.0, eps, -eps):
            v = (mags * (1 + shift)).clamp_max(7.0) * s
            rows.append(torch.cat([v[:15], -v[:15], torch.tensor([4.0 * s, -7.0 * s if e < 125 else -4.0 * s])]))
    x = torch.stack(rows).to(F32).to(dtype).to(dev)
    q, s = R.quantize_fp4(x)
    wq, ws = F.quantize(x)
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
    F.same(R.dequantize_fp4(q, s, dtype=F32), F.values(wq, ws))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_blocks_of_zero_subnormal_and_non_finite_values(dev, R, dtype):
    x = _rand(dev, 1, 6, 96)
    x[0] = 0.0
    x[1, :32] = 1e-42 if dtype == F32 else 9.2e-41  # subnormal: the smallest scale
    x[2, 40], x[3, 1], x[3, 95] = math.nan, math.inf, -math.inf
    x[4, 7], x[5] = 3e38, -0.0
    x = x.to(dtype)
    q, s = R.quantize_fp4(x)
    wq, ws = F.quantize(x)
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
    assert s[2].tolist()[1] == 255 and s[3].tolist()[::2] == [255, 255] and s[0].tolist() == [0, 0, 0]
    F.same(R.dequantize_fp4(q, s, dtype=F32), F.values(wq, ws))


def test_every_code_and_scale(dev, R):
    """All 16 codes at all 256 scale bytes; past the range of the result infinite."""
    codes = torch.arange(16, dtype=torch.int32)
    q = (codes | (15 - codes) << 4).to(U8).expand(256, 16).contiguous().to(dev)
    s = torch.arange(256, dtype=torch.int32).to(U8).view(256, 1).to(dev)
    want = F.values(q, s)
    for kind in (F32, BF16):
        F.same(R.dequantize_fp4(q, s, dtype=kind), want.to(kind))


@pytest.mark.parametrize("K", [33, 64, 95])
def test_block_strides(dev, R, K):
    """Inputs and results off any alignment; no byte between the rows is written."""
    x = _rand(dev, 3, 9, K + 3)[:, 1:K + 1]
    wq, ws = F.quantize(x)
    (q, qb), (s, sb) = _rows(torch.zeros(9, -(-K // 2), dtype=U8, device=dev), 5, 3), \
        _rows(torch.zeros(9, -(-K // 32), dtype=U8, device=dev), 2, 1)
    R.quantize_fp4(x, q=q, scale=s)
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
    for view, buf in ((q, qb), (s, sb)):
        again = torch.full_like(buf, 0xA5)
        again[-view.shape[0] * view.stride(0):].view(9, -1)[:, :view.shape[1]] = view
        assert torch.equal(buf, again)
    out = torch.full((9, K + 4), 7.0, device=dev)
    R.dequantize_fp4(q, s, columns=K, out=out[:, 1:K + 1])
    F.same(out[:, 1:K + 1], F.values(wq, ws)[:, :K])
    assert (out[:, 0] == 7).all() and (out[:, K + 1:] == 7).all()
    shared = _rand(dev, 4, 1, 64).expand(5, 64)
    assert torch.equal(R.quantize_fp4(shared)[0].cpu(), F.quantize(shared)[0])


def test_block_offsets_past_32_bits(dev, R):
    buf = torch.zeros((1 << 31) + 4096, dtype=U8, device=dev)
    far = buf.as_strided((2, 64), ((1 << 31) + 256, 1))
    x = _rand(dev, 1, 2, 128).to(BF16)
    _, s = R.quantize_fp4(x, q=far)
    wq, ws = F.quantize(x)
    assert torch.equal(far.cpu(), wq)
    wide = buf.view(BF16).as_strided((2, 128), ((1 << 30) + 256, 1))
    wide.copy_(x)
    q, s = R.quantize_fp4(wide)
    assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
    R.dequantize_fp4(q, s, out=wide)
    F.same(wide, F.values(wq, ws))


# ------------------------------------------------------------- product
# (M, N, K) that reach every tile of the planner, with remainders; test_plan_fp4 asks for that
TILES = [
    (1, 64, 64), (1, 4608, 1536), (3, 40, 30), (16, 33, 258), (17, 200, 512), (31, 65, 994),
    (64, 256, 256), (70, 130, 770), (137, 512, 512), (200, 648, 320), (333, 1000, 1218), (514, 1031, 600),
    (864, 768, 768), (1030, 1550, 514), (900, 2310, 768), (2100, 1600, 130), (2754, 1216, 1216),
    (2536, 387, 770), (8336, 451, 130), (7223, 1027, 130), (8205, 1292, 130), (3900, 2100, 1026), (7223, 1027, 770),
    (8205, 1292, 770), (10170, 1530, 1026), (2712, 1106, 130),
]


BLOCK_TILES = [t for t in TILES if t[2] <= 1218]  # of 4-bit results


def _operands(R, dev, M, N, K, seed=1):
    a, w = _rand(dev, seed, M, K), _rand(dev, seed + 1, N, K, std=0.02)
    return (*R.quantize_fp4(a), *R.quantize_fp4(w))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", TILES)
def test_matmul(dev, R, M, N, K, dtype):
    ops = _operands(R, dev, M, N, K)
    bias = _rand(dev, 5, N, std=0.02)
    F.check(R.matmul_fp4(*ops, bias=bias, out_dtype=dtype), *F.matmul(*ops, bias), dtype)
    F.check(R.matmul_fp4(*ops, gelu=True, out_dtype=dtype), *F.matmul(*ops, act=True), dtype)


@pytest.mark.parametrize("M,N,K", BLOCK_TILES)
def test_matmul_into_blocks(dev, R, M, N, K):
    """The codes are those of the float32 result, which the same tiles give."""
    ops = _operands(R, dev, M, N, K, seed=3)
    for gelu in (False, True):
        q, s = R.matmul_fp4(*ops, gelu=gelu, out_dtype=U8)
        c, err = F.matmul(*ops, act=gelu)
        got = F.values(q, s)[:, :N]
        # a code is off by at most half a step, 1/4 of the value or of the scale; where the sum's error
        # moves a value over a border, or a block's maximum over a power of two, twice that
        step = torch.exp2(s.cpu().to(F.F64) - 127).repeat_interleave(32, 1)[:, :N]
        assert ((got - c).abs() <= torch.maximum(torch.maximum(0.25 * step, 0.25 * c.abs()), c.abs() - 6 * step) + err).all()
        if N % 2:
            assert (q[:, -1] >> 4 == 0).all()


def test_matmul_far_scales(dev, R):
    """Blocks whose scales lie far apart: the bound counts by magnitude, no range is lost.
    What is compared are sums whose magnitudes stay in the float32 range: of scales up to
    2^198 the first step's part alone can be 1.5e48 (row 2, column 31 of the last spread) and
    cancel exactly in float64, where any float32 sum is infinite."""
    g = torch.Generator().manual_seed(2)
    for spread in (8, 60, 200):
        a, w = (torch.randint(0, 256, (n, 256), generator=g, dtype=torch.int32).to(U8).to(dev) for n in (40, 72))
        sa, sw = (torch.randint(127 - spread // 2, 127 + spread // 2, (n, 16), generator=g, dtype=torch.int32).to(U8)
                  .to(dev) for n in (40, 72))
        c, err = F.matmul(a, sa, w, sw)
        fits = F.values(a, sa).abs() @ F.values(w, sw).abs().t() < 2.0 ** 127
        assert fits.float().mean() > 0.2
        got = R.matmul_fp4(a, sa, w, sw, out_dtype=F32).cpu().to(F.F64)
        assert ((got - c).abs() <= err + 2.0 ** -24 * c.abs() + 2.0 ** -126)[fits].all()


def test_matmul_strides_and_tail_bytes(dev, R):
    """Rows further apart, NaN scales and codes in the bytes past a row's end, results off
    their words; nothing is written beside a row."""
    M, N, K = 37, 83, 70
    ops = _operands(R, dev, M, N, K)
    want = R.matmul_fp4(*ops, out_dtype=F32)
    a, w = (_rows(t, 16 - 35 % 16 + 32, 16, 0xFF)[0] for t in (ops[0], ops[2]))
    sa, sw = (_rows(t, 1 + 4, 4, 0xFF)[0] for t in (ops[1], ops[3]))
    out = torch.full((M, N + 5), 7.0, device=dev)
    assert torch.equal(R.matmul_fp4(a, sa, w, sw, out=out[:, 2:N + 2]), want)
    assert (out[:, :2] == 7).all() and (out[:, N + 2:] == 7).all()
    for ld, off in ((N + 1, 0), (N + 2, 1), (N + 5, 0)):
        half = torch.full((M * ld + 8,), 7.0, dtype=BF16, device=dev)
        view = half[off:off + M * ld].view(M, ld)[:, :N]
        R.matmul_fp4(a, sa, w, sw, out=view)
        F.check(view, *F.matmul(*ops), BF16)
        rest = half.clone()
        rest[off:off + M * ld].view(M, ld)[:, :N] = 7
        assert (rest == 7).all()


def test_matmul_non_finite_rows(dev, R):
    """A NaN block spoils its own row or column and no other."""
    ops = _operands(R, dev, 70, 90, 320)
    ops[1][33, 4], ops[3][17, 0] = 255, 255
    for dtype in (F32, BF16):
        got = R.matmul_fp4(*ops, out_dtype=dtype).isnan()
        want = torch.zeros_like(got)
        want[33], want[:, 17] = True, True
        assert torch.equal(got, want)


def test_matmul_rows_far_apart(dev, R):
    """Rows past 32-bit offsets inside a tile."""
    far = (1 << 23) + 4096
    buf = torch.full((70 * far,), 0xFF, dtype=U8, device=dev)
    a, sa, w, sw = _operands(R, dev, 70, 65, 300)
    view = buf.as_strided((70, 150), (far, 1))
    view.copy_(a)
    for dtype in (F32, BF16):
        F.check(R.matmul_fp4(view, sa, w, sw, out_dtype=dtype), *F.matmul(a, sa, w, sw), dtype)
    q, s = R.matmul_fp4(view, sa, w, sw, out_dtype=U8)
    c, err = F.matmul(a, sa, w, sw)
    step = torch.exp2(s.cpu().to(F.F64) - 127).repeat_interleave(32, 1)[:, :65]
    near = torch.maximum(torch.maximum(0.25 * step, 0.25 * c.abs()), c.abs() - 6 * step) + err
    assert ((F.values(q, s)[:, :65] - c).abs() <= near).all()


def test_mlp_in_blocks(dev, R):
    """Up projection with GELU into blocks, down projection of them."""
    M, D, H = 75, 256, 1000
    x, sx = R.quantize_fp4(_rand(dev, 1, M, D))
    w1, s1 = R.quantize_fp4(_rand(dev, 2, H, D, std=0.1))
    w2, s2 = R.quantize_fp4(_rand(dev, 3, D, H, std=0.1))
    u, su = R.matmul_fp4(x, sx, w1, s1, gelu=True, out_dtype=U8)
    assert u.shape == (M, H // 2) and su.shape == (M, 32)
    F.check(R.matmul_fp4(u, su, w2, s2), *F.matmul(u, su, w2, s2), BF16)


def test_empty_shapes(dev, R):
    q, s = R.quantize_fp4(torch.empty(0, 64, device=dev))
    assert q.shape == (0, 32) and s.shape == (0, 2) and R.dequantize_fp4(q, s).shape == (0, 64)
    q, s = R.quantize_fp4(torch.empty(3, 0, device=dev))
    assert q.shape == (3, 0) and s.shape == (3, 0)
    a, sa, w, sw = _operands(R, dev, 4, 64, 128)
    assert R.matmul_fp4(a[:0], sa[:0], w, sw).shape == (0, 64)
    assert R.matmul_fp4(a, sa, w[:0], sw[:0]).shape == (4, 0)


def test_binding_refusals(dev, R):
    x = _rand(dev, 1, 8, 128)
    for bad in (dict(x=x[0]), dict(x=x.half()), dict(x=x.cpu()), dict(x=x.t()), dict(q=torch.empty(8, 63, dtype=U8, device=dev)),
                dict(scale=torch.empty(8, 4, device=dev)), dict(x=x.clone().requires_grad_())):
        kw = dict(x=x)
        kw.update(bad)
        with pytest.raises(R.WamError):
            R.quantize_fp4(kw.pop("x"), **kw)
    q, s = R.quantize_fp4(x)
    for bad in (dict(columns=126), dict(columns=129), dict(dtype=torch.float16), dict(scale=s[:, :3]), dict(q=q.int()),
                dict(out=torch.empty(8, 127, device=dev))):
        kw = dict(q=q, scale=s)
        kw.update(bad)
        with pytest.raises(R.WamError):
            R.dequantize_fp4(kw.pop("q"), kw.pop("scale"), **kw)
    a, sa, w, sw = _operands(R, dev, 8, 64, 256)
    for bad in (dict(w=w[:, :64]), dict(a_scale=sa[:, :7]), dict(w_scale=sw.int()), dict(bias=torch.ones(65, device=dev)),
                dict(out_dtype=torch.float16), dict(out_dtype=torch.int32), dict(a=a[:, 1:], w=w[:, 1:]), dict(a=a.float()),
                dict(out=torch.empty(8, 64, dtype=torch.float16, device=dev)), dict(a=a[0])):
        kw = dict(a=a, a_scale=sa, w=w, w_scale=sw)
        kw.update(bad)
        with pytest.raises(R.WamError):
            R.matmul_fp4(kw.pop("a"), kw.pop("a_scale"), kw.pop("w"), kw.pop("w_scale"), **kw)
