"""Edges of the layer operators on the GPU: values past the rotated pairs, blocks and
scales at the ends of the float32 range, rows further apart than 32-bit offsets, and
tensors that a gradient is asked of."""
import numpy as np
import pytest
import torch

import layer_ops_ref as F
from gpu_common import device

pytestmark = pytest.mark.gpu

BF16, F32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


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


def _bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == F32 else torch.int16)


# ------------------------------------------------------------- rotary positions
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dh,sec", [(64, (16, 0, 0)), (64, (0, 0, 0)), (96, (8, 8, 8)), (160, (16, 8, 0)), (64, (5, 6, 7))])
def test_rope_passes_what_it_does_not_turn(dev, R, dh, sec, dtype, layout):
    """NaN, infinities and -0 past the pairs: those elements come out as they are, and
    no other element knows of them."""
    P = sum(sec)
    pos = torch.arange(27, device=dev, dtype=F32).view(9, 3)
    freq = R.rope_frequencies(sec)
    q, k = _rand(dev, 1, 2, 9, 3, dh).to(dtype), _rand(dev, 2, 2, 9, 2, dh).to(dtype)
    want = R.rope(q, k, pos, sec, freq, layout=layout)
    special = (float("nan"), float("inf"), -float("inf"), -0.0)
    for x, w, name in ((q, want[0], "q"), (k, want[1], "k")):
        for at, v in enumerate(special):
            for e in (2 * P, 2 * P + 1 + at, dh - 8, dh - 1):
                z = x.clone()
                z[0, 3, 1, e] = v
                z[1, 8, 0, e] = v
                z[1, 2, 1, 2 * P:] = -0.0
                got = R.rope(*((z, k) if name == "q" else (q, z)), pos, sec, freq, layout=layout)[name == "k"]
                expect = w.clone()
                expect[..., 2 * P:] = z[..., 2 * P:]
                if v != v:
                    assert got[0, 3, 1, e].isnan() and got[1, 8, 0, e].isnan()
                    for t in (got, expect):
                        t[0, 3, 1, e] = t[1, 8, 0, e] = 0.0
                assert torch.equal(_bits(got), _bits(expect))


def test_rope_refuses_a_table_of_frequencies(dev, R):
    """One frequency per pair: a table of as many rows is none."""
    q, pos = _rand(dev, 1, 1, 4, 2, 64), torch.zeros(4, 3, device=dev)
    with pytest.raises(R.WamError, match="frequency"):
        R.rope(q, None, pos, (8, 12, 12), np.ones((32, 2)))


# ------------------------------------------------------------- gradients
def test_gradients_are_refused(dev, R):
    """Nothing here has a backward pass: a tensor that asks for a gradient is refused
    where torch would record one, as an input and as a result's buffer."""
    q, pos, sec, freq = _rand(dev, 1, 1, 4, 2, 64), torch.zeros(4, 3, device=dev), (8, 12, 12), R.rope_frequencies((8, 12, 12))
    h, gain = _rand(dev, 2, 1, 4, 64), torch.ones(64, device=dev)
    a, sa = R.quantize_fp8(h[0])
    w, sw = R.quantize_fp8(_rand(dev, 3, 32, 64), block_rows=128)
    need = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    calls = [lambda: R.rope(need(q), None, pos, sec, freq), lambda: R.rope(q, need(q), pos, sec, freq),
             lambda: R.rope(q, None, need(pos), sec, freq), lambda: R.rope(q, None, pos, sec, freq, q_gain=need(gain)),
             lambda: R.rope(q, None, pos, sec, freq, q_out=need(q)), lambda: R.norm_residual(need(h)),
             lambda: R.norm_residual(h, need(h)), lambda: R.norm_residual(h, scale=need(gain)),
             lambda: R.norm_residual(h, h_out=need(h)), lambda: R.norm_residual(h, post_gain=need(gain)),
             lambda: R.quantize_fp8(need(h[0])), lambda: R.matmul_fp8(a, need(sa), w, sw),
             lambda: R.matmul_fp8(a, sa, w, sw, bias=need(gain[:32])),
             lambda: R.matmul_fp8(a, sa, w, sw, out=need(torch.zeros(4, 32, device=dev)))]
    for call in calls:
        with pytest.raises(R.WamError, match="gradient"):
            call()
        with torch.no_grad():
            call()


# ------------------------------------------------------------- ends of the float32 range
def _blocks32(x, rows):
    """Bytes and scales of x (float32, on the host) by the definition, a division in
    float32 and one rounding."""
    M, K = x.shape
    q, s = torch.empty(M, K, dtype=torch.uint8), torch.empty(-(-M // rows), -(-K // 128))
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = (slice(i * rows, (i + 1) * rows), slice(j * 128, (j + 1) * 128))
            top = x[at].abs().max()
            s[i, j] = torch.where(top == 0, torch.ones(()), (top / torch.tensor(448.0)).clamp_min(2.0 ** -126))
            q[at] = (x[at] / s[i, j]).to(FP8).view(torch.uint8)
    return q, s


@pytest.mark.parametrize("rows", [1, 128])
def test_blocks_of_the_smallest_scales(dev, R, rows):
    """Blocks down to the smallest scale, their values on the borders between two e4m3
    values or beside one: the bytes of the float32 quotient."""
    rng = np.random.default_rng(7)
    M, K = 256, 384
    scale = np.float32(2.0) ** rng.integers(-126, -112, (M // rows, 3)) * rng.uniform(1, 2, (M // rows, 3)).astype(np.float32)
    scale = np.repeat(np.repeat(scale.astype(np.float32), rows, 0), 128, 1)
    odd = 2.0 * rng.integers(8, 16, (M, K)) + 1.0
    v = np.where(rng.random((M, K)) < 0.3, (2 * rng.integers(0, 8, (M, K)) + 1) * 2.0 ** -10,
                 odd / 16 * 2.0 ** rng.integers(-6, 8, (M, K)))
    v[:, ::128] = 448.0
    x = torch.from_numpy((v * scale.astype(np.float64)).astype(np.float32))
    want = _blocks32(x, rows)
    q, s = R.quantize_fp8(x.to(dev), block_rows=rows)
    assert torch.equal(s.cpu(), want[1])
    assert torch.equal(q.contiguous().view(torch.uint8).cpu(), want[0])
    if rows == 1:  # the same values as a norm's result
        _, q, s = R.norm_residual(x.to(dev)[None], pre="none", u_dtype=FP8)
        assert torch.equal(s[0].cpu(), want[1])
        assert torch.equal(q[0].contiguous().view(torch.uint8).cpu(), want[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N", [(1, 64), (40, 200), (700, 1000)])
@pytest.mark.parametrize("ea,ew", [(-62, -62), (-114, -10), (63, 62), (14, 111)])
def test_products_of_far_scales(dev, R, ea, ew, M, N, dtype):
    """Scales whose product is at either end of the normal float32 range: no digit is
    lost, and a zero block stays zero."""
    K = 384
    kb = 3
    a, w = _rand(dev, 1, M, K), _rand(dev, 2, N, K)
    if ea < 0:  # values that bring the result back into the range: sums of large ones, or small ones
        a, w = ((100.0 * t).abs().clamp_max(448.0) for t in (a, w))
    else:
        a, w = a * 2.0 ** -7, w * 2.0 ** -7
    a, w = a.to(FP8), w.to(FP8)
    sa = 2.0 ** ea * (1 + torch.rand(M, kb, generator=torch.Generator().manual_seed(3))).to(dev)
    sw = 2.0 ** ew * (1 + torch.rand(-(-N // 128), kb, generator=torch.Generator().manual_seed(4))).to(dev)
    near = torch.arange(M, device=dev) % 3 == 1  # rows of ordinary products between the others
    sa[near] = sa[near] * 2.0 ** -ea * 2.0 ** -ew
    a.view(torch.uint8)[M // 2, 128:256] = 0
    c, err = F.matmul(a, sa, w, sw, None, False, dtype)
    out = F.f64(R.matmul_fp8(a, sa, w, sw, out_dtype=dtype))
    assert c.abs().max() < 2.0 ** 127 and out.isfinite().all()
    # below the normal range a rounding is off by 2^-150, three a block
    tol = err * (1 + 2.0 ** -8) + F.HALF[dtype] * (c.abs() + err) + (3 * kb + 1) * 2.0 ** -150
    assert ((out - c).abs() <= tol).all(), float(((out - c).abs() / tol).max())


# ------------------------------------------------------------- rows far apart
@pytest.mark.parametrize("K", [256, 333])
@pytest.mark.parametrize("far", ["a", "w"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matmul_rows_far_apart(dev, R, dtype, far, K):
    """Rows past the 32-bit offsets of a tile (2^23 bytes apart): the same bits as rows
    side by side, where the near ones take the same tile, and the bound either way."""
    M, N = 70, 90
    a, sa = R.quantize_fp8(_rand(dev, 1, M, K))
    w, sw = R.quantize_fp8(_rand(dev, 2, N, K), block_rows=128)
    bias = _rand(dev, 3, N)
    step = (1 << 23) + 16
    x = a if far == "a" else w
    buf = torch.empty((x.shape[0] - 1) * step + 352, dtype=torch.uint8, device=dev)
    view = buf.as_strided((x.shape[0], 352), (step, 1))
    view.fill_(127)  # NaN behind the rows
    view[:, :K] = x.view(torch.uint8)
    there = view.view(FP8)[:, :K]
    ops = (there, sa, w, sw) if far == "a" else (a, sa, there, sw)
    for gelu in (False, True):
        out = R.matmul_fp8(*ops, bias=bias, gelu=gelu, out_dtype=dtype)
        F.check(out, *F.matmul(a, sa, w, sw, bias, gelu, dtype), dtype=dtype)
        assert torch.equal(out, R.matmul_fp8(a, sa, w, sw, bias=bias, gelu=gelu, out_dtype=dtype))


def test_matmul_last_row_ends_inside_a_chunk(dev, R):
    """One contiguous row of K off 16: what lies behind it does not enter."""
    K, N = 333, 40
    w, sw = R.quantize_fp8(_rand(dev, 2, N, K), block_rows=128)
    a, sa = R.quantize_fp8(_rand(dev, 1, 1, K))
    want = R.matmul_fp8(a, sa, w, sw, out_dtype=F32)
    buf = torch.full((400,), 127, dtype=torch.uint8, device=dev)
    buf[:K] = a.view(torch.uint8)[0]
    assert torch.equal(R.matmul_fp8(buf.view(FP8)[:K].view(1, K), sa, w, sw, out_dtype=F32), want)
