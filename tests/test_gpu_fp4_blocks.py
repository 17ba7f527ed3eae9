"""Products into 4-bit blocks: every code and scale byte is that of the float32 result."""
import math

import pytest
import torch

import fp4_ref as F
from gpu_common import device
from test_gpu_fp4 import BLOCK_TILES, F32, U8, _operands, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.fixture(scope="module")
def R():
    from paper_2609_34608_amd import runtime
    return runtime


def _blocks_of(R, ops, **kw):
    """4-bit result, checked byte for byte against blocks of the float32 one: every tile takes
    a sum's terms in the same order, so both round the same numbers."""
    q, s = R.matmul_fp4(*ops, out_dtype=U8, **kw)
    c = R.matmul_fp4(*ops, out_dtype=F32, **kw)
    wq, ws = F.quantize(c)
    assert torch.equal(s.cpu(), ws)
    assert torch.equal(q.cpu(), wq)
    return q, s, c


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", BLOCK_TILES)
def test_product_into_blocks(dev, R, M, N, K, gelu):
    ops = _operands(R, dev, M, N, K, seed=3)
    _blocks_of(R, ops, gelu=gelu)
    _blocks_of(R, ops, gelu=gelu, bias=_rand(dev, 5, N, std=0.5))


@pytest.mark.parametrize("M,N,K", [(3, 40, 30), (70, 130, 770), (514, 1031, 600), (2754, 1216, 1216)])
def test_non_finite_blocks(dev, R, M, N, K):
    """A NaN row spoils its blocks, a NaN column the one block of each row that holds it."""
    ops = _operands(R, dev, M, N, K)
    row, col = M // 3, N - 7
    ops[1][row, 0], ops[3][col, -1] = 255, 255
    bias = _rand(dev, 6, N)
    bias[5] = math.inf
    q, s, _ = _blocks_of(R, ops, bias=bias)
    bad = torch.zeros_like(s, dtype=torch.bool)
    bad[row], bad[:, col // 32], bad[:, 0] = True, True, True
    assert torch.equal(s == 255, bad)
    assert (F.values(q, torch.zeros_like(s))[:, :N][bad.repeat_interleave(32, 1)[:, :N].cpu()] == 0).all()


def test_rows_far_apart_into_blocks(dev, R):
    """Rows past 32-bit offsets inside a tile."""
    far = (1 << 23) + 4096
    a, sa, w, sw = _operands(R, dev, 70, 65, 300)
    view = torch.full((70 * far,), 0xFF, dtype=U8, device=dev).as_strided((70, 150), (far, 1))
    view.copy_(a)
    for gelu in (False, True):
        got = _blocks_of(R, (view, sa, w, sw), gelu=gelu)
        for x, y in zip(got, _blocks_of(R, (a, sa, w, sw), gelu=gelu)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("spread", [40, 120])
def test_blocks_of_far_scales(dev, R, spread):
    """Results from subnormal to next to the largest, whose blocks' scales span the bytes."""
    g = torch.Generator().manual_seed(2)
    ops = []
    for n in (40, 72):
        ops.append(torch.randint(0, 256, (n, 128), generator=g, dtype=torch.int32).to(U8).to(dev))
        ops.append(torch.randint(127 - spread // 2, 127 + spread // 2, (n, 1), generator=g, dtype=torch.int32)
                   .expand(n, 8).to(U8).contiguous().to(dev))
    _, s, _ = _blocks_of(R, ops)
    assert int(s.max()) - int(s.min()) > spread // 2
