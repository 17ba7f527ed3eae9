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
