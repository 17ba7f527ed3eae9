"""The README's operator examples run as they stand, one after the other, on a layer's tensors."""
import os
import re

import pytest
import torch

from gpu_common import device

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_operator_examples():
    dev = device()
    g = torch.Generator().manual_seed(1)

    def rand(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g).to(dtype).to(dev)

    B, T, H, dh = 2, 40, 4, 64
    D, pages, bf16 = H * dh, 16, torch.bfloat16
    i = torch.arange(T)
    names = dict(
        B=B, T=T, H=H, dh=dh, D=D, pages=pages, h=rand(B, T, D), y=rand(B, T, D, dtype=bf16), g=rand(B, 1, D), sc=rand(B, 1, D),
        sh=rand(B, 1, D), weight=0.06 * rand(3 * D, D), b=rand(3 * D), q=rand(B, T, H, dh, dtype=bf16),
        k=rand(B, T, H, dh, dtype=bf16), pos=torch.stack([i // 8, i // 4 % 2, i % 4], -1).float().to(dev), qg=1 + 0.1 * rand(dh),
        kg=1 + 0.1 * rand(dh), table=torch.randperm(pages, generator=g).view(B, -1).to(torch.int32).to(dev),
        lengths=torch.tensor([30, 70], dtype=torch.int32, device=dev))
    with open(README) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    assert len(blocks) == 2
    for block in blocks:
        exec(block, names)
    assert names["qkv"].shape == (B, T, 3, H, dh) and names["q"].shape == (B, T, H, dh)
    assert names["o"].shape == (B, T, H, dh) and names["o"].isfinite().all()
