"""Checks of the layer operators' binding that need no GPU."""
import pytest
import torch

from paper_2609_34608_amd import runtime as R


def test_tensors_that_need_a_gradient_are_refused():
    t = torch.zeros(4, requires_grad=True)
    with pytest.raises(R.WamError, match="x: .*gradient"):
        R._operand(t, "x", (torch.float32,), -1)
    with torch.no_grad():
        assert R._operand(t, "x", (torch.float32,), -1) is t
    assert R._operand(t.detach(), "x", (torch.float32,), -1).shape == (4,)


@pytest.mark.parametrize("sections", [(2**32 + 8, 12, 12), (2**32, 0, 0), (-2**32 + 4, 0, 0), (8, 12, 2**40)])
def test_sections_past_32_bits_are_refused(sections):
    with pytest.raises(R.WamError):
        R.rope_frequencies(sections)
