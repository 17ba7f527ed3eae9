"""The model's layer variants in each form that their kernels take: the attention's
score bound under rotary positions."""
import pytest
import torch

from synth import make_initial_noise, make_observations, make_weights
from gpu_common import device, f32_sigmas, to_dev
from test_gpu_layer_variants import SECTIONS, _positions, _spec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _make(dev, spec, dtype, W):
    from paper_2609_34608_amd import runtime as R
    cfg = R.make_config(spec.B, spec.L, spec.D, spec.H, spec.F, spec.Nv, spec.Cv, spec.Na, spec.A, spec.No, spec.Co,
                        dtype, spec.qk_norm, spec.ln_eps)
    m = R.WamModel(cfg, W, device=dev)
    m.set_schedule(f32_sigmas(spec.K))
    return m


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("gain,bounded_turned", [(2.267, False), (2.255, True)])
def test_score_bound_of_turned_heads(dev, dtype, gain, bounded_turned):
    """The fixed softmax reference covers every score: q and k of unit RMS times their
    gains, rounded to bf16 (2^-8 each at most), and with rotary positions rounded once
    more.  log2(e) / 8 * 64 * gain^2 times 1 + 2^-7 is 59.78 and 59.15, times that again
    60.25 and 59.61: the first gains have a bound (60 at most) without rotary positions
    only, and the second with them too, so that a bounded form is what runs or is
    not."""
    from paper_2609_34608_amd import _lib as L, runtime as R
    spec = _spec(dtype, L=1)
    W = make_weights(spec, bias_std=0.02)
    W["l0.q_g"][:] = W["l0.k_g"][:] = gain
    m = _make(dev, spec, dtype, W)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)

    def out(form):
        m.set_option(L.WAM_OPT_ATTENTION, form)
        return m.hidden(3, x, cond, 1)

    assert not torch.equal(out(L.WAM_ATTN_BOUNDED), out(L.WAM_ATTN_RUNNING_MAX))
    m.set_rotary(to_dev(_positions(spec), dev), SECTIONS[64], R.rope_frequencies(SECTIONS[64], 100.0))
    assert torch.equal(out(L.WAM_ATTN_BOUNDED), out(L.WAM_ATTN_RUNNING_MAX)) != bounded_turned
    m.set_rotary(None)
    assert not torch.equal(out(L.WAM_ATTN_BOUNDED), out(L.WAM_ATTN_RUNNING_MAX))
    m.close()
