"""The model's layer variants in each form that their kernels take: the attention's
score bound under rotary positions, and every tile of the projections."""
import numpy as np
import pytest
import torch

from synth import make_initial_noise, make_observations, make_weights
from gpu_common import device, f32_sigmas, to_dev
from test_gpu_layer_variants import SECTIONS, _check, _positions, _spec

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


# (B, T, D, F).  Batches whose projections take the larger tiles of the 8-bit mode, each
# epilogue (QKV, MLP-up into blocks, gated residual, bias in front of a post-norm) on
# every tile that the planner gives it, with rows left over and, of 256 columns,
# columns too (tests/test_plan_layer_forms.py).
FP8_TILES = [(16, 113, 448, 1792), (15, 159, 576, 1920), (16, 691, 320, 896), (15, 685, 448, 1536), (15, 503, 1088, 896),
             (2, 3, 192, 256), (16, 619, 1088, 128)]
# the same for the bias alone of bf16 projections in front of a post-norm
BF16_TILES = [(2, 3, 64, 256), (16, 161, 640, 2432), (15, 637, 832, 128), (16, 261, 256, 896), (15, 107, 640, 2432),
              (16, 613, 320, 128), (16, 673, 448, 128), (16, 621, 1088, 256), (16, 689, 1344, 128)]
# and of float32 ones
FP32_TILES = [(15, 411, 128, 256), (13, 539, 448, 128), (16, 389, 256, 128), (16, 469, 320, 640)]


def _shape(dtype, B, T, D, F):
    na, no = min(7, T // 3), min(5, T // 4)
    return _spec(dtype, L=1, B=B, D=D, F=F, Nv=T - na - no, Na=na, No=no)


def _gains(spec, dev):
    post = (0.3 + 0.1 * np.random.default_rng(5).standard_normal((spec.L, 2, spec.D))).astype(np.float32)
    return post.astype(np.float64), to_dev(post, dev)


@pytest.mark.parametrize("dtype,B,T,D,F", [("fp8", *s) for s in FP8_TILES] + [("bf16", *s) for s in BF16_TILES])
def test_tiles_give_the_bits_of_single_samples(dev, dtype, B, T, D, F):
    """A sample's layer does not depend on the others of its batch, whatever tiles the
    batch takes: the same bits as by itself, where its few rows take small tiles; and
    those against the float64 layer.  (One attention kernel for both, the one that
    has a single form.)"""
    from paper_2609_34608_amd import _lib as L
    spec = _shape(dtype, B, T, D, F)
    W = make_weights(spec, bias_std=0.02, gain_std=0.1)
    post, gains = _gains(spec, dev)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    one = spec.replace(B=1)
    batch, single = _make(dev, spec, dtype, W), _make(dev, one, dtype, W)
    for m in (batch, single):
        m.set_option(L.WAM_OPT_ATTENTION, L.WAM_ATTN_PINGPONG)
    for g in ((None, gains) if dtype == "fp8" else (gains,)):
        for m in (batch, single):
            m.set_post_norm(g)
        h0, h1 = (batch.hidden(3, x, cond, n) for n in (0, 1))
        assert h1.isfinite().all() and not torch.equal(h0, h1)
        for b in (0, B // 2, B - 1):
            assert torch.equal(h0[b], single.hidden(3, x[b:b + 1], cond[b:b + 1], 0)[0])
            assert torch.equal(h1[b], single.hidden(3, x[b:b + 1], cond[b:b + 1], 1)[0])
        _check(dev, one, dtype, single, W, f32_sigmas(spec.K), post=None if g is None else post)
    batch.close()
    single.close()


@pytest.mark.parametrize("B,T,D,F", FP32_TILES)
def test_float32_post_norm_tiles(dev, B, T, D, F):
    spec = _shape("fp32", B, T, D, F)
    W = make_weights(spec, bias_std=0.02, gain_std=0.1)
    post, gains = _gains(spec, dev)
    m = _make(dev, spec, "fp32", W)
    m.set_post_norm(gains)
    _check(dev, spec, "fp32", m, W, f32_sigmas(spec.K), post=post)
    m.close()
