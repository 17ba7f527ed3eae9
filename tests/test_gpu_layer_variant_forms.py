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


def _near(got, h, gate, y, bias):
    """got = h + gate (y + bias), y known to half a bf16 step: three float32 roundings."""
    y, h, gate, bias = (t.double().cpu() for t in (y, h, gate, bias))
    want = h + gate * (y + bias)
    tol = gate.abs() * (2.0 ** -8 * y.abs() + 2.0 ** -24 * (y + bias).abs()) + 2.0 ** -23 * (want.abs() + h.abs())
    off = (got.double().cpu() - want).abs()
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("B,T,D,F", [(2, 89, 320, 640), (16, 1, 192, 384), (16, 70, 704, 1408)])
def test_fp8_layer_is_its_operators(dev, B, T, D, F):
    """A layer of the 8-bit mode from the operators without a handle, on the weights
    that they quantise: the MLP behind a closed attention gate, and (one row a sample, so
    that attention returns v) the attention block in front of a closed MLP gate.  What is
    left is the product's rounding to bf16, which the layer does without."""
    from paper_2609_34608_amd import runtime as R
    spec = _shape("fp8", B, T, D, F)
    W = make_weights(spec, bias_std=0.02, gain_std=0.1)
    W["l0.mod_w"][:] = 0  # the modulation is its bias
    rng = np.random.default_rng(3)
    shift1, scale1, gate1, shift2, scale2, gate2 = mod = (0.3 * rng.standard_normal((6, D))).astype(np.float32)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    dv = lambda a: to_dev(np.ascontiguousarray(a), dev)  # noqa: E731
    weight = {n: R.quantize_fp8(dv(np.asarray(W[f"l0.{n}_w"]).T), block_rows=128) for n in ("qkv", "proj", "fc1", "fc2")}

    def layer(closed):
        own = mod.copy()
        own[closed] = 0
        W["l0.mod_b"][:] = own.reshape(-1)
        m = _make(dev, spec, "fp8", W)
        h0, h1 = (m.hidden(3, x, cond, n).view(1, B * T, D).clone() for n in (0, 1))
        m.close()
        return h0, h1

    def project(u, s, name, **kw):
        return R.matmul_fp8(u.reshape(B * T, -1), s.reshape(B * T, -1), *weight[name], **kw)

    h0, h1 = layer(2)
    _, u, s = R.norm_residual(h0, scale=dv(scale2), shift=dv(shift2), eps=spec.ln_eps, u_dtype=R.FP8)
    q, s = project(u, s, "fc1", bias=dv(W["l0.fc1_b"]), gelu=True, out_dtype=R.FP8)
    _near(h1[0], h0[0], dv(gate2), project(q, s, "fc2"), dv(W["l0.fc2_b"]))
    if T > 1:
        return
    h0, h1 = layer(5)
    _, u, s = R.norm_residual(h0, scale=dv(scale1), shift=dv(shift1), eps=spec.ln_eps, u_dtype=R.FP8)
    v = project(u, s, "qkv", bias=dv(W["l0.qkv_b"]))[:, 2 * D:]
    q, s = R.quantize_fp8(v)
    _near(h1[0], h0[0], dv(gate1), project(q, s, "proj"), dv(W["l0.proj_b"]))


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("sections", [(8, 8, 0), (0, 0, 8), (10, 10, 10), (1, 0, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_layers_that_turn_a_part_of_the_head(dev, dtype, sections, layout):
    """Fewer pairs than half the head, whole units of eight and others, where q and k
    lie."""
    from paper_2609_34608_amd import runtime as R
    spec = _spec(dtype, L=1)
    W = make_weights(spec, bias_std=0.02, gain_std=0.1)
    m = _make(dev, spec, dtype, W)
    pos, freq = _positions(spec), R.rope_frequencies(sections, 100.0)
    m.set_rotary(to_dev(pos, dev), sections, freq, layout)
    _check(dev, spec, dtype, m, W, f32_sigmas(spec.K), rot=(pos, freq, sections, layout))
    m.close()
