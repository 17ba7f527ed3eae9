"""The layer operators inside the model: 8-bit projections (WAM_FP8), rotary
positions (wam_set_rotary) and post-norms (wam_set_post_norm), single layers
teacher-forced on the device's own hidden state against a float64 layer, and
their ways through replans, graphs and Residual Rescaling.

Tolerances.  float32: the longest sums, (F + 3 D) 2^-24 of the update's largest
value.  bf16: BF16_UPDATE_TOL covers four roundings of activations; rotated q / k and
a post-norm's input are two more, so sqrt(6 / 4) of it.  fp8, 2-norm: the reference
has the same weights and the same blocks, but where a value lies within the bf16
rounding of a block boundary the two sides round apart, by a step; were that so for
every value, an operand would be off by 2^-4 / sqrt(3) in the 2-norm, and the two
terms of the update by sqrt(2) of it together: 5.1%, and 1% for the rest.
"""
import numpy as np
import pytest
import torch

from oracle import dit as OD
from synth import get_workload, make_initial_noise, make_observations, make_remap_noise, make_weights
from gpu_common import BF16_UPDATE_TOL, device, f32_sigmas, rel_err, to_dev

pytestmark = pytest.mark.gpu

SECTIONS = {64: (8, 12, 12), 32: (4, 6, 6)}


@pytest.fixture(scope="module")
def dev():
    return device()


def _spec(dtype="bf16", L=2, B=2, D=256, H=None, F=512, Nv=60, Na=16, No=13, **kw):
    return get_workload("small").replace(L=L, D=D, H=H or D // 64, F=F, Nv=Nv, Na=Na, No=No, B=B,
                                         dtype="fp32" if dtype == "fp32" else "bf16", **kw)


def _model(dev, spec, dtype, **kw):
    from paper_2609_34608_amd import runtime as R
    W = make_weights(spec, bias_std=0.02, gain_std=0.1)
    cfg = R.make_config(spec.B, spec.L, spec.D, spec.H, spec.F, spec.Nv, spec.Cv, spec.Na, spec.A, spec.No, spec.Co,
                        dtype, spec.qk_norm, spec.ln_eps)
    m = R.WamModel(cfg, W, device=dev, **kw)
    sig = f32_sigmas(spec.K)
    m.set_schedule(sig)
    return W, m, sig


def _e4m3(v):
    return torch.from_numpy(np.asarray(v, np.float32)).to(torch.float8_e4m3fn).to(torch.float64).numpy()


def _blocks(x, rows):
    """x [M, K] as it comes back from blocks of (rows x 128)."""
    x = np.asarray(x, np.float32)
    out = np.empty(x.shape, np.float64)
    for i in range(0, x.shape[0], rows):
        for j in range(0, x.shape[1], 128):
            b = x[i:i + rows, j:j + 128]
            top = np.abs(b).max(axis=(None if rows > 1 else 1), keepdims=True).astype(np.float32)
            s = np.where(top > 0, top / np.float32(448), np.float32(1)).astype(np.float32)
            out[i:i + rows, j:j + 128] = _e4m3(b / s) * s.astype(np.float64)
    return out


def _turn(x, pos, freq, sections, layout):
    """x [B, H, T, dh] turned by the rows' positions."""
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    ang = pos[:, axis] * np.asarray(freq)
    P = len(axis)
    i1 = np.arange(P) if layout == "halves" else 2 * np.arange(P)
    i2 = i1 + (P if layout == "halves" else 1)
    out = x.copy()
    c, s = np.cos(ang), np.sin(ang)
    out[..., i1] = x[..., i1] * c - x[..., i2] * s
    out[..., i2] = x[..., i1] * s + x[..., i2] * c
    return out


def _layer(W, spec, l, h, c, fp8=False, rot=None, post=None):
    """oracle.dit.dit_layer with the variants."""
    B, T, D = h.shape
    H, dh = spec.H, D // spec.H
    h = np.asarray(h, np.float64)
    sh1, sc1, g1, sh2, sc2, g2 = OD.layer_modulation(W, l, c)

    def lin(x, name):
        w = OD.as64(W[f"l{l}.{name}_w"])
        if fp8:
            w = _blocks(w.T, 128).T
            x = _blocks(x.reshape(-1, x.shape[-1]), 1).reshape(x.shape)
        return x @ w + OD.as64(W[f"l{l}.{name}_b"])

    def after(y, i):
        return y if post is None else OD.rms_norm(y, spec.ln_eps) * post[l, i]

    u = OD.layer_norm(h, spec.ln_eps) * (1.0 + sc1) + sh1
    q, k, v = (a.reshape(B, T, H, dh).transpose(0, 2, 1, 3) for a in np.split(lin(u, "qkv"), 3, axis=-1))
    if spec.qk_norm:
        q = OD.rms_norm(q, spec.ln_eps) * OD.as64(W[f"l{l}.q_g"])
        k = OD.rms_norm(k, spec.ln_eps) * OD.as64(W[f"l{l}.k_g"])
    if rot is not None:
        q, k = _turn(q, *rot), _turn(k, *rot)
    o = OD.attention(q, k, v).transpose(0, 2, 1, 3).reshape(h.shape)
    h = h + g1 * after(lin(o, "proj"), 0)
    u = OD.layer_norm(h, spec.ln_eps) * (1.0 + sc2) + sh2
    return h + g2 * after(lin(OD.gelu_tanh(lin(u, "fc1")), "fc2"), 1)


def _positions(spec):
    """Video rows on a grid, action rows along time, observation rows before it."""
    T = spec.T
    i = np.arange(T, dtype=np.float64)
    p = np.stack([i // 12, (i // 4) % 3, i % 4], -1)
    p[spec.Nv:spec.Nv + spec.Na] = np.stack([0.25 * np.arange(spec.Na), *(np.zeros((2, spec.Na)))], -1)
    p[spec.Nv + spec.Na:] = [-1.0, 0.5, 7.0]
    return p


def _check(dev, spec, dtype, m, W, sig, rot=None, post=None, layers=None):
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    for k in (0, 6):
        c = OD.cond_vector(W, sig[k])
        h = m.hidden(k, x, cond, 0).cpu().numpy()
        for l in range(spec.L if layers is None else layers):
            out = m.hidden(k, x, cond, l + 1).cpu().numpy()
            ref = _layer(W, spec, l, h, c, dtype == "fp8", rot, post) - h
            got = out.astype(np.float64) - h
            if dtype == "fp8":
                err, tol = np.linalg.norm(got - ref) / np.linalg.norm(ref), 0.061
            else:
                err = rel_err(got, ref)
                # the update is a difference of float32 hidden states: half a step each
                step = 2.0 ** -23 * np.abs(h).max() / np.abs(ref).max()
                tol = (spec.F + 3 * spec.D) * 2.0 ** -24 + step if dtype == "fp32" else BF16_UPDATE_TOL * (6 / 4) ** 0.5
            print(f"{dtype} step {k} layer {l}: update err {err:.2e} of {tol:.2e}")
            assert err <= tol
            h = out


@pytest.mark.parametrize("kw", [dict(), dict(D=128, H=2, F=384, B=1, Nv=1, Na=0, No=0), dict(D=320, H=5, F=640, Nv=200),
                                dict(qk_norm=False), dict(D=704, H=11, F=1408, B=3, Nv=400, L=1)])
def test_fp8_layers(dev, kw):
    spec = _spec("fp8", **kw)
    W, m, sig = _model(dev, spec, "fp8")
    _check(dev, spec, "fp8", m, W, sig)
    m.close()


@pytest.mark.parametrize("name", ["small", "mid"])
def test_fp8_layer_at_model_sizes(dev, name):
    """One layer of the single-arm and of the bimanual model (rows sampled by the
    reference's own cost: one sample)."""
    spec = get_workload(name).replace(L=1, B=1)
    W, m, sig = _model(dev, spec, "fp8")
    _check(dev, spec, "fp8", m, W, sig)
    m.close()


def test_fp8_weights_are_the_operator_blocks(dev):
    """The weights wam_init packs are those of wam_quantize_fp8, bit for bit."""
    from paper_2609_34608_amd import runtime as R
    spec = _spec("fp8", L=1, D=192, H=3, F=384)
    W, m, sig = _model(dev, spec, "fp8")
    raw = m.wdev.cpu().numpy().tobytes()
    for name in ("qkv", "proj", "fc1", "fc2"):
        w = np.ascontiguousarray(np.asarray(W[f"l0.{name}_w"], np.float32).T)
        q, s = R.quantize_fp8(to_dev(w, dev), block_rows=128)
        assert q.contiguous().view(torch.uint8).cpu().numpy().tobytes() in raw
        assert s.cpu().numpy().tobytes() in raw
    m.close()


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("fp32", 64), ("fp32", 32), ("fp8", 64)])
def test_rotary_layers(dev, dtype, dh, layout):
    from paper_2609_34608_amd import runtime as R
    spec = _spec(dtype, H=256 // dh)
    W, m, sig = _model(dev, spec, dtype)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    plain = m.hidden(3, x, cond, spec.L).cpu().numpy()
    table = m.hidden(3, x, cond, 0).cpu().numpy()
    pos, sec = _positions(spec), SECTIONS[dh]
    freq = R.rope_frequencies(sec, 100.0)
    m.set_rotary(to_dev(pos, dev), sec, freq, layout)
    _check(dev, spec, dtype, m, W, sig, rot=(pos, freq, sec, layout))
    # the additive table is gone, and stays with keep_table
    got = m.hidden(3, x, cond, 0).cpu().numpy()
    want = OD.embed_tokens(W, spec, make_initial_noise(spec), make_observations(spec, 0)[0])
    want = want - OD.positional_embedding(spec.T, spec.D)[None]
    assert rel_err(got, want) <= 1e-6
    m.set_rotary(to_dev(pos, dev), sec, freq, layout, keep_table=True)
    np.testing.assert_array_equal(m.hidden(3, x, cond, 0).cpu().numpy(), table)
    assert rel_err(m.hidden(3, x, cond, 1).cpu().numpy(), plain) > 1e-4
    # back to the model as it was
    m.set_rotary(None)
    np.testing.assert_array_equal(m.hidden(3, x, cond, spec.L).cpu().numpy(), plain)
    m.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("kw", [dict(), dict(D=128, H=2, F=384, B=1, Nv=40), dict(D=320, H=5, F=640, Nv=200)])
def test_post_norm_layers(dev, dtype, kw):
    from paper_2609_34608_amd import runtime as R
    spec = _spec(dtype, **kw)
    W, m, sig = _model(dev, spec, dtype)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    plain = m.hidden(3, x, cond, spec.L).cpu().numpy()
    post = (0.3 + 0.1 * np.random.default_rng(5).standard_normal((spec.L, 2, spec.D))).astype(np.float32)
    m.set_post_norm(to_dev(post, dev))
    _check(dev, spec, dtype, m, W, sig, post=post.astype(np.float64))
    # with rotary positions as well
    pos, sec = _positions(spec), SECTIONS[64]
    freq = R.rope_frequencies(sec, 100.0)
    m.set_rotary(to_dev(pos, dev), sec, freq)
    _check(dev, spec, dtype, m, W, sig, rot=(pos, freq, sec, "halves"), post=post.astype(np.float64))
    m.set_rotary(None)
    m.set_post_norm(None)
    np.testing.assert_array_equal(m.hidden(3, x, cond, spec.L).cpu().numpy(), plain)
    m.close()


def _variants(m, spec, dev):
    from paper_2609_34608_amd import runtime as R
    sec = SECTIONS[64]
    m.set_rotary(to_dev(_positions(spec), dev), sec, R.rope_frequencies(sec, 100.0))
    post = 0.3 + 0.1 * np.random.default_rng(5).standard_normal((spec.L, 2, spec.D))
    m.set_post_norm(to_dev(post, dev))


@pytest.mark.parametrize("rr_mode", ["AUTO", "FORCE_SKIP"])
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_replans_agree_in_every_mode(dev, dtype, rr_mode):
    """Closed-loop replans of a model with every variant: host decision, device
    decision and captured graphs, replayed with eager work between, give the same
    bits."""
    from paper_2609_34608_amd import _lib as L, runtime as R
    spec = _spec(dtype, L=4, B=1, K=10)
    rr = R.rr_profile(1, 2, 3, getattr(L, f"WAM_RR_{rr_mode}"))
    obs = make_observations(spec, 4)
    outs = []
    for own, devdec, graphs in ((False, 0, 0), (False, 1, 0), (True, 1, 1)):
        W, m, sig = _model(dev, spec, dtype, own_stream=own)
        _variants(m, spec, dev)
        m.set_option(L.WAM_OPT_DEVICE_DECISION, devdec)
        m.set_option(L.WAM_OPT_GRAPHS, graphs)
        x_out, got = m.new_traj(), []
        for t in range(4):
            cr, cp = to_dev(obs[t], dev), to_dev(0.9 * obs[max(t - 1, 0)], dev)
            m.replan(cr, x_out, to_dev(make_remap_noise(spec, t), dev), cond_pred=cp, u_hat=[cp], u=[cr], delta=[2.3],
                     weight=[1.0], noise_first=to_dev(make_initial_noise(spec), dev), rr=rr, b0=5, r=5, shift_action=3,
                     k1=2, tau=10.0)
            got.append(x_out.cpu().numpy())
            if t == 2:  # turned off and on again: the next replans capture anew
                m.set_post_norm(None)
                _variants(m, spec, dev)
        outs.append(got)
        m.close()
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert np.isfinite(a).all()
            np.testing.assert_array_equal(a, b)


def test_changing_a_variant_drops_the_layer_state(dev):
    from paper_2609_34608_amd import _lib as L, runtime as R
    spec = _spec("bf16", L=4, B=1)
    W, m, sig = _model(dev, spec, "bf16")
    rr = R.rr_profile(1, 2, 3, L.WAM_RR_FORCE_SKIP)
    x, cond = to_dev(make_initial_noise(spec), dev), to_dev(make_observations(spec, 0)[0], dev)
    m.velocity(0, x, cond, rr=rr)
    assert m.velocity(1, x, cond, rr=rr)[1].accepted
    _variants(m, spec, dev)
    assert not m.velocity(1, x, cond, rr=rr)[1].attempted
    m.close()


def test_refusals(dev):
    from paper_2609_34608_amd import _lib as L, runtime as R
    spec = _spec("bf16")
    W, m, sig = _model(dev, spec, "bf16")
    pos, sec, freq = to_dev(_positions(spec), dev), (8, 12, 12), R.rope_frequencies((8, 12, 12))
    for bad in (dict(pos=pos[:-1]), dict(sections=(8, 12)), dict(freq=freq[1:]), dict(layout="x"),
                dict(sections=(33, 0, 0), freq=np.ones(33)), dict(sections=(0, 0, 0), freq=[]),
                dict(sections=(-1, 2, 0), freq=[1.0]), dict(pos=pos.double())):
        kw = dict(pos=pos, sections=sec, freq=freq)
        kw.update(bad)
        with pytest.raises(R.WamError):
            m.set_rotary(**kw)
    with pytest.raises(R.WamError):
        m.set_post_norm(torch.ones(spec.L, spec.D, device=dev))
    # while a replan is open
    x0 = to_dev(make_initial_noise(spec), dev)
    cond = to_dev(make_observations(spec, 0)[0], dev)
    args = m.replan_args(cond, m.new_traj(), x0, cond_pred=cond, u_hat=[cond], u=[cond], delta=[1.0], weight=[1.0],
                         noise_first=x0, b0=5, r=5, k1=2)
    m.replan_begin(args)
    for call in (lambda: m.set_rotary(pos, sec, freq), lambda: m.set_rotary(None), lambda: m.set_post_norm(None)):
        with pytest.raises(R.WamError, match="open"):
            call()
    m.replan_end(args)
    m.close()
