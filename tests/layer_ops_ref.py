"""Plain float64 forms of the layer operators and the bounds on what their float32
arithmetic may be off by (d = 2^-24, half a float32 step), for the tests."""
import torch

D = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}
FP8 = torch.float8_e4m3fn
EPS = 1e-6


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


def f64_there(t):
    """The same, left on its device."""
    return None if t is None else t.detach().to(torch.float64)


def rope(x, pos, sections, freq, layout, gain=None, eps=EPS):
    """(result, bound): x [B, T, H, dh], pos [T, 3] or [B, T, 3]."""
    x, pos = f64(x), f64(pos)
    pos = pos.expand(x.shape[0], *pos.shape[-2:])
    dh = x.shape[-1]
    rel = 0.0
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * f64(gain)
        # the mean of squares: dh + 2 roundings; its root: half of that, and two
        # steps of its own; the products with the gain and the root
        rel = (dh + 2) / 2 * D + 6 * D
    P = sum(sections)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    ang = pos[..., axis] * torch.as_tensor(freq, dtype=torch.float64)
    c, s = torch.cos(ang)[:, :, None], torch.sin(ang)[:, :, None]
    if layout == "halves":
        i1, i2 = torch.arange(P), torch.arange(P) + P
    else:
        i1, i2 = 2 * torch.arange(P), 2 * torch.arange(P) + 1
    a, b = x[..., i1], x[..., i2]
    out = x.clone()
    out[..., i1], out[..., i2] = a * c - b * s, a * s + b * c
    # cos and sin: the reduced angle's rounding (2 pi 2^-26) and four steps of the
    # function; two products and their sum
    bound = rel * x.abs()
    for i in (i1, i2):
        bound[..., i] = (a.abs() + b.abs()) * (rel + 6.3 * 2.0 ** -26 + 4 * D + 3 * D)
    return out, bound


def standard(x, err, kind, eps=EPS):
    """(normalised x, bound), x off by at most err."""
    if kind == "none":
        return x, err
    n = x.shape[-1]
    if kind == "layer":
        mean = x.mean(-1, keepdim=True)
        # sum of n values: n roundings of partial sums of at most sum |x|
        emean = err.mean(-1, keepdim=True) + (n + 1) * D * x.abs().mean(-1, keepdim=True)
        x, err = x - mean, err + emean + D * (x - mean).abs()
    var = (x * x).mean(-1, keepdim=True)
    evar = 2 * (x.abs() * err).mean(-1, keepdim=True) + (err * err).mean(-1, keepdim=True) + (n + 2) * D * var
    rs = 1.0 / torch.sqrt(var + eps)
    rel = 0.5 * evar / (var + eps) + 5 * D
    return x * rs, (err + x.abs() * (rel + 2 * D)) * rs * (1 + rel)


def norm_residual(h, y=None, post="rms", post_gain=None, gate=None, res_scale=1.0, pre="layer", pre_gain=None,
                  scale=None, shift=None, eps=EPS):
    """((h_out, bound), (u, bound)) before the results' rounding."""
    h = f64(h)
    out = res_scale * h
    err = (D + abs(float(torch.tensor(res_scale, dtype=torch.float32)) - res_scale) / max(abs(res_scale), 1e-30)) * out.abs()
    if y is not None:
        v = f64(y)
        v, ev = standard(v, torch.zeros_like(v), post, eps)
        if post_gain is not None:
            v, ev = v * f64(post_gain), (ev + D * v.abs()) * f64(post_gain).abs()
        if gate is not None:
            v, ev = v * f64(gate), (ev + D * v.abs()) * f64(gate).abs()
        out = out + v
        err = err + ev + D * (out.abs() + v.abs())
    u, eu = standard(out, err, pre, eps) if pre is not None else (None, None)
    if u is not None:
        if pre_gain is not None:
            u, eu = u * f64(pre_gain), (eu + D * u.abs()) * f64(pre_gain).abs()
        if scale is not None:
            f = 1.0 + f64(scale)
            u, eu = u * f, eu * f.abs() + 2 * D * (u * f).abs()
        if shift is not None:
            u = u + f64(shift)
            eu = eu + D * u.abs() + D * f64(shift).abs()
    return (out, err), (u, eu)


def check(got, ref, bound, dtype=None, wide=f64):
    """|got - ref| within the bound and half a step of the result's type."""
    got = wide(got)
    tol = bound * (1 + 2.0 ** -8) + HALF[dtype or torch.float32] * (ref.abs() + bound) + 2.0 ** -133
    assert got.shape == ref.shape
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {((got - ref).abs() / tol).max():.3g} of the bound"


def check_blocks(q, s, x, bound, rows=1):
    """q (e4m3) and s stand for x [M, K], itself known to bound."""
    q, s = f64(q), f64(s)
    M, K = x.shape
    kb, mb = -(-K // 128), -(-M // rows)
    assert s.shape == (mb, kb)
    for i in range(mb):
        for j in range(kb):
            at = (slice(i * rows, (i + 1) * rows), slice(j * 128, (j + 1) * 128))
            most, off = x[at].abs().max(), bound[at].max()
            if most == 0 and off == 0:
                assert s[i, j] == 1
            elif most - off > 448 * 2.0 ** -126:
                assert abs(s[i, j] * 448 - most) <= off + 2 * D * most
            assert q[at].abs().max() <= 448
    full = s.repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]
    # half a step of e4m3: 2^-4 of the value, 2^-10 scales among the subnormals
    tol = bound + 2.0 ** -4 * (1 + 4 * D) * (x.abs() + bound) + full * 2.0 ** -10 * (1 + 4 * D)
    off = (q * full - x).abs()
    assert (off <= tol).all(), float((off / tol).max())


def check_row_blocks(q, s, x, bound):
    """check_blocks for blocks of 1 x 128, on the device of x."""
    q, s = f64_there(q), f64_there(s)
    M, K = x.shape
    for j in range(-(-K // 128)):
        at = slice(j * 128, (j + 1) * 128)
        most, off = x[:, at].abs().max(1).values, bound[:, at].max(1).values
        scale = s[:, j]
        # a block whose bound reaches zero may be a block of zeros, whose scale is 1 (a
        # GELU of -30 is 0 in float32 and 1e-40 here)
        zero = (scale == 1) & (most <= off) & (q[:, at] == 0).all(1)
        assert (((scale * 448 - most).abs() <= off + 2 * D * most + 448 * 2.0 ** -126) | zero).all()
        tol = bound[:, at] + 2.0 ** -4 * (1 + 4 * D) * (x[:, at].abs() + bound[:, at])
        tol = tol + scale[:, None] * 2.0 ** -10 * (1 + 4 * D)
        off = (q[:, at] * scale[:, None] - x[:, at]).abs()
        assert (off <= tol).all(), float((off / tol).max())


def values(q, s, rows, wide=f64):
    """The float64 matrix that blocks of (rows x 128) stand for."""
    q, s = wide(q), wide(s)
    M, K = q.shape
    return q * s.repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]


def _cut(a, a_scale, w, w_scale, wide):
    """What the 8-bit matrix instruction may cut off a bf16 result's sums: in a group
    of 8 consecutive k, with E the largest sum of the two operands' exponents (of
    subnormals and normals below 2^-6: -6), each of at most 8 products loses less
    than 2^(E - 13)."""
    def power(q):  # 2^exponent, 0 for a zero
        q = wide(q).abs()
        e = torch.exp2(torch.floor(torch.log2(q.clamp_min(2.0 ** -20))).clamp_min(-6.0))
        return torch.where(q > 0, e, torch.zeros_like(q))
    (M, K), N = a.shape, w.shape[0]
    pa, pw = power(a), power(w)
    total = torch.zeros(M, N, dtype=torch.float64, device=pa.device)
    sa, sw = wide(a_scale), wide(w_scale).repeat_interleave(128, 0)[:N]
    for k in range(0, K, 8):
        top = torch.zeros_like(total)
        for i in range(k, min(K, k + 8)):
            top = torch.maximum(top, pa[:, i:i + 1] * pw[:, i])
        total += 8 * 2.0 ** -13 * top * sa[:, k // 128, None] * sw[:, k // 128]
    return total


def matmul(a, a_scale, w, w_scale, bias=None, gelu=False, dtype=torch.float32, wide=f64):
    """(product, bound): the 128 products of a block are exact in float32; their sum
    takes 128 roundings (of a full step each at most), its scaling and the sum over
    the blocks four half steps a block.  With a bf16 result the products are cut
    first (_cut)."""
    A, W = values(a, a_scale, 1, wide), values(w, w_scale, 128, wide)
    c, most = A @ W.t(), A.abs() @ W.abs().t()
    blocks = -(-A.shape[1] // 128)
    err = most * D * (2 * 128 + 4 * blocks)
    if dtype == torch.bfloat16:
        err = err + _cut(a, a_scale, w, w_scale, wide)
    if bias is not None:
        c = c + wide(bias)
        err = err + D * c.abs()
    if gelu:
        x, z = c, 2.0 * (2.0 / torch.pi) ** 0.5 * (c + 0.044715 * c ** 3)
        c = x * torch.sigmoid(z)
        # slope at most 1.13; the exponent's relative error (four roundings) moves the
        # sigmoid by |z| times that at most, the rest is three steps of the result
        err = 1.13 * err + 8 * D * c.abs() * (1 + z.abs())
    return c, err
