"""Plain forms of the 4-bit operators in float64, and how far a kernel may be from them.

Everything held in 4 bits is compared exactly: the operators fix each code.  Products
and attention come with a bound per element, derived beside it."""
import math

import torch

F64 = torch.float64
MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def quantize(x):
    """(codes, scale bytes) of the last axis of x (float32 values, on the CPU): the nearest
    magnitude by distance, ties to the even code."""
    x = x.detach().cpu().to(F64)
    K = x.shape[-1]
    kb = -(-K // 32)
    p = torch.nn.functional.pad(x, (0, kb * 32 - K)).unflatten(-1, (kb, 32))
    most = p.abs().amax(-1)
    bad = ~torch.isfinite(p).all(-1)
    clean = torch.where(bad, 0.0, most)
    e = torch.where(clean > 0, torch.frexp(clean)[1].to(F64) - 3, torch.tensor(-127.0, dtype=F64)).clamp_min(-127)
    y = torch.where(bad[..., None], 0.0, p) / torch.exp2(e)[..., None]
    dist = (y.abs()[..., None] - MAGNITUDES).abs()
    dist = dist + 1e-9 * (torch.arange(8) % 2)  # a tie goes to the even code
    code = dist.argmin(-1) + 8 * torch.signbit(y)
    code = torch.where(bad[..., None], 0, code).flatten(-2)[..., :K]
    if K % 2:
        code = torch.nn.functional.pad(code, (0, 1))
    q = (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)
    return q, torch.where(bad, 255, e.to(torch.int64) + 127).to(torch.uint8)


def values(q, scale):
    """float64 values of codes and scale bytes [..., n], [..., ceil(n / 16)]."""
    q, scale = q.cpu(), scale.cpu()
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2).long()
    v = MAGNITUDES[code & 7] * torch.where(code >= 8, -1.0, 1.0).to(F64)
    s = torch.exp2(scale.to(F64) - 127)
    s = torch.where(scale == 255, math.nan, s)
    return v * s.repeat_interleave(32, -1)[..., :v.shape[-1]]


def same(got, want):
    """Equal values, NaN where NaN."""
    got, want = got.detach().cpu().to(F64), want.cpu().to(F64)
    assert got.shape == want.shape
    ok = (got == want) | (got.isnan() & want.isnan())
    assert ok.all(), f"{int((~ok).sum())} of {ok.numel()} differ, first at {(~ok).nonzero()[0].tolist()}"


def check(got, ref, bound, dtype):
    """|got - ref| <= bound + half a step of the result's type; NaN and infinities alike."""
    got, ref, bound = got.detach().cpu().to(F64), ref.cpu(), bound.cpu()
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)) and torch.equal(got.isnan(), ref.isnan())
    tol = bound + half_step(dtype) * (ref.abs() + bound) + torch.finfo(dtype).smallest_normal
    over = ((got - ref).abs() / tol)[fine]
    assert over.numel() == 0 or over.max() <= 1.0, f"{over.max():.3g} of the bound"


def gelu(c):
    return c / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (c + 0.044715 * c ** 3)))


def matmul(a, sa, w, sw, bias=None, act=False):
    """Product and bound: each matrix step of 128 of K adds at most 2^-22 of the magnitudes of
    its products and of what it adds to, which stays below the sum of all magnitudes; the
    bias one rounding.  The GELU has a slope of at most 1.13 and its float32 arithmetic
    (an exponential and a reciprocal of 1 ulp, the argument 2^-22 of |2 u log2 e| <= 3.2 |c| +
    0.15 |c|^3, which counts only where the exponential does: below 90 of it) is within
    2^-22 (4 + 90) of the result."""
    a, w = values(a, sa), values(w, sw)
    steps = -(-a.shape[-1] // 128)
    c, mag = a @ w.t(), a.abs() @ w.abs().t()
    err = 2.0 ** -22 * (steps + 1) * mag
    if bias is not None:
        c = c + bias.cpu().to(F64)
        err = err + 2.0 ** -24 * (c.abs() + err)
    if act:
        c = gelu(c)
        err = 1.13 * err + 2.0 ** -22 * 94 * c.abs() + 1e-30
    return c, err


def keys(k, sections, freq, layout, pos, gain, eps=1e-6):
    """k [B, T, H, dh] as it goes into blocks: normed and turned in float64, then float32."""
    k = k.detach().cpu().to(F64)
    if gain is not None:
        k = k / torch.sqrt((k * k).mean(-1, keepdim=True) + eps) * gain.cpu().to(F64)
    P = sum(sections)
    if P == 0:
        return k.to(torch.float32)
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)])
    pos = pos.cpu().to(F64)
    ang = (pos if pos.dim() == 3 else pos[None])[..., axis] * torch.as_tensor(list(freq), dtype=F64)
    c, s = ang.cos()[:, :, None], ang.sin()[:, :, None]
    first = torch.arange(P) if layout == "halves" else 2 * torch.arange(P)
    second = first + (P if layout == "halves" else 1)
    out = k.clone()
    out[..., first] = k[..., first] * c - k[..., second] * s
    out[..., second] = k[..., first] * s + k[..., second] * c
    return out.to(torch.float32)


def append(cache, k, v, table, start, rows=None):
    """The cache's four arrays (CPU copies) after the rows of k (from keys) and v."""
    out = [t.detach().cpu().clone() for t in cache]
    pages, page = out[0].shape[:2]
    table, start = table.cpu(), start.cpu()
    for b in range(k.shape[0]):
        for t in range(k.shape[1] if rows is None else min(int(rows[b]), k.shape[1])):
            at = int(start[b]) + t
            if at < 0 or at // page >= table.shape[1] or not 0 <= int(table[b, at // page]) < pages:
                continue
            p, i = int(table[b, at // page]), at % page
            out[0][p, i], out[1][p, i] = quantize(k[b, t])
            out[2][p, i], out[3][p, i] = quantize(v[b, t].to(torch.float32))
    return out


def seen(length, room, causal, rows, t):
    held = max(0, min(length, room))
    if t >= rows:
        return 0
    return held if not causal else max(0, min(held, length - rows + t + 1))


def attention(q, cache, table, lengths, *, rows=None, causal=False, scale=None):
    """(out, lse, bound of out, bound of lse).  With p the float32 probabilities the kernel
    forms, relative errors of p: its score is a float32 sum of dh exact products in dh / 32
    matrix steps (2^-22 each of the magnitudes X = scale sum |q k|), one product with the
    scale and one difference in log2 units (2^-24 of |x| <= 1.45 X and of |m| <= 1.45 X),
    then an exponential of 2^-22; with bf16 q also half a step of bf16.  float32 q and p
    are used in three bf16 parts, which drop nothing above 2^-24.  A sum over n tokens in
    steps of 32 adds 2^-22 (n / 32 + 16) (steps, tiles' rescales and the joins).  A
    relative error d of every p moves out = sum p v / sum p by at most d (sum p |v| / sum p +
    |out|), and the sums' as much again."""
    B, T, Hq, dh = q.shape
    exact = q.dtype == torch.float32
    q = q.detach().cpu().to(F64)
    k, v = values(cache[0], cache[1]), values(cache[2], cache[3])
    pages, page, H = k.shape[:3]
    table, lengths = table.cpu(), lengths.cpu()
    scale = 1.0 / math.sqrt(dh) if scale is None else scale
    out, bound = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((B, T, Hq), -math.inf, dtype=F64)
    lse_bound = torch.zeros(B, T, Hq, dtype=F64)
    room = table.shape[1] * page
    for b in range(B):
        tokens = [(int(table[b, t // page]), t % page, t) for t in range(max(0, min(int(lengths[b]), room)))
                  if 0 <= int(table[b, t // page]) < pages]
        if not tokens:
            continue
        pg, place, index = (torch.tensor(x) for x in zip(*tokens))
        n = T if rows is None else min(int(rows[b]), T)
        for t in range(T):
            sees = index < seen(int(lengths[b]), room, causal, n, t)
            if not sees.any():
                continue
            for h in range(Hq):
                kk, vv = (x[pg[sees], place[sees], h * H // Hq] for x in (k, v))
                s = scale * (kk @ q[b, t, h])
                X = float((scale * (kk.abs() @ q[b, t, h].abs())).max())
                p = torch.exp(s - s.max())
                total = p.sum()
                o, mag = p @ vv / total, p @ vv.abs() / total
                d = 2.0 ** -22 * (2 + dh / 32 * X + 2 * X) + (0 if exact else half_step(torch.bfloat16))
                d += 2.0 ** -22 * (len(s) / 32 + 16)
                out[b, t, h], bound[b, t, h] = o, d * (mag + o.abs())
                lse[b, t, h] = s.max() + torch.log(total)
                lse_bound[b, t, h] = d + 2.0 ** -22 * (abs(float(lse[b, t, h])) + X)
    return out, lse, bound, lse_bound


def attention_whole(q, cache, table, lengths, *, rows=None, causal=False, scale=None):
    """attention (same results and bounds), a head's rows at once and on q's device, for sizes
    past a row at a time."""
    B, T, Hq, dh = q.shape
    dev, exact = q.device, q.dtype == torch.float32
    k, v = (values(*c).to(dev) for c in (cache[:2], cache[2:]))
    pages, page, H = k.shape[:3]
    scale = 1.0 / math.sqrt(dh) if scale is None else scale
    out, bound = (torch.zeros(q.shape, dtype=F64, device=dev) for _ in range(2))
    lse = torch.full((B, T, Hq), -math.inf, dtype=F64, device=dev)
    lse_bound = torch.zeros(B, T, Hq, dtype=F64, device=dev)
    room = table.shape[1] * page
    for b in range(B):
        length = int(lengths[b])
        token = torch.arange(max(0, min(length, room)), device=dev)
        entry = table[b].long()[token // page]
        token, entry = token[(entry >= 0) & (entry < pages)], entry[(entry >= 0) & (entry < pages)]
        if not len(token):
            continue
        n = T if rows is None else min(int(rows[b]), T)
        sees = token < torch.tensor([seen(length, room, causal, n, t) for t in range(T)], device=dev)[:, None]
        some = sees.any(-1)
        for h in range(Hq):
            kk, vv = (x[entry, token % page, h * H // Hq] for x in (k, v))
            x = q[b, :, h].to(F64)
            s = torch.where(sees, scale * (x @ kk.t()), -math.inf)
            X = torch.where(sees, scale * (x.abs() @ kk.abs().t()), 0.0).amax(-1, keepdim=True)
            top = s.amax(-1, keepdim=True).clamp_min(-1e300)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True).clamp_min(1e-300)
            o, mag = p @ vv / total, p @ vv.abs() / total
            d = 2.0 ** -22 * (2 + dh / 32 * X + 2 * X) + (0 if exact else half_step(torch.bfloat16))
            d = d + 2.0 ** -22 * (sees.sum(-1, keepdim=True) / 32 + 16)
            value = (top + torch.log(total))[:, 0]
            out[b, :, h], bound[b, :, h] = torch.where(some[:, None], o, 0.0), d * (mag + o.abs())
            lse[b, :, h] = torch.where(some, value, -math.inf)
            lse_bound[b, :, h] = torch.where(some, d[:, 0] + 2.0 ** -22 * (value.abs() + X[:, 0]), 0.0)
    return out, lse, bound, lse_bound
