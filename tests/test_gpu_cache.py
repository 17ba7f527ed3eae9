"""The paged cache of 4-bit blocks on the GPU: appending and attention against float64
(fp4_ref), at the lengths, pages, masks, strides and values where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import fp4_ref as F
from gpu_common import device

pytestmark = pytest.mark.gpu

BF16, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


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


def _ints(dev, *v):
    return torch.tensor(v, dtype=I32, device=dev)


def _table(dev, seed, B, width, extra=2):
    """Pages in no order; and how many the pool has."""
    g = torch.Generator().manual_seed(seed)
    pages = B * width + extra
    return torch.randperm(pages, generator=g)[:B * width].view(B, width).to(I32).to(dev), pages


def _strided(x, order, pad=0, offset=0):
    """x with its leading dimensions laid out in `order` (outermost first), rows `pad`
    elements further apart, `offset` elements into its storage."""
    shape = [x.shape[i] for i in order] + [x.shape[-1] + pad]
    buf = torch.zeros(int(np.prod(shape)) + offset, device=x.device).to(x.dtype)[offset:].view(shape)
    view = buf[..., :x.shape[-1]].permute(*[list(order).index(i) for i in range(len(order))], len(order))
    view.copy_(x)
    return view


def _filled(R, dev, seed, pages, page, H, dh):
    """A cache whose every byte holds something: codes of unit normal values, or, as an older
    history may leave them, NaN scales in its last page."""
    cache = R.new_kv_cache(pages, page, H, dh, dev)
    for i, (q, s) in enumerate((cache[:2], cache[2:])):
        x = _rand(dev, seed + i, pages * page * H, dh)
        a, b = R.quantize_fp4(x)
        q.copy_(a.view(pages, page, H, dh // 2))
        s.copy_(b.view(pages, page, H, dh // 32))
    return cache


def _positions(dev, T, B=None, far=0.0):
    i = torch.arange(T, dtype=F.F64)
    p = torch.stack([0.75 * (i // 6) + far, (i // 3) % 2, i % 3 - 1], -1)
    if B is not None:
        p = torch.stack([p + 0.5 * b for b in range(B)])
    return p.to(F32).to(dev)


def _equal(cache, want):
    for got, w in zip(cache, want):
        assert torch.equal(got.cpu(), w)


# ------------------------------------------------------------- appending
# B, T, H, dh, sections, page, layout
APPEND = [
    (1, 1, 1, 64, (8, 12, 12), 16, "halves"),
    (2, 33, 3, 64, (8, 12, 12), 32, "pairs"),
    (3, 7, 5, 32, (4, 6, 6), 16, "halves"),
    (1, 130, 24, 128, (16, 24, 24), 64, "pairs"),
    (2, 19, 2, 96, (16, 16, 16), 16, "halves"),
    (1, 5, 2, 64, (16, 0, 0), 128, "pairs"),
    (2, 4, 3, 64, (5, 6, 7), 16, "halves"),
    (1, 21, 2, 96, (3, 2, 3), 32, "pairs"),
    (4, 2, 19, 64, (0, 16, 16), 16, "halves"),
    (1, 9, 1, 128, (64, 0, 0), 4096, "halves"),
    (2, 17, 2, 64, (0, 0, 0), 16, "halves"),
]


def _append_case(R, dev, size, dtype, norm, far=0.0, seed=1):
    B, T, H, dh, sections, page, layout = size
    start = [(7 * b) % 40 + 3 for b in range(B)]
    table, pages = _table(dev, seed, B, -(-(max(start) + T) // page))
    cache = _filled(R, dev, seed + 10, pages, page, H, dh)
    k, v = _rand(dev, seed + 2, B, T, H, dh, std=1.5).to(dtype), _rand(dev, seed + 3, B, T, H, dh).to(dtype)
    kw = dict(pos=_positions(dev, T, B, far), sections=sections, freq=R.rope_frequencies(sections), layout=layout,
              k_gain=1 + 0.2 * _rand(dev, seed + 4, dh) if norm else None)
    return cache, k, v, table, _ints(dev, *start), kw


def _appended(cache, k, v, table, start, kw, rows=None):
    turned = F.keys(k, kw["sections"], kw["freq"], kw["layout"], kw["pos"], kw["k_gain"])
    return F.append(cache, turned, v, table, start, rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("size", APPEND)
def test_append(dev, R, size, norm, dtype):
    """Every byte of the pool, written ones and others."""
    cache, k, v, table, start, kw = _append_case(R, dev, size, dtype, norm)
    want = _appended(cache, k, v, table, start, kw)
    assert R.cache_append(cache, k, v, table, start, **kw) is cache
    _equal(cache, want)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_append_far_positions(dev, R, layout):
    case = _append_case(R, dev, (2, 40, 2, 64, (8, 12, 12), 16, layout), BF16, True, far=3e5)
    want = _appended(*case)
    R.cache_append(*case[:5], **case[5])
    _equal(case[0], want)


def test_append_without_positions(dev, R):
    cache, k, v, table, start, kw = _append_case(R, dev, APPEND[1], BF16, False)
    want = F.append(cache, k.float(), v, table, start)
    R.cache_append(cache, k, v, table, start)
    _equal(cache, want)


def test_append_rows_pages_and_ends(dev, R):
    """Padded rows, tokens before the first and past the table's last, entries that are no
    page: dropped, and nothing else is touched."""
    cache, k, v, table, _, kw = _append_case(R, dev, (5, 40, 3, 64, (8, 12, 12), 16, "halves"), BF16, True)
    start = _ints(dev, -5, 0, 30, 2**31 - 20, 7)
    rows = _ints(dev, 40, 0, 99, 40, 13)
    table = table.clone()
    table[0, 1], table[2, 2], table[4, 0] = -1, cache.k.shape[0], 2**31 - 1
    want = _appended(cache, k, v, table, start, kw, rows.cpu())
    R.cache_append(cache, k, v, table, start, rows=rows, **kw)
    _equal(cache, want)
    before = [t.clone() for t in cache]
    R.cache_append(cache, k, v, table, start, rows=_ints(dev, 0, -1, 0, 0, -(2**31)), **kw)
    R.cache_append(cache, k, v, table[:, :0], start, **kw)
    R.cache_append(cache, k[:, :0], v[:, :0], table, start, **dict(kw, pos=kw["pos"][:, :0]))
    _equal(cache, [t.cpu() for t in before])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("order,pad,offset", [((0, 2, 1), 0, 0), ((2, 1, 0), 8, 0), ((1, 0, 2), 3, 1)])
def test_append_strides(dev, R, order, pad, offset, dtype):
    """Rows in any order and off any alignment; pools with tokens outside heads, padded."""
    cache, k, v, table, start, kw = _append_case(R, dev, (2, 21, 3, 64, (8, 12, 12), 16, "halves"), dtype, True)
    k, v = _strided(k, order, pad, offset), _strided(v, order, pad, offset)
    pool = R.KvCache(*(_strided(t, (0, 1, 2), 4 if t.shape[-1] > 2 else 1, 4) for t in cache))
    want = _appended(pool, k, v, table, start, kw)
    R.cache_append(tuple(pool), k, v, table, start, **kw)
    _equal(pool, want)
    shared = v[:, :, :1].expand_as(v)  # one head for all (stride 0)
    want = _appended(pool, k, shared, table, start, kw)
    R.cache_append(pool, k, shared, table, start, **kw)
    _equal(pool, want)


def test_append_non_finite_rows(dev, R):
    """A NaN or an infinity spoils its own blocks (its head where there is a norm)."""
    cache, k, v, table, start, kw = _append_case(R, dev, (1, 6, 2, 96, (8, 4, 4), 16, "halves"), F32, False)
    k[0, 1, 0, 90], k[0, 2, 1, 3], v[0, 3, 0, 40] = math.nan, math.inf, -math.inf
    k[0, 4] = 0.0
    for norm in (None, 1 + 0.2 * _rand(dev, 5, 96)):
        kw["k_gain"] = norm
        want = _appended(cache, k, v, table, start, kw)
        R.cache_append(cache, k, v, table, start, **kw)
        for got, w in zip(cache, want):
            assert torch.equal(got.cpu(), w)


# ------------------------------------------------------------- attention
# B, T, Hq, H, dh, page, lengths
ATTEND = [
    (1, 1, 1, 1, 64, 16, (1,)),
    (1, 1, 12, 12, 64, 64, (864,)),
    (3, 1, 8, 2, 128, 16, (17, 0, 130)),
    (2, 5, 6, 2, 96, 32, (64, 65)),
    (2, 33, 3, 3, 64, 16, (100, 31)),
    (1, 70, 2, 1, 32, 128, (257,)),
    (2, 16, 7, 1, 64, 16, (63, 2)),
    (1, 40, 4, 4, 128, 64, (200,)),
    (1, 2, 2, 2, 64, 256, (5000,)),
    (2, 3, 4, 1, 32, 16, (1500, 40)),
]


def _attend_case(R, dev, size, dtype, seed=1):
    B, T, Hq, H, dh, page, lengths = size
    table, pages = _table(dev, seed, B, max(1, -(-max(lengths) // page)))
    cache = _filled(R, dev, seed + 10, pages, page, H, dh)
    q = _rand(dev, seed + 5, B, T, Hq, dh, std=1.2).to(dtype)
    return q, cache, table, _ints(dev, *lengths)


def _check(R, q, cache, table, lengths, **kw):
    lse = torch.full(q.shape[:3], 7.0, device=q.device)
    out = R.cache_attention(q, cache, table, lengths, lse=lse, **kw)
    kw.pop("out", None), kw.pop("stream", None)
    if kw.get("rows") is not None:
        kw["rows"] = kw["rows"].cpu()
    o, l, eo, el = F.attention(q, cache, table, lengths, **kw)
    F.check(out, o, eo, q.dtype)
    F.check(lse, l, el, F32)
    return out, lse


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", ATTEND)
def test_attention(dev, R, size, causal, dtype):
    _check(R, *_attend_case(R, dev, size, dtype), causal=causal)


# Sizes that choose how rows and tokens go to waves: rows of their own over few tiles of tokens, and
# over more where there are many blocks; parts that one wave or four join; 32 float32 rows a wave
# B, T, Hq, H, dh, page, lengths, dtype
FORMS = [
    (3, 150, 4, 2, 64, 16, (200, 1, 256), BF16),
    (2, 333, 3, 3, 128, 32, (100, 37), BF16),
    (2, 70, 5, 5, 96, 16, (130, 64), F32),
    (1, 65, 7, 1, 32, 16, (50,), F32),
    (8, 1000, 16, 16, 64, 64, tuple(range(700, 300, -50)), BF16),
    (4, 864, 12, 12, 64, 64, (864, 863, 100, 0), F32),
    (1, 1, 2, 2, 64, 64, (20000,), BF16),
    (1, 3, 8, 2, 128, 128, (30011,), F32),
    (2, 2, 6, 3, 32, 16, (9000, 4001), BF16),
    (2, 1366, 24, 24, 64, 64, (2177, 2300), F32),
    (2, 2750, 24, 12, 32, 64, (2177, 2111), F32),
    (300, 1, 2, 1, 32, 16, tuple((7 * i) % 130 for i in range(300)), BF16),
    (2, 4096, 16, 16, 96, 64, (2112, 2200), F32),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", FORMS)
def test_attention_forms(dev, R, size, causal):
    q, cache, table, lengths = _attend_case(R, dev, size[:7], size[7])
    rows = lengths.clamp(max=size[1] - 1)  # the last row of each sequence is padding
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    out = R.cache_attention(q, cache, table, lengths, rows=rows, causal=causal, lse=lse)
    o, l, eo, el = F.attention_whole(q, cache, table, lengths, rows=rows, causal=causal)
    F.check(out, o, eo, q.dtype)
    F.check(lse, l, el, F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_tables_wider_than_the_sequences(dev, R, dtype):
    """Most parts of the tokens hold none, and some sequences are empty."""
    q, cache, table, lengths = _attend_case(R, dev, (3, 2, 4, 2, 64, 16, (5, 0, 700)), dtype)
    wide = torch.full((3, 4000), -1, dtype=I32, device=dev)
    wide[:, :table.shape[1]] = table
    for causal in (False, True):
        _check(R, q, cache, wide, lengths, causal=causal)


def test_whole_and_row_references_agree(dev, R):
    case = _attend_case(R, dev, (2, 21, 6, 2, 64, 16, (90, 30)), F32)
    for causal in (False, True):
        one, all_ = (f(*case, causal=causal, rows=_ints(dev, 21, 13).cpu()) for f in (F.attention, F.attention_whole))
        for a, b in zip(one, all_):
            assert torch.allclose(a, b.cpu(), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 40, 2, 1, 64, 16, (300,)), (2, 90, 3, 3, 128, 16, (120, 77)), (1, 24, 2, 2, 32, 16, (9000,)),
                                  (1, 130, 2, 2, 96, 32, (256,))])
def test_attention_values_past_the_range(dev, R, size, dtype):
    """Values of v past the bf16 range are NaN for the rows that see them, in their dims alone;
    the largest that it holds are values."""
    q, cache, table, lengths = _attend_case(R, dev, size, dtype)
    g = torch.Generator().manual_seed(3)
    dh, n = size[4], size[1]
    for b in range(size[0]):
        for t in torch.randint(max(0, int(lengths[b]) - n), int(lengths[b]), (6,), generator=g).tolist():
            head, block = int(torch.randint(size[3], (1,), generator=g)), int(torch.randint(dh // 32, (1,), generator=g))
            scale = [253, 254, 255][t % 3]
            cache.v_scale[int(table[b, t // size[5]]), t % size[5], head, block] = scale
    v = F.values(cache.v, cache.v_scale)
    far = ~(v.abs() < 2.0 ** 128)  # NaN, or from where bf16 has no value
    clean = R.KvCache(cache.k, cache.k_scale, cache.v.clone(), cache.v_scale.clone())
    codes = torch.stack([cache.v & 15, cache.v >> 4], -1).flatten(-2).cpu()
    codes[far] = 0
    clean.v.copy_(codes[..., 0::2] | codes[..., 1::2] << 4)
    clean.v_scale[clean.v_scale == 255] = 0
    got = R.cache_attention(q, cache, table, lengths, causal=True).cpu()
    o, _, eo, _ = F.attention_whole(q, clean, table, lengths, causal=True)
    bad = torch.zeros_like(got, dtype=torch.bool)
    for b in range(size[0]):
        j = torch.arange(int(lengths[b]))
        first = far[table[b].cpu().long()[j // size[5]], j % size[5]].cumsum(0) > 0  # one by then
        for t in range(n):
            seen = F.seen(int(lengths[b]), 1 << 30, True, n, t)
            if seen:
                bad[b, t] = first[seen - 1].repeat_interleave(size[2] // size[3], 0)
    assert bad.any()
    assert got[bad].isnan().all()
    # sums of values next to the range's end may pass it: a probability is at most 2^8 of the row's last reference
    whole = ~bad & (o.abs().cpu() < 2.0 ** 110)
    if whole.any():
        F.check(got[whole], o.cpu()[whole], eo.cpu()[whole], dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 320])
def test_attention_lengths(dev, R, length, dtype):
    """Around pages, groups of 16 and tiles of 64; more rows than tokens."""
    q, cache, table, _ = _attend_case(R, dev, (1, 19, 2, 2, 64, 16, (320,)), dtype)
    for causal in (False, True):
        _check(R, q, cache, table, _ints(dev, length), causal=causal)


def test_attention_padded_rows_and_lengths_past_the_table(dev, R):
    q, cache, table, _ = _attend_case(R, dev, (5, 20, 4, 2, 64, 16, (80,) * 5), BF16)
    lengths, rows = _ints(dev, 80, 200, -3, 2**31 - 1, 30), _ints(dev, 20, 7, 20, 13, 0)
    for causal in (False, True):
        out, lse = _check(R, q, cache, table, lengths, rows=rows, causal=causal)
        assert (out[4] == 0).all() and (lse[4] == -math.inf).all() and (out[2] == 0).all()
        _check(R, q, cache, table, lengths, rows=_ints(dev, 99, -4, 5, 20, 1), causal=causal)
    assert (R.cache_attention(q, cache, table[:, :0], lengths) == 0).all()
    none = R.new_kv_cache(0, 16, 2, 64, dev)
    assert (R.cache_attention(q, none, table, lengths) == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_without_pages(dev, R, dtype):
    """Entries that are no page leave their tokens out; a sequence of none is empty."""
    q, cache, table, lengths = _attend_case(R, dev, (3, 9, 4, 2, 64, 16, (150, 150, 150)), dtype)
    table = table.clone()
    table[0, 0], table[0, 3], table[0, 9], table[2, 5] = -1, cache.k.shape[0], 2**31 - 1, -(2**31)
    table[1] = -1
    for causal in (False, True):
        out, _ = _check(R, q, cache, table, lengths, causal=causal)
        assert (out[1] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dh", [32, 64, 96, 128])
def test_attention_ignores_what_no_row_sees(dev, R, dh, dtype):
    """NaN keys, values and scales behind the last token, in unused pages and in later tokens
    of a causal chunk; seen ones reach the rows that see them and no other."""
    q, cache, table, lengths = _attend_case(R, dev, (2, 24, 2, 1, dh, 16, (90, 55)), dtype)
    clean = R.cache_attention(q, cache, table, lengths, causal=True)
    dirty = R.KvCache(*(t.clone() for t in cache))
    used = torch.zeros(cache.k.shape[:2], dtype=torch.bool)
    for b in range(2):
        for t in range(int(lengths[b])):
            used[int(table[b, t // 16]), t % 16] = True
    for s in (dirty.k_scale, dirty.v_scale):
        s[~used.to(dev)] = 255
    assert torch.equal(R.cache_attention(q, dirty, table, lengths, causal=True), clean)
    _check(R, q, dirty, table, lengths)
    # token 80 of sequence 0 is row 80 - 90 + 24 = 14's own
    at = int(table[0, 5]), 0
    for s in (dirty.v_scale, dirty.k_scale):
        before = int(s[at[0], at[1], 0, -1])
        s[at[0], at[1], 0, -1] = 255
        got = R.cache_attention(q, dirty, table, lengths, causal=True)
        assert torch.equal(got[0, :14], clean[0, :14]) and torch.equal(got[1], clean[1])
        if s is dirty.v_scale:
            assert got[0, 14:, :, -32:].isnan().all() and not got[0, 14:, :, :-32].isnan().any()
        else:
            assert got[0, 14:].isnan().all()
        s[at[0], at[1], 0, -1] = before


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_extreme_scores(dev, R, dtype):
    """Scores far apart and of any sign and size, growing and falling along the tokens."""
    q, cache, table, lengths = _attend_case(R, dev, (1, 4, 2, 2, 64, 16, (400,)), dtype)
    ramp = torch.exp2(torch.arange(400, dtype=F32, device=dev) / 50.0)
    for order in (ramp, ramp.flip(0)):
        k = (_rand(dev, 9, 400, 2, 64) * order[:, None, None])[None]
        R.cache_append(cache, k, torch.ones_like(k) * _rand(dev, 8, 1, 400, 2, 64), table, _ints(dev, 0))
        for scale in (None, 1.0, 1e-3, 30.0):
            _check(R, q, cache, table, lengths, scale=scale)
    cache.k.zero_(), cache.k_scale.fill_(127)  # all scores zero
    _check(R, q, cache, table, lengths, causal=True)
    q2 = q.clone()
    q2[0, 1, 0, 5] = math.nan
    out = R.cache_attention(q2, cache, table, lengths)
    bad = out.isnan()
    assert bad[0, 1, 0].all() and bad.sum() == 64


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1e-37, 1e-42, 1e-60, 5e-324])
def test_attention_scales_near_and_past_the_smallest_float(dev, R, scale, dtype):
    """Every token that a row sees counts alike, also next to tokens that it does not see."""
    for size in ((2, 5, 6, 2, 96, 32, (64, 65)), (2, 150, 4, 2, 64, 16, (200, 1)), (1, 1, 2, 2, 64, 64, (9001,))):
        for causal in (False, True):
            _check(R, *_attend_case(R, dev, size, dtype), causal=causal, scale=scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("order,pad,offset", [((0, 2, 1), 0, 0), ((2, 1, 0), 8, 0), ((1, 0, 2), 3, 1)])
def test_attention_strides(dev, R, order, pad, offset, dtype):
    q, cache, table, lengths = _attend_case(R, dev, (2, 21, 6, 3, 64, 16, (77, 60)), dtype)
    want = R.cache_attention(q, cache, table, lengths, causal=True)
    sq = _strided(q, order, pad, offset)
    out = _strided(torch.full_like(q, 7.0), order, pad, offset)
    pool = R.KvCache(*(_strided(t, (0, 1, 2), 4 if t.shape[-1] > 2 else 1, 4) for t in cache))
    wide = torch.full((2, 9), -1, dtype=I32, device=dev)
    wide[:, :table.shape[1]] = table
    got = R.cache_attention(sq, pool, wide[:, :table.shape[1]], lengths, causal=True, out=out)
    assert got is out and torch.equal(got, want)
    if pad:
        whole = out.as_strided((out.numel() // 64 * (64 + pad),), (1,), out.storage_offset()).view(-1, 64 + pad)
        assert (whole[:, 64:] == 0).all()
    shared = q[:, :, :1].expand_as(q)
    _check(R, shared, cache, table, lengths)


def test_attention_offsets_past_32_bits(dev, R):
    """Pages more than 4 GB apart."""
    far = (1 << 32) + 4096
    buf = torch.zeros(2 * far + (1 << 20), dtype=U8, device=dev)
    small = _filled(R, dev, 3, 3, 16, 2, 64)
    pool = []
    for i, t in enumerate(small):
        n = t.shape[-1]
        view = buf[i * 65536:].as_strided((3, 16, 2, n), (far, n, 16 * n, 1))
        view.copy_(t)
        pool.append(view)
    q, table = _rand(dev, 5, 1, 3, 2, 64).to(BF16), _ints(dev, 2, 0, 1).view(1, 3)
    want = R.cache_attention(q, small, table, _ints(dev, 45))
    assert torch.equal(R.cache_attention(q, tuple(pool), table, _ints(dev, 45)), want)
    k, v = _rand(dev, 6, 1, 9, 2, 64), _rand(dev, 7, 1, 9, 2, 64)
    for c in (small, tuple(pool)):
        R.cache_append(c, k, v, table, _ints(dev, 12))
    for a, b in zip(small, pool):
        assert torch.equal(a, b)


def test_results_of_two_caches_join(dev, R):
    """Attention over two parts of the tokens joins, by lse, to that over both."""
    q, cache, table, lengths = _attend_case(R, dev, (2, 6, 4, 2, 64, 16, (192, 192)), F32)
    whole, lse = _check(R, q, cache, table, lengths)
    parts = []
    for t in (table[:, :5], table[:, 5:]):
        l = torch.empty(2, 6, 4, device=dev)
        parts.append((R.cache_attention(q, cache, t, _ints(dev, *[16 * t.shape[1]] * 2), lse=l), l))
    w = torch.softmax(torch.stack([l for _, l in parts]).double(), 0)
    joined = sum(o.double() * x[..., None] for (o, _), x in zip(parts, w))
    _, _, bound, _ = F.attention(q, cache, table, lengths)
    assert ((joined - whole.double()).abs().cpu() <= 4 * bound + 2.0 ** -22 * whole.abs().cpu()).all()


# ------------------------------------------------------------- together
def _steps(R, dev, dtype=BF16, seed=1, B=2, H=3, dh=64, page=16):
    """A layer's history: a prompt, then single rows."""
    sections = (8, 12, 12)
    table, pages = _table(dev, seed, B, 6)
    return dict(cache=R.new_kv_cache(pages, page, H, dh, dev), table=table, sections=sections,
                freq=R.rope_frequencies(sections), gain=1 + 0.1 * _rand(dev, seed + 1, dh),
                q=_rand(dev, seed + 2, B, 50, 2 * H, dh).to(dtype), k=_rand(dev, seed + 3, B, 50, H, dh).to(dtype),
                v=_rand(dev, seed + 4, B, 50, H, dh).to(dtype), pos=_positions(dev, 50), B=B)


def _run_rows(R, st, dev, lo, hi, cache=None, **kw):
    cut = slice(lo, hi)
    cache = st["cache"] if cache is None else cache
    R.cache_append(cache, st["k"][:, cut], st["v"][:, cut], st["table"], _ints(dev, *[lo] * st["B"]), pos=st["pos"][cut],
                   sections=st["sections"], freq=st["freq"], k_gain=st["gain"])
    return R.cache_attention(st["q"][:, cut], cache, st["table"], _ints(dev, *[hi] * st["B"]), causal=True, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_and_single_rows(dev, R, dtype):
    """A prompt in one call and row after row: the same cache, bit for bit, and attention
    within both results' bounds of the definition."""
    st = _steps(R, dev, dtype)
    whole = _run_rows(R, st, dev, 0, 50)
    keys = F.keys(st["k"], st["sections"], st["freq"], "halves", st["pos"], st["gain"])
    empty = [torch.zeros_like(t).cpu() for t in st["cache"]]
    _equal(st["cache"], F.append(empty, keys, st["v"], st["table"], torch.zeros(2, dtype=I32)))
    o, _, eo, _ = F.attention(st["q"], st["cache"], st["table"], _ints(dev, 50, 50), causal=True)
    F.check(whole, o, eo, dtype)
    rows = R.new_kv_cache(*st["cache"].k.shape[:3], 64, dev)
    got = [_run_rows(R, st, dev, 0, 30, rows)] + [_run_rows(R, st, dev, t, t + 1, rows) for t in range(30, 50)]
    _equal(rows, [t.cpu() for t in st["cache"]])
    F.check(torch.cat(got, 1), o, eo, dtype)


def test_layer_in_four_bits(dev, R):
    """The operators of a layer in their order: norm, 4-bit blocks, QKV product, rotation of q,
    append, attention, blocks, output product."""
    B, T, D, H = 2, 40, 256, 4
    dh, sections = D // H, (8, 12, 12)
    freq, pos = R.rope_frequencies(sections), _positions(dev, T)
    wqkv, wo = (R.quantize_fp4(_rand(dev, s, n, D, std=0.06)) for s, n in ((1, 3 * D), (2, D)))
    g = 1 + 0.1 * _rand(dev, 3, dh)
    h = _rand(dev, 4, B, T, D)
    u = R.norm_residual(h, u_dtype=BF16)[1]
    x = R.quantize_fp4(u.view(B * T, D))
    q, k, v = R.matmul_fp4(*x, *wqkv).view(B, T, 3, H, dh).unbind(2)
    q = R.rope(q, None, pos, sections, freq, q_gain=g)[0]
    table, pages = _table(dev, 5, B, 3)
    cache = R.new_kv_cache(pages, 16, H, dh, dev)
    R.cache_append(cache, k, v, table, _ints(dev, 0, 0), pos=pos, sections=sections, freq=freq, k_gain=g)
    o = R.cache_attention(q, cache, table, _ints(dev, T, T))
    y = R.matmul_fp4(*R.quantize_fp4(o.view(B * T, D)), *wo)
    # each step against its own definition on the inputs it got
    F.same(R.dequantize_fp4(*x, dtype=F32), F.values(*F.quantize(u.view(B * T, D))))
    F.check(torch.stack([t for t in (k, v)]), *map(torch.stack, zip(*[
        tuple(t.view(B, T, 3, H, dh)[:, :, i] for t in F.matmul(*x, *wqkv)) for i in (1, 2)])), BF16)
    keys = F.keys(k, sections, freq, "halves", pos, g)
    _equal(cache, F.append([torch.zeros_like(t).cpu() for t in cache], keys, v, table, torch.zeros(B, dtype=I32)))
    ref, _, err, _ = F.attention(q, cache, table, _ints(dev, T, T))
    F.check(o, ref, err, BF16)
    F.check(y, *F.matmul(*R.quantize_fp4(o.view(B * T, D)), *wo), BF16)


def _long(R, dev, seed, length=3000):
    """Attention whose tokens are split over blocks, into a buffer of its own."""
    q, cache, table, lengths = _attend_case(R, dev, (1, 2, 2, 2, 64, 64, (length,)), BF16, seed)
    return dict(q=q, cache=cache, table=table, lengths=lengths, out=torch.empty_like(q))


def _attend(R, st, **kw):
    return R.cache_attention(st["q"], st["cache"], st["table"], st["lengths"], out=st["out"], **kw)


def test_split_tokens_in_overlapping_calls(dev, R):
    """Calls on two streams at once do not share their parts' memory."""
    a, b = _long(R, dev, 1), _long(R, dev, 50)
    want = [_attend(R, st).clone() for st in (a, b)]
    streams = [torch.cuda.Stream(dev) for _ in range(2)]
    torch.cuda.synchronize()
    for st in (a, b):
        st["out"].zero_()
    torch.cuda.synchronize()
    for _ in range(30):
        for st, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                _attend(R, st)
    torch.cuda.synchronize()
    for st, w in zip((a, b), want):
        assert torch.equal(st["out"], w)
    s = torch.cuda.Stream(dev)
    s.wait_stream(torch.cuda.current_stream())
    got = R.cache_attention(a["q"], a["cache"], a["table"], a["lengths"], stream=s)
    s.synchronize()
    assert torch.equal(got, want[0])


def test_results_belong_to_the_given_stream(dev, R):
    """Memory that the current stream has freed but still writes is no result (or
    workspace) of another stream's call."""
    x = _rand(dev, 1, 4096, 512)
    q, s = R.quantize_fp4(x)
    w = R.quantize_fp4(_rand(dev, 2, 512, 512))
    st = _long(R, dev, 3)
    calls = (lambda t: R.quantize_fp4(x, stream=t), lambda t: (R.dequantize_fp4(q, s, stream=t),),
             lambda t: (R.matmul_fp4(q, s, *w, out_dtype=F32, stream=t),), lambda t: R.matmul_fp4(q, s, *w, out_dtype=U8, stream=t),
             lambda t: (R.cache_attention(st["q"], st["cache"], st["table"], st["lengths"], stream=t),))
    side, slow = torch.cuda.Stream(dev), torch.empty(1 << 28, device=dev)
    for call in calls:
        want = [t.clone() for t in call(None)]
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        junk = [torch.empty_like(t) for t in call(None)] + [torch.empty(1 << 20, device=dev)]
        for _ in range(20):
            slow.zero_()
        for t in junk:
            t.fill_(1)
        del junk, t
        got = call(side)
        torch.cuda.synchronize()
        for g, t in zip(got, want):
            assert torch.equal(g, t)


def test_captured_and_replayed(dev, R):
    """A decode step (quantise, product, append, attention over split tokens) in a graph, its
    inputs changed in place, with the program's eager work between the replays; two graphs
    of one memory pool, replayed in turn."""
    st = _long(R, dev, 1)
    w = R.quantize_fp4(_rand(dev, 2, 128, 128))
    x, start = _rand(dev, 3, 2, 128).to(BF16), _ints(dev, 2990)
    k = torch.empty(1, 2, 2, 64, dtype=BF16, device=dev)
    freq, pos = R.rope_frequencies((8, 12, 12)), _positions(dev, 2)

    def step():
        y = R.matmul_fp4(*R.quantize_fp4(x), *w)
        k.copy_(y.view(1, 2, 2, 64))
        R.cache_append(st["cache"], k, k, st["table"], start, pos=pos, sections=(8, 12, 12), freq=freq)
        return _attend(R, st, causal=True)

    other = _long(R, dev, 50, 2000)
    step(), _attend(R, other)
    torch.cuda.synchronize()
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        step()
    with torch.cuda.graph(second, pool=first.pool()):
        _attend(R, other)
    for seed in range(4):
        x.copy_(_rand(dev, 100 + seed, 2, 128))
        start.fill_(2980 + seed)
        st["lengths"].fill_(2982 + seed)
        other["lengths"].fill_(1900 + seed)
        first.replay(), second.replay()
        torch.cuda.synchronize()
        got = st["out"].clone(), other["out"].clone(), [t.clone() for t in st["cache"]]
        assert torch.equal(step(), got[0]) and torch.equal(_attend(R, other), got[1])
        _equal(st["cache"], [t.cpu() for t in got[2]])


def test_same_bits_twice(dev, R):
    st = _long(R, dev, 5)
    first = _attend(R, st).clone()
    for _ in range(3):
        assert torch.equal(_attend(R, st), first)


# ------------------------------------------------------------- refusals in the binding
def test_binding_refusals(dev, R):
    q, cache, table, lengths = _attend_case(R, dev, (2, 3, 4, 2, 64, 16, (40, 20)), BF16)
    for bad in (dict(q=q[0]), dict(q=q.half()), dict(q=q.cpu()), dict(q=q[:, :, :3]), dict(q=q[..., :32]), dict(cache=cache[:3]),
                dict(cache=list(cache)), dict(cache=(cache.k[0], *cache[1:])), dict(cache=(None, *cache[1:])), dict(cache=(*cache[:3], None)),
                dict(cache=(*cache[:3], cache.v_scale.cpu())), dict(cache=(cache.k, cache.k_scale, cache.v.flip(3)[:, :, :, ::2], cache.v_scale)), dict(cache=(cache.k, cache.k_scale[..., :1], *cache[2:])),
                dict(cache=(cache.k.int(), *cache[1:])), dict(table=table.long()), dict(table=table[:1]), dict(table=table[0]),
                dict(lengths=lengths[:1]), dict(lengths=lengths.long()), dict(rows=lengths.float()), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=math.nan), dict(out=torch.empty_like(q)[:1]), dict(out=q), dict(out=q.float()),
                dict(out=q[:, :, :1].expand_as(q)), dict(lse=torch.empty(2, 4, 3, device=dev)),
                dict(q=q.clone().requires_grad_())):
        kw = dict(q=q, cache=cache, table=table, lengths=lengths)
        kw.update(bad)
        with pytest.raises(R.WamError):
            R.cache_attention(kw.pop("q"), kw.pop("cache"), kw.pop("table"), kw.pop("lengths"), **kw)
    k, start = _rand(dev, 1, 2, 3, 2, 64).to(BF16), _ints(dev, 0, 5)
    pos, freq = _positions(dev, 3), R.rope_frequencies((8, 12, 12))
    for bad in (dict(v=k.float()), dict(v=k[:1]), dict(k=k[0]), dict(k=k[:, :, :1], v=k[:, :, :1]), dict(start=start[:1]),
                dict(start=start.long()), dict(rows=start.long()), dict(pos=None), dict(pos=pos.double()), dict(pos=pos[:2]),
                dict(freq=freq[:-1]), dict(sections=(8, 24)), dict(sections=(20, 12, 1), freq=np.ones(33)), dict(layout="x"),
                dict(k_gain=torch.ones(63, device=dev)), dict(k_gain=torch.ones(64, device=dev), eps=-1.0),
                dict(cache=(cache.k[:, :, :1].expand_as(cache.k), *cache[1:]))):
        kw = dict(cache=cache, k=k, v=k, table=table, start=start, pos=pos, freq=freq, sections=(8, 12, 12))
        kw.update(bad)
        with pytest.raises(R.WamError):
            R.cache_append(kw.pop("cache"), kw.pop("k"), kw.pop("v"), kw.pop("table"), kw.pop("start"), **kw)
    with pytest.raises(R.WamError):
        R.new_kv_cache(4, 16, 2, 48, dev)
    odd = R.new_kv_cache(4, 24, 2, 64, dev)
    with pytest.raises(R.WamError, match="power of two"):
        R.cache_attention(q, odd, table, lengths)


def test_empty_shapes(dev, R):
    q, cache, table, lengths = _attend_case(R, dev, (2, 3, 4, 2, 64, 16, (40, 20)), BF16)
    assert R.cache_attention(q[:, :0], cache, table, lengths).shape == (2, 0, 4, 64)
    assert R.cache_attention(q[:0], cache, table[:0], lengths[:0]).shape == (0, 3, 4, 64)
