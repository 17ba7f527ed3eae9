"""Attention over the 4-bit cache where values, keys and scores come next to the ends of
their types' ranges or pass them, against float64 (fp4_ref)."""
import math

import pytest
import torch

import fp4_ref as F
from gpu_common import device
from test_gpu_cache import BF16, F32, _attend_case, _ints, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.fixture(scope="module")
def R():
    from paper_2609_34608_amd import runtime
    return runtime


# B, T, Hq, H, dh, page, lengths: waves that share tokens, waves with rows of their own, tokens split
# over blocks (parts that one wave joins, and four), 32 and 64 rows a wave
SIZES = [
    (1, 40, 2, 1, 64, 16, (300,)),
    (2, 90, 3, 3, 128, 16, (120, 177)),
    (1, 24, 2, 2, 32, 16, (9000,)),
    (1, 130, 2, 2, 96, 32, (256,)),
    (3, 3, 4, 2, 64, 64, (3000, 200, 2500)),
    (1, 2, 2, 2, 128, 64, (20000,)),
]


def _place(table, size, b, t):
    return int(table[b, t // size[5]]), t % size[5]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_values_past_the_range_without_a_mask(dev, R, size, dtype):
    """A value of v past the bf16 range is NaN, not infinite, for every row that sees it, in
    its dim alone; the others are as if it were zero.  Rows that see nothing stay 0."""
    q, cache, table, lengths = _attend_case(R, dev, size, dtype)
    B, T, Hq, H, dh = size[:5]
    g = torch.Generator().manual_seed(3)
    bad = torch.zeros(B, T, Hq, dh, dtype=torch.bool)
    clean = R.KvCache(cache.k, cache.k_scale, cache.v.clone(), cache.v_scale.clone())
    for b in range(B):
        for i, t in enumerate(torch.randperm(int(lengths[b]), generator=g)[:4].tolist()):
            h, block, e = (int(torch.randint(n, (1,), generator=g)) for n in (H, dh // 32, 32))
            at = *_place(table, size, b, t), h
            half = slice(block * 16, block * 16 + 16)
            for c in (cache, clean):
                c.v[at][half], c.v_scale[at][block] = 0, 0
            cache.v_scale[at][block] = (253, 254, 255, 254)[i]
            cache.v[at][half][e // 2] = (7 if i % 2 else 15) << 4 * (e % 2)  # 6 or -6
            dims = slice(block * 32, block * 32 + 32) if i == 2 else block * 32 + e
            bad[b, :, h * Hq // H:(h + 1) * Hq // H, dims] = True
    rows = torch.full((B,), T - 1)
    bad[:, T - 1] = False
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, rows=rows.to(torch.int32).to(dev), lse=lse).cpu()
    o, l, eo, el = (x.cpu() for x in F.attention_whole(q, clean, table, lengths, rows=rows))
    F.check(got, torch.where(bad, math.nan, o), eo, dtype)
    F.check(lse, l, el, F32)


def _scores_of_one_dim(R, dev, size, dtype, levels, e):
    """A cache whose keys are zero but in dim 0, where they are 2^e times a value of levels, in
    random order, and random values."""
    q, cache, table, lengths = _attend_case(R, dev, size, dtype)
    B, _, _, H, dh, page = size[:6]
    g = torch.Generator().manual_seed(4)
    k = torch.zeros(B, table.shape[1] * page, H, dh)
    k[..., 0] = torch.tensor(levels)[torch.randint(len(levels), k.shape[:3], generator=g)] * 2.0 ** e
    v = _rand(dev, 8, *k.shape)
    R.cache_append(cache, k.to(dev), v, table, _ints(dev, *[0] * B))
    q.zero_()
    return q, cache, table, lengths


def _tied(size, dtype, values):
    """Bound of attention whose rows' tokens have weights of 0 or exactly 1: the float32 sums
    over n tokens, as in fp4_ref.attention."""
    return 2.0 ** -22 * (max(size[6]) / 32 + 16) * 2 * float(values.nan_to_num().abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1e7, 3e9, 1e13, 1e28])
@pytest.mark.parametrize("size", SIZES)
def test_scores_whose_steps_pass_the_exponent(dev, R, size, scale, dtype):
    """From scores of 2^32 on a step of float32 is more than exp's range: the tokens of the
    largest score share a row evenly all the same, and the row's sum is theirs.  Beside such
    rows there are ordinary ones and ones whose scores are all zero.

    The products with q are exact or, for tokens of one score, round alike, and scores differ
    by half the largest at least; the logarithm takes the rounding of the scaled score
    (2^-22 a matrix step, four roundings of 2^-24), which leaves no doubt about the weights."""
    q, cache, table, lengths = _scores_of_one_dim(R, dev, size, dtype, (6.0, 3.0, 1.0, -3.0, -6.0, 0.5), 0)
    B, T, Hq, _, dh = size[:5]
    lead = (1 + torch.rand(B, T, Hq, generator=torch.Generator().manual_seed(5))).to(dev)
    kind = (torch.arange(T, device=dev)[:, None] + torch.arange(Hq, device=dev)) % 5
    small, none = kind == 3, kind == 4
    lead = torch.where(kind == 1, -lead, lead)
    lead = torch.where(none, 0.0, torch.where(small, lead / scale, lead))
    q[..., 0] = lead.to(dtype)
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    for causal in (False, True):
        got = R.cache_attention(q, cache, table, lengths, causal=causal, scale=scale, lse=lse)
        o, l, eo, el = F.attention_whole(q, cache, table, lengths, causal=causal, scale=scale)
        far = ~(small | none).expand(B, T, Hq)
        eo[far] = _tied(size, dtype, F.values(cache.v, cache.v_scale))
        el[far] = 2.0 ** -22 * (dh / 32 + 2) * l[far].nan_to_num(neginf=0).abs()
        F.check(got, o, eo, dtype)
        F.check(lse, l, el, F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_scores_near_the_lowest_float(dev, R, size, dtype):
    """A row whose scores are the lowest that float32 holds still sees its tokens: -2^127 times
    1.3 log2(e) is -3.19e38, of -3.40e38."""
    q, cache, table, lengths = _scores_of_one_dim(R, dev, size, dtype, (1.0,), 0)
    q[..., 0] = -2.0 ** 127
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, scale=1.3, lse=lse)
    o, l, _, _ = F.attention_whole(q, cache, table, lengths, scale=1.3)
    F.check(got, o, torch.full_like(o, _tied(size, dtype, F.values(cache.v, cache.v_scale))), dtype)
    F.check(lse, l, 2.0 ** -22 * (size[4] / 32 + 2) * l.abs(), F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_keys_past_the_range(dev, R, size, causal, dtype):
    """A value of k past the bf16 range is an infinity: where the row's q has the other sign
    the token has no weight, and the row is what it is without the token; where it has the
    same sign or is zero the score is infinite or NaN, and the row NaN."""
    q, cache, table, lengths = _attend_case(R, dev, size, dtype)
    B, T, Hq, H, dh, page = size[:6]
    one, rest = dh - 5, slice(dh // 2 - 16, dh // 2)
    kind = (torch.arange(T, device=dev)[:, None] + torch.arange(Hq, device=dev)) % 4
    x = q[..., one].float().abs() + 0.25
    x = torch.where(kind == 1, 0.5, x)  # exact in bf16
    x = torch.where(kind == 2, -x, x)
    q[..., one] = torch.where(kind == 3, 0.0, x).to(dtype)
    without = table.clone()
    for b in range(B):
        for p in (0, (int(lengths[b]) - T) // page - 1):  # pages that every row sees
            at = int(table[b, p])
            without[b, p] = -1
            cache.k[at, ..., rest] = 0
            cache.k[at, ..., one // 2] = 0xf << 4 * (one % 2)  # -6
            cache.k_scale[at, ..., -1] = torch.tensor([253, 254])[torch.arange(page) % 2][:, None].to(dev)
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, causal=causal, lse=lse)
    o, l, eo, el = F.attention_whole(q, cache, without, lengths, causal=causal)
    bad = (kind >= 2).expand(B, T, Hq)
    o[bad], l[bad] = math.nan, math.nan
    F.check(got, o, eo, dtype)
    F.check(lse, l, el, F32)


@pytest.mark.parametrize("byte", [0, 2])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_queries_past_the_bf16_range(dev, R, size, causal, byte):
    """The largest float32 values, which bf16 rounds to an infinity, against the smallest keys,
    subnormal ones too; and an infinite q, which makes its own row NaN."""
    q, cache, table, lengths = _attend_case(R, dev, size, F32)
    g = torch.Generator().manual_seed(6)
    q.copy_(torch.where(torch.rand(q.shape, generator=g) < 0.5, -1.0, 1.0)
            * (3.39e38 + 1e36 * torch.rand(q.shape, generator=g)))
    cache.k_scale.fill_(byte)
    q[:, -1, -1, 3] = math.inf
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, causal=causal, lse=lse)
    q[:, -1, -1, 3] = 0.0
    o, l, eo, el = F.attention_whole(q, cache, table, lengths, causal=causal)
    o[:, -1, -1], l[:, -1, -1] = math.nan, math.nan
    F.check(got, o, eo, F32)
    F.check(lse, l, el, F32)


@pytest.mark.parametrize("size", SIZES)
def test_queries_next_to_the_smallest(dev, R, size):
    """float32 q whose later bits are subnormal in bf16 lose none down to its smallest, 2^-133."""
    q, cache, table, lengths = _attend_case(R, dev, size, F32)
    q.copy_(torch.round(q * 2.0 ** 18) * 2.0 ** -133)
    cache.k_scale.copy_((cache.k_scale.int() + 115).to(torch.uint8))
    lse = torch.full(q.shape[:3], 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, lse=lse)
    o, l, eo, el = F.attention_whole(q, cache, table, lengths)
    F.check(got, o, eo, F32)
    F.check(lse, l, el, F32)
