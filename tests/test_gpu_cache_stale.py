"""Attention over a 4-bit cache that an older history has left full of NaN, and results in
buffers with gaps: every way that rows and tokens go to waves."""
import pytest
import torch

from gpu_common import device
from test_gpu_cache import ATTEND, BF16, F32, FORMS, _attend_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.fixture(scope="module")
def R():
    from paper_2609_34608_amd import runtime
    return runtime


def _used(table, lengths, pages, page):
    """Places that hold a token of some sequence."""
    used = torch.zeros(pages * page, dtype=torch.bool, device=table.device)
    for row, n in zip(table.long(), lengths.tolist()):
        t = torch.arange(min(n, len(row) * page), device=table.device)
        used[row[t // page] * page + t % page] = True
    return used.view(pages, page)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("size", [(*s, t) for s in ATTEND for t in (F32, BF16)] + FORMS)
def test_stale_places_hold_nan(dev, R, size, causal):
    """NaN keys and values in unused pages and behind each sequence's last token, in every
    page size: not a bit of a result changes.  The logarithms go to a buffer whose rows and
    samples lie apart, and the gaps stay as they were."""
    q, cache, table, lengths = _attend_case(R, dev, size[:7], size[7])
    B, T, Hq = q.shape[:3]
    rows = lengths.clamp(max=T)  # fewer where the sequence is shorter
    want_lse = torch.full((B, T, Hq), 7.0, device=dev)
    want = R.cache_attention(q, cache, table, lengths, rows=rows, causal=causal, lse=want_lse)
    assert not want.isnan().any()
    stale = ~_used(table, lengths, *cache.k.shape[:2])
    assert stale.any()
    for s in (cache.k_scale, cache.v_scale):
        s[stale] = 255
    wide = torch.full((B, T + 1, Hq + 3), 7.0, device=dev)
    got = R.cache_attention(q, cache, table, lengths, rows=rows, causal=causal, lse=wide[:, :T, 2:Hq + 2])
    assert torch.equal(got, want) and torch.equal(wide[:, :T, 2:Hq + 2], want_lse)
    wide[:, :T, 2:Hq + 2] = 7
    assert (wide == 7).all()
