"""Refusals of buffers that a call on the cache would write twice (CPU: every check comes
before any device work)."""
import pytest

from paper_2609_34608_amd import _lib as L
from test_fp4_refusals import P, _append, _attend, _i64, _refused

KEYS, KEY_SCALES, VALUES, VALUE_SCALES = P, P + 16384, P + 32768, P + 49152


@pytest.mark.parametrize("kw", [
    dict(cache__v=KEYS), dict(cache__v_scale=KEY_SCALES), dict(cache__k_scale=KEYS), dict(cache__v_scale=KEYS),
    dict(cache__k_scale=VALUES), dict(cache__v_scale=VALUES)])
def test_append_refuses_one_buffer_for_two_arrays(kw):
    a, _ = _append(**kw)
    _refused("wam_cache_append", a, L.WAM_E_ARG, "different buffers")


@pytest.mark.parametrize("at", [P, P + 65536])
def test_attention_refuses_logarithms_in_another_buffer(at):
    _refused("wam_cache_attention", _attend(lse=at, lse_stride=_i64(16, 4, 1)), L.WAM_E_ARG, "lse must be")
