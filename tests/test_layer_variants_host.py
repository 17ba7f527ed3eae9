"""The model's layer variants without a GPU: the 8-bit mode's configurations and the
refusals of a null handle."""
import ctypes as C

import pytest

from paper_2609_34608_amd import _lib as L
from paper_2609_34608_amd import runtime as R


def _cfg(dtype, **kw):
    base = dict(B=1, L=2, D=128, H=2, F=512, Nv=64, Cv=16, Na=16, A=7, No=8, Co=16, dtype=dtype)
    base.update(kw)
    return R.make_config(**base)


def test_fp8_mode_is_accepted_and_smaller():
    lib = L.lib()
    f8, bf = _cfg("fp8"), _cfg("bf16")
    assert f8.dtype == L.WAM_FP8
    assert lib.wam_host_weight_count(C.byref(f8)) == lib.wam_host_weight_count(C.byref(bf)) > 0
    assert 0 < lib.wam_weight_bytes(C.byref(f8)) < lib.wam_weight_bytes(C.byref(bf))
    assert lib.wam_workspace_bytes(C.byref(f8)) > 0


@pytest.mark.parametrize("bad", [dict(H=4), dict(F=192), dict(D=100), dict(B=0)])
def test_fp8_mode_has_the_limits_of_bf16(bad):
    lib = L.lib()
    assert lib.wam_workspace_bytes(C.byref(_cfg("fp8", **bad))) == lib.wam_workspace_bytes(C.byref(_cfg("bf16", **bad))) == 0


def test_null_handle():
    lib = L.lib()
    assert lib.wam_set_rotary(None, None) == L.WAM_E_ARG
    assert lib.wam_set_post_norm(None, None) == L.WAM_E_ARG
