"""Sizes past what a launch or a 32-bit column number can hold are refused, and those just below are not (no GPU: every
call here fails a check, the last of them that of its pointers)."""
import pytest

from paper_2607_18631_amd import moe
from test_abi_serving import BASE, UNSUPPORTED, INVALID, decode, norm, norm_bwd, refused

MANY = BASE.replace(T=64, d=64, E=1024, E_local=1024, top_k=16)


@pytest.mark.parametrize("change", [dict(F=(1 << 20) - 8), dict(d=(1 << 20) - 8, F=64), dict(F=1048568, F_shared=64)])
def test_few_token_layer_of_too_many_workgroups(change):
    sh = MANY.replace(**change)
    refused(decode(sh, x=None), UNSUPPORTED, "2^24 workgroups")
    with pytest.raises(moe.MoEError, match="2\\^24 workgroups"):
        moe.workspace_size(sh, moe.MOE_WS_DECODE)


@pytest.mark.parametrize("change", [dict(F=1 << 19), dict(d=1 << 19), dict(F=(1 << 20) - 8, E_local=512),
                                    dict(F=(1 << 20) - 8, T=32, F_shared=(1 << 20) - 8)])
def test_few_token_layer_just_below(change):
    refused(decode(MANY.replace(**change), x=None), INVALID, "x is NULL")


@pytest.mark.parametrize("d", [(1 << 31) - 24, (1 << 31) - 16, (1 << 31) - 8])
def test_norm_of_too_long_rows(d):
    refused(norm(d=d, x=None, q=None, s=None), UNSUPPORTED, "> 2^31 - 32")
    refused(norm_bwd(d=d, dy=None), UNSUPPORTED, "> 2^31 - 32")
    with pytest.raises(moe.MoEError, match="2\\^31 - 32"):
        moe.add_rmsnorm_workspace_size(1, d)


def test_norm_of_the_longest_rows():
    d = (1 << 31) - 32
    refused(norm(d=d, x=None), INVALID, "x is NULL")
    refused(norm_bwd(d=d, dy=None), INVALID, "dy is NULL")
    assert moe.add_rmsnorm_workspace_size(1, d) >= 4 * d
