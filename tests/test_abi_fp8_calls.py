"""C-ABI and binding checks of the 8-bit layer that need no GPU, beside those of
tests/test_abi_fp8.py."""
import ctypes as C

import pytest


from paper_2604_07725_amd import sevo

F = 1 << 20   # a pointer that no check reads


@pytest.mark.parametrize("kw,status", [
    (dict(clear_unlisted=2), sevo.INVALID_ARGUMENT), (dict(clear_unlisted=-1), sevo.INVALID_ARGUMENT),
    (dict(clear_unlisted=1, n=0), sevo.OK)])
def test_moe_linear_fp8_refuses(kw, status):
    a = dict(n=64, top_k=8, n_experts=128, n_out=128, k=256, down=0, ldx=256, lds=64, x=F,
             x_scales=F, w=F, w_scales=F, lists=F, out=F)
    a.update(kw)
    assert sevo.lib().sevo_moe_linear_fp8(C.byref(sevo.MoeLinearFp8Args(**a)), None) == status
