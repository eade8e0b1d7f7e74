"""C-ABI and binding checks of the 8-bit layer that need no GPU, beside those of
tests/test_abi_fp8.py."""
import ctypes as C

import pytest
import torch

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


def test_lists_of_other_sizes_are_refused():
    """Lists in a buffer too small for their sizes are refused before the kernels
    follow them out of it."""
    f8 = torch.float8_e4m3fn
    x, xs = torch.zeros(64, 256).to(f8), torch.zeros(2, 64)
    w, ws = torch.zeros(3, 64, 256).to(f8), torch.zeros(3, 1, 2)
    need = sevo.sevo_moe_lists_bytes(64, 2, 3)
    for size in (0, 256, need - 1):
        with pytest.raises(ValueError, match="lists"):
            sevo.sevo_moe_linear_fp8(x, xs, w, ws, sevo.MoeLists(64, 2, 3, torch.zeros(size, dtype=torch.uint8)))
    with pytest.raises(ValueError, match="GPU"):      # the size will do
        sevo.sevo_moe_linear_fp8(x, xs, w, ws, sevo.MoeLists(64, 2, 3, torch.zeros(need, dtype=torch.uint8)))


def test_one_row_of_any_buffer():
    """One token out of a buffer whose rows are no multiple of 16 bytes apart, or far
    apart: the stride between rows that are not there is not refused."""
    f8, bf = torch.float8_e4m3fn, torch.bfloat16
    x = torch.zeros(3, 264).to(f8)[:1, :256]
    assert sevo._ld(x, 1, 256) == 256
    assert sevo._ld(torch.zeros(256, 1).t(), 1, 256) == 256
    assert sevo._ld(torch.zeros(3, 264)[:, :256], 3, 256) == 264
    assert sevo._ld(torch.zeros(1, 1 << 24, dtype=bf)[:, :512], 1, 512) == 512


def test_sizes_near_the_end_of_int32():
    """Refused, or planned, without an int32 that overflows (undefined, so that the
    host-sanitized build ends there)."""
    L = sevo.lib()
    top = 2 ** 31
    for m, n_out, k in ((top - 1, 64, 128), (top - 1, 4096, 25600), (1 << 29, 64, 128), (4, top - 64, 128),
                        (4, (1 << 30) + 64, 128)):
        assert L.sevo_linear_fp8_workspace_bytes(m, n_out, k) == 0
    L.sevo_linear_fp8_workspace_bytes((1 << 29) - 1, 1 << 30, 128)
    a = dict(m=4, n_out=top - 64, k=128, out_type=sevo.BF16, ldx=128, lds=4, ldo=top, x=F, x_scales=F,
             w=F, w_scales=F, out=F, workspace=F, workspace_bytes=1 << 40)
    assert L.sevo_linear_fp8(C.byref(sevo.LinearFp8Args(**a)), None) == sevo.UNSUPPORTED
    a = dict(n=4, top_k=2, n_experts=8, n_out=top - 64, k=128, down=0, ldx=128, lds=4, x=F, x_scales=F,
             w=F, w_scales=F, lists=F, out=F)
    assert L.sevo_moe_linear_fp8(C.byref(sevo.MoeLinearFp8Args(**a)), None) == sevo.UNSUPPORTED


def test_rows_of_more_than_a_launch():
    """Calls of 2^32 threads and more are refused on the host, whatever the launch
    would do with them."""
    L = sevo.lib()
    for rows, cols in ((1 << 26, 512), (1 << 24, 2048), (1 << 23, 4096), (1 << 22, 32768)):
        a = dict(rows=rows, cols=cols, n_partials=0, eps=1e-6, x=F, gain=F, out=F, scales=F)
        assert L.sevo_add_rmsnorm_fp8(C.byref(sevo.AddRmsnormFp8Args(**a)), None) == sevo.UNSUPPORTED
        a.update(rows=rows - 1, x=0)                                   # one fewer: the next check
        assert L.sevo_add_rmsnorm_fp8(C.byref(sevo.AddRmsnormFp8Args(**a)), None) == sevo.INVALID_ARGUMENT
    for m, k in ((1 << 28, 512), (1 << 24, 8192)):
        assert L.sevo_quantize_fp8(F, k, m, k, 0, F, F, None) == sevo.UNSUPPORTED
        assert L.sevo_quantize_fp8(0, k, m - 16, k, 0, F, F, None) == sevo.INVALID_ARGUMENT
    a = dict(n=1 << 28, n_experts=1, top_k=1, n_groups=1, top_groups=1, group_best=1, scaling=1.0, ld=1,
             logits=F, out_experts=F, out_weights=F)
    assert L.sevo_moe_route(C.byref(sevo.MoeRouteArgs(**a)), None) == sevo.UNSUPPORTED
    a.update(n=(1 << 28) - 16, logits=0)
    assert L.sevo_moe_route(C.byref(sevo.MoeRouteArgs(**a)), None) == sevo.INVALID_ARGUMENT
