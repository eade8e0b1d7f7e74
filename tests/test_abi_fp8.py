"""C-ABI checks of the 8-bit layer that need no GPU: struct layouts, refusals."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2604_07725_amd import sevo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {"sevo_add_rmsnorm_fp8_args": sevo.AddRmsnormFp8Args,
           "sevo_linear_fp8_args": sevo.LinearFp8Args,
           "sevo_moe_route_args": sevo.MoeRouteArgs,
           "sevo_moe_linear_fp8_args": sevo.MoeLinearFp8Args}


def test_ctypes_structs_match_c_layout(tmp_path):
    src, exe = tmp_path / "layout.c", str(tmp_path / "layout")
    lines = []
    for t, py in STRUCTS.items():
        lines.append(f'printf("{t} %zu\\n", sizeof({t}));')
        lines += [f'printf("{t}.{f} %zu\\n", offsetof({t}, {f}));' for f, _ in py._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sevo.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    for line in subprocess.check_output([exe], text=True).splitlines():
        key, val = line.split()
        if "." in key:
            t, f = key.split(".")
            assert getattr(STRUCTS[t], f).offset == int(val), key
        else:
            assert C.sizeof(STRUCTS[key]) == int(val), key


F = 1 << 20   # a pointer that no check reads


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), sevo.INVALID_ARGUMENT), (dict(cols=0), sevo.INVALID_ARGUMENT),
    (dict(cols=4160), sevo.UNSUPPORTED), (dict(cols=32896), sevo.UNSUPPORTED),
    (dict(n_partials=17), sevo.INVALID_ARGUMENT), (dict(n_partials=-1), sevo.INVALID_ARGUMENT),
    (dict(partial_type=2), sevo.INVALID_ARGUMENT), (dict(eps=0.0), sevo.INVALID_ARGUMENT),
    (dict(eps=float("nan")), sevo.INVALID_ARGUMENT), (dict(x=0), sevo.INVALID_ARGUMENT),
    (dict(partials=0), sevo.INVALID_ARGUMENT), (dict(gain=F + 2), sevo.INVALID_ARGUMENT),
    (dict(out_bf16=F + 8), sevo.INVALID_ARGUMENT), (dict(scales=0), sevo.INVALID_ARGUMENT),
    (dict(rows=0, x=0), sevo.OK)])
def test_add_rmsnorm_fp8_refuses(kw, status):
    a = dict(rows=4, cols=4096, n_partials=1, partial_type=sevo.BF16, eps=1e-6, x=F, partials=F,
             gain=F, out=F, scales=F)
    a.update(kw)
    assert sevo.lib().sevo_add_rmsnorm_fp8(C.byref(sevo.AddRmsnormFp8Args(**a)), None) == status
    assert sevo.lib().sevo_add_rmsnorm_fp8(None, None) == sevo.INVALID_ARGUMENT


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), sevo.INVALID_ARGUMENT), (dict(k=0), sevo.INVALID_ARGUMENT),
    (dict(k=192), sevo.UNSUPPORTED), (dict(swiglu=2), sevo.INVALID_ARGUMENT),
    (dict(ldx=248), sevo.INVALID_ARGUMENT), (dict(ldx=260), sevo.INVALID_ARGUMENT),
    (dict(swiglu=1), sevo.INVALID_ARGUMENT), (dict(x=0), sevo.INVALID_ARGUMENT),
    (dict(out=F + 8), sevo.INVALID_ARGUMENT), (dict(m=0, x=0), sevo.OK)])
def test_quantize_fp8_refuses(kw, status):
    a = dict(x=F, ldx=256, m=4, k=256, swiglu=0, out=F, scales=F)
    a.update(kw)
    assert sevo.lib().sevo_quantize_fp8(a["x"], a["ldx"], a["m"], a["k"], a["swiglu"], a["out"],
                                        a["scales"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n_out=96), sevo.UNSUPPORTED), (dict(k=64), sevo.UNSUPPORTED),
    (dict(n_out=-64), sevo.INVALID_ARGUMENT), (dict(src=0), sevo.INVALID_ARGUMENT),
    (dict(dst=F + 4096), sevo.INVALID_ARGUMENT), (dict(dst=F - 4096), sevo.INVALID_ARGUMENT),
    (dict(n_out=0, src=0), sevo.OK)])
def test_pack_weight_fp8_refuses(kw, status):
    a = dict(src=F, dst=1 << 24, n_out=64, k=128)
    a.update(kw)
    assert sevo.lib().sevo_pack_weight_fp8(a["src"], a["dst"], a["n_out"], a["k"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), sevo.INVALID_ARGUMENT), (dict(out_type=2), sevo.INVALID_ARGUMENT),
    (dict(n_out=0), sevo.INVALID_ARGUMENT), (dict(n_out=96), sevo.UNSUPPORTED),
    (dict(k=192), sevo.UNSUPPORTED), (dict(k=1 << 23, ldx=1 << 23), sevo.UNSUPPORTED),
    (dict(ldx=240), sevo.INVALID_ARGUMENT), (dict(ldx=264), sevo.INVALID_ARGUMENT),
    (dict(ldx=1 << 23), sevo.INVALID_ARGUMENT), (dict(lds=1 << 28), sevo.UNSUPPORTED), (dict(lds=3), sevo.INVALID_ARGUMENT),
    (dict(ldo=124), sevo.INVALID_ARGUMENT), (dict(ldo=130), sevo.INVALID_ARGUMENT),
    (dict(x=0), sevo.INVALID_ARGUMENT), (dict(x_scales=0), sevo.INVALID_ARGUMENT),
    (dict(w=F + 8), sevo.INVALID_ARGUMENT), (dict(w_scales=0), sevo.INVALID_ARGUMENT),
    (dict(out=0), sevo.INVALID_ARGUMENT), (dict(m=0, x=0), sevo.OK)])
def test_linear_fp8_refuses(kw, status):
    a = dict(m=4, n_out=128, k=256, out_type=sevo.BF16, ldx=256, lds=4, ldo=128, x=F, x_scales=F,
             w=F, w_scales=F, out=F, workspace=F, workspace_bytes=1 << 30)
    a.update(kw)
    assert sevo.lib().sevo_linear_fp8(C.byref(sevo.LinearFp8Args(**a)), None) == status


def test_linear_fp8_workspace():
    L = sevo.lib()
    need = L.sevo_linear_fp8_workspace_bytes(64, 5120, 25600)
    assert need > 0
    a = dict(m=64, n_out=5120, k=25600, out_type=sevo.BF16, ldx=25600, lds=64, ldo=5120, x=F,
             x_scales=F, w=F, w_scales=F, out=F)
    short = sevo.LinearFp8Args(**a, workspace=F, workspace_bytes=need - 1)
    assert L.sevo_linear_fp8(C.byref(short), None) == sevo.WORKSPACE_TOO_SMALL
    assert L.sevo_linear_fp8(C.byref(sevo.LinearFp8Args(**a)), None) == sevo.INVALID_ARGUMENT
    for bad in ((0, 64, 128), (4, 96, 128), (4, 64, 64), (-1, 64, 128)):
        assert L.sevo_linear_fp8_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), sevo.INVALID_ARGUMENT), (dict(n_experts=257, ld=257), sevo.UNSUPPORTED),
    (dict(n_experts=0), sevo.UNSUPPORTED), (dict(top_k=17), sevo.UNSUPPORTED),
    (dict(top_k=0), sevo.UNSUPPORTED), (dict(score=2), sevo.INVALID_ARGUMENT),
    (dict(renormalise=2), sevo.INVALID_ARGUMENT), (dict(scaling=float("inf")), sevo.INVALID_ARGUMENT),
    (dict(n_groups=0), sevo.INVALID_ARGUMENT), (dict(n_groups=5), sevo.INVALID_ARGUMENT),
    (dict(n_groups=128, top_groups=64), sevo.INVALID_ARGUMENT),
    (dict(top_groups=9), sevo.INVALID_ARGUMENT), (dict(top_groups=0), sevo.INVALID_ARGUMENT),
    (dict(group_best=3), sevo.INVALID_ARGUMENT), (dict(group_best=0), sevo.INVALID_ARGUMENT),
    (dict(n_groups=64, top_groups=3), sevo.INVALID_ARGUMENT),          # 6 experts left, 8 a token
    (dict(ld=127), sevo.INVALID_ARGUMENT), (dict(logits=0), sevo.INVALID_ARGUMENT),
    (dict(out_weights=0), sevo.INVALID_ARGUMENT), (dict(n=0, logits=0), sevo.OK)])
def test_moe_route_refuses(kw, status):
    a = dict(n=4, n_experts=128, top_k=8, score=0, n_groups=8, top_groups=4, group_best=2,
             renormalise=1, scaling=1.0, ld=128, logits=F, out_experts=F, out_weights=F)
    a.update(kw)
    assert sevo.lib().sevo_moe_route(C.byref(sevo.MoeRouteArgs(**a)), None) == status


def test_moe_lists_refuses():
    L = sevo.lib()
    need = L.sevo_moe_lists_bytes(64, 8, 128)
    assert need >= 4 * (129 + 64 * 8)
    assert L.sevo_moe_lists_bytes(64, 8, 257) == 0 and L.sevo_moe_lists_bytes(0, 8, 128) == 0
    assert L.sevo_moe_lists_bytes(1 << 28, 16, 128) == 0
    call = L.sevo_moe_lists
    assert call(F, 64, 8, 128, F, need - 1, None) == sevo.WORKSPACE_TOO_SMALL
    assert call(0, 64, 8, 128, F, need, None) == sevo.INVALID_ARGUMENT
    assert call(F + 4, 64, 8, 128, F, need, None) == sevo.INVALID_ARGUMENT
    assert call(F, 64, 8, 128, F + 4, need, None) == sevo.INVALID_ARGUMENT
    assert call(F, 64, 8, 257, F, need, None) == sevo.UNSUPPORTED
    assert call(F, 1 << 28, 16, 128, F, 1 << 40, None) == sevo.INVALID_ARGUMENT
    assert call(0, 0, 8, 128, 0, 0, None) == sevo.OK


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), sevo.INVALID_ARGUMENT), (dict(top_k=17), sevo.UNSUPPORTED),
    (dict(n_experts=300), sevo.UNSUPPORTED), (dict(down=2), sevo.INVALID_ARGUMENT),
    (dict(n_out=96), sevo.UNSUPPORTED), (dict(k=192), sevo.UNSUPPORTED),
    (dict(ldx=240), sevo.INVALID_ARGUMENT), (dict(lds=63), sevo.INVALID_ARGUMENT),
    (dict(down=1, lds=64, weights=F), sevo.INVALID_ARGUMENT),          # scales of n top_k rows
    (dict(down=1, lds=512), sevo.INVALID_ARGUMENT),                    # no weights
    (dict(x=0), sevo.INVALID_ARGUMENT), (dict(lists=0), sevo.INVALID_ARGUMENT),
    (dict(out=F + 4), sevo.INVALID_ARGUMENT),
    (dict(n=1 << 23, lds=1 << 23), sevo.UNSUPPORTED),                  # x of 2^31 bytes
    (dict(n=0, x=0), sevo.OK)])
def test_moe_linear_fp8_refuses(kw, status):
    a = dict(n=64, top_k=8, n_experts=128, n_out=128, k=256, down=0, ldx=256, lds=64, x=F,
             x_scales=F, w=F, w_scales=F, lists=F, out=F)
    a.update(kw)
    assert sevo.lib().sevo_moe_linear_fp8(C.byref(sevo.MoeLinearFp8Args(**a)), None) == status


def test_binding_refuses_wrong_tensors():
    """Types, shapes and layouts are checked before the call."""
    f8 = torch.float8_e4m3fn
    x8, xs = torch.zeros(4, 256).to(f8), torch.zeros(2, 4)
    w8, ws = torch.zeros(64, 256).to(f8), torch.zeros(1, 2)
    for bad in ((x8.float(), xs, w8, ws), (x8, xs.t().contiguous(), w8, ws), (x8, xs.double(), w8, ws),
                (x8, xs, w8[:, :128], ws), (x8, xs, w8, torch.zeros(2, 2)),
                (x8.t().contiguous().t(), xs, w8, ws)):
        with pytest.raises(ValueError):
            sevo.sevo_linear_fp8(*bad)
    with pytest.raises(ValueError):
        sevo.sevo_linear_fp8(x8, xs, w8, ws, out=torch.zeros(4, 64, dtype=torch.float16))
    x, gain = torch.zeros(4, 256), torch.zeros(256, dtype=torch.bfloat16)
    for a in ((x.double(), None, gain), (x.t(), None, gain), (x, torch.zeros(4, 256), gain),
              (x, torch.zeros(1, 4, 256, dtype=torch.float16), gain), (x, None, gain.float())):
        with pytest.raises(ValueError):
            sevo.sevo_add_rmsnorm_fp8(*a, 1e-6)
    with pytest.raises(ValueError):
        sevo.sevo_quantize_fp8(x)
    with pytest.raises(ValueError):
        sevo.sevo_quantize_fp8(torch.zeros(4, 257, dtype=torch.bfloat16), swiglu=True)
    with pytest.raises(ValueError):
        sevo.sevo_pack_weight_fp8(torch.zeros(2, 96, 128).to(f8))
    with pytest.raises(ValueError):
        sevo.sevo_moe_route(torch.zeros(4, 8), 2, score="relu")
    with pytest.raises(ValueError):
        sevo.sevo_moe_route(torch.zeros(4, 8), 2, bias=torch.zeros(9))
    with pytest.raises(ValueError):
        sevo.sevo_moe_lists(torch.zeros(4, 2, dtype=torch.int64), 8)
    lists = sevo.MoeLists(4, 2, 3, torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError):                     # weights of another expert count
        sevo.sevo_moe_linear_fp8(x8, xs, torch.zeros(2, 64, 256).to(f8), torch.zeros(2, 1, 2), lists)
    with pytest.raises(ValueError):                     # rows per entry needed
        sevo.sevo_moe_linear_fp8(x8, xs, torch.zeros(3, 64, 256).to(f8), torch.zeros(3, 1, 2), lists,
                                 weights=torch.zeros(4, 2))
