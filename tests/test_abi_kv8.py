"""C-ABI and binding checks of the 8-bit cache and of drafted tokens that need no GPU:
struct layouts, refusals, workspaces, the cache's layout, stream arguments."""
import ctypes as C
import os
import subprocess
import types

import pytest
import torch

from paper_2604_07725_amd import sevo
from tests.kv8_ref import k_offsets, v_offsets
from tests.test_streams import Library, bf, ints, watched  # noqa: F401  (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

STRUCTS = {"sevo_kv_pages_args": sevo.KvPagesArgs, "sevo_attn_fp8_args": sevo.AttnFp8Args,
           "sevo_verify_args": sevo.VerifyArgs}
F = 1 << 20   # a pointer that no check reads
BAD, UNS, SMALL, OK = sevo.INVALID_ARGUMENT, sevo.UNSUPPORTED, sevo.WORKSPACE_TOO_SMALL, sevo.OK


def test_ctypes_structs_match_c_layout(tmp_path):
    src, exe = tmp_path / "layout.c", str(tmp_path / "layout")
    lines = [f'printf("tile.64 %d\\n", (int)SEVO_KV8_TILE_BYTES(64));',
             f'printf("tile.128 %d\\n", (int)SEVO_KV8_TILE_BYTES(128));']
    for t, py in STRUCTS.items():
        lines.append(f'printf("{t} %zu\\n", sizeof({t}));')
        lines += [f'printf("{t}.{f} %zu\\n", offsetof({t}, {f}));' for f, _ in py._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sevo.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    for line in subprocess.check_output([exe], text=True).splitlines():
        key, val = line.split()
        if key.startswith("tile."):
            assert sevo.sevo_kv8_tile_bytes(int(key[5:])) == int(val)
        elif "." in key:
            t, f = key.split(".")
            assert getattr(STRUCTS[t], f).offset == int(val), key
        else:
            assert C.sizeof(STRUCTS[key]) == int(val), key


@pytest.mark.parametrize("d", [64, 128])
def test_cache_layout_is_a_permutation(d):
    for at in (k_offsets(d), v_offsets(d)):
        assert sorted(at.reshape(-1).tolist()) == list(range(16 * d))


@pytest.mark.parametrize("kw,status", [
    (dict(n_kv_heads=0), BAD), (dict(count=-1), BAD), (dict(src_num_pages=-1), BAD),
    (dict(dst_num_pages=-1), BAD), (dict(head_dim=96), UNS), (dict(count=1 << 30), UNS),
    (dict(count=9), BAD), (dict(count=9, src_pages=F), BAD), (dict(count=9, dst_pages=F), BAD),
    (dict(src=0), BAD), (dict(dst=0), BAD), (dict(src=F + 8), BAD), (dict(src_pages=F + 2), BAD),
    (dict(dst_pages=F + 1), BAD), (dict(dst=F + 4096), BAD), (dict(dst=F - 4096), BAD),
    (dict(src_num_pages=1 << 50, src_pages=F), BAD),
    (dict(count=0, src=0, dst=0), OK)])
@pytest.mark.parametrize("name", ["sevo_pack_kv_fp8", "sevo_unpack_kv_fp8"])
def test_kv_pages_refuses(name, kw, status):
    a = dict(n_kv_heads=2, head_dim=128, count=8, src_num_pages=8, dst_num_pages=8, src=F, dst=1 << 24)
    a.update(kw)
    fn = getattr(sevo.lib(), name)
    assert fn(C.byref(sevo.KvPagesArgs(**a)), None) == status
    assert fn(None, None) == BAD


ATTN = dict(n=4, n_tokens=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, max_pages=100,
            num_pages=50, q=F, kv_pool=F, page_table=F, seq_lens=F, q_lens=F, scale=0.1, out=F,
            workspace=F, workspace_bytes=1 << 30)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), BAD), (dict(max_pages=0), BAD), (dict(head_dim=32), UNS), (dict(n_tokens=0), UNS),
    (dict(n_tokens=17), UNS), (dict(n_q_heads=9), UNS), (dict(n_q_heads=34), UNS),
    (dict(n_kv_heads=0), UNS), (dict(n_q_heads=0), UNS), (dict(page_size=32), UNS),
    (dict(max_pages=1 << 28), UNS), (dict(n=1 << 22), UNS), (dict(n=1 << 17, max_pages=2), UNS),
    (dict(n=1 << 15, max_pages=(1 << 15) + 1), UNS), (dict(num_pages=0), BAD),
    (dict(scale=0.0), BAD), (dict(scale=float("nan")), BAD), (dict(clear_rest=2), BAD),
    (dict(q=0), BAD), (dict(kv_pool=F + 8), BAD), (dict(page_table=0), BAD), (dict(seq_lens=0), BAD),
    (dict(out=0), BAD), (dict(q_lens=F + 2), BAD), (dict(seq_lens=F + 1), BAD), (dict(workspace=0), BAD),
    (dict(workspace=F + 4), BAD), (dict(workspace_bytes=100), SMALL), (dict(n=0, q=0), OK)])
def test_attn_decode_fp8_refuses(kw, status):
    fn = sevo.lib().sevo_attn_decode_fp8
    assert fn(C.byref(sevo.AttnFp8Args(**{**ATTN, **kw})), None) == status
    assert fn(None, None) == BAD


def test_attn_fp8_workspace():
    size = sevo.lib().sevo_attn_fp8_workspace_bytes
    need = size(4, 3, 8, 2, 128, 100)
    assert need > 0
    short = sevo.AttnFp8Args(**{**ATTN, "workspace_bytes": need - 1})
    assert sevo.lib().sevo_attn_decode_fp8(C.byref(short), None) == SMALL
    assert size(4, 3, 8, 2, 128, 2) == 0          # a candidate's pages are one split
    for bad in ((0, 1, 8, 2, 128, 100), (4, 17, 8, 2, 128, 100), (4, 1, 7, 2, 128, 100), (4, 1, 8, 2, 96, 100),
                (4, 1, 8, 2, 128, 0), (-1, 1, 8, 2, 128, 9)):
        assert size(*bad) == 0


VERIFY = dict(n=4, n_drafts=3, vocab=1000, ld=1000, ld_draft=1000, temperature=1.0, logits=F,
              draft_logits=F, draft_tokens=F, uniforms=F, counts=F, out_tokens=F, out_logprobs=F,
              out_accepted=F, workspace=F, workspace_bytes=1 << 30)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), BAD), (dict(vocab=0), BAD), (dict(n_drafts=-1), UNS), (dict(n_drafts=17), UNS),
    (dict(vocab=(1 << 24) + 1, ld=1 << 25, ld_draft=1 << 25), UNS), (dict(n=1 << 22), UNS),
    (dict(temperature=-1.0), BAD), (dict(temperature=float("nan")), BAD),
    (dict(temperature=float("inf")), BAD), (dict(temperature=1e-40), UNS), (dict(temperature=1e31), UNS), (dict(ld=996), BAD),
    (dict(ld=1002), BAD), (dict(ld_draft=996), BAD), (dict(ld_draft=1001), BAD), (dict(logits=0), BAD),
    (dict(logits=F + 4), BAD), (dict(draft_logits=F + 4), BAD), (dict(draft_tokens=0), BAD),
    (dict(uniforms=0), BAD), (dict(counts=F + 2), BAD), (dict(out_tokens=0), BAD),
    (dict(out_logprobs=0), BAD), (dict(out_accepted=F + 2), BAD), (dict(workspace=0), BAD),
    (dict(workspace_bytes=64), SMALL), (dict(n=0, logits=0), OK)])
def test_verify_drafts_refuses(kw, status):
    fn = sevo.lib().sevo_verify_drafts
    assert fn(C.byref(sevo.VerifyArgs(**{**VERIFY, **kw})), None) == status
    assert fn(None, None) == BAD


def test_verify_workspace():
    size = sevo.lib().sevo_verify_workspace_bytes
    need = size(4, 3, 1000)
    assert need > 0
    short = sevo.VerifyArgs(**{**VERIFY, "workspace_bytes": need - 1})
    assert sevo.lib().sevo_verify_drafts(C.byref(short), None) == SMALL
    for bad in ((0, 3, 1000), (4, 17, 1000), (4, -1, 1000), (4, 3, 0), (4, 3, (1 << 24) + 1)):
        assert size(*bad) == 0


def test_append_refuses_without_a_model():
    assert sevo.lib().sevo_qk_norm_rope_append_fp8(None, 0, F, 1, F, None, F, 1, 1, 1, F, F, None) == BAD


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def fp(*shape):
    return torch.zeros(shape)


MODEL = types.SimpleNamespace(handle=0, config=types.SimpleNamespace(n_q_heads=4, n_kv_heads=2, head_dim=64))
TILE = 32 * 64 + 128
CALLS = {
    "append": lambda **k: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(3), ints(2, 3),
                                                            u8(5, 2, TILE), rows=ints(3), **k),
    "pack": lambda **k: sevo.sevo_pack_kv_fp8(bf(3, 2, 2, 1024), src_pages=ints(2), **k),
    "unpack": lambda **k: sevo.sevo_unpack_kv_fp8(u8(3, 2, TILE), **k),
    "attn": lambda **k: sevo.sevo_attn_decode_fp8(bf(2, 3, 4, 64), u8(5, 2, TILE), ints(2, 90), ints(2), **k),
    "verify": lambda **k: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 2), fp(2, 3), **k),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_stream(watched, monkeypatch, name):  # noqa: F811
    for size in ("sevo_attn_fp8_workspace_bytes", "sevo_verify_workspace_bytes"):   # (they keep their answers)
        monkeypatch.setattr(sevo, size, lambda *a: 4096)
    out = CALLS[name](stream=1234)
    assert watched.under is None and watched.launched == [1234]
    made = [p for s, p in watched.made if s == 1234]
    returned = [t.data_ptr() for t in (out if isinstance(out, tuple) else (out,))]
    assert returned and all(p in made for p in returned)
    assert all((p, 7) in watched.marked for p in returned)
    assert len(made) == len(returned) + (name in ("attn", "verify"))    # outputs and the workspace
    CALLS[name]()
    assert watched.launched == [1234, None]


@pytest.mark.parametrize("call", [
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 500), ints(3), ints(2, 3), u8(5, 2, TILE)),
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(2), ints(2, 3), u8(5, 2, TILE)),
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(3), ints(2, 3), u8(5, 2, TILE + 1)),
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(3), ints(2, 3), u8(5, 4, TILE)[:, ::2]),
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(3), ints(2, 3), u8(5, 2, TILE),
                                              rows=ints(4)),
    lambda: sevo.sevo_qk_norm_rope_append_fp8(MODEL, 0, fp(3, 512), ints(3).long(), ints(2, 3), u8(5, 2, TILE)),
    lambda: sevo.sevo_pack_kv_fp8(bf(3, 2, 2, 1000)),
    lambda: sevo.sevo_pack_kv_fp8(bf(3, 2, 1024)),
    lambda: sevo.sevo_pack_kv_fp8(bf(3, 2, 2, 1024), u8(3, 4, TILE)),
    lambda: sevo.sevo_pack_kv_fp8(bf(3, 2, 2, 1024), u8(3, 2, TILE), src_pages=ints(2), dst_pages=ints(3)),
    lambda: sevo.sevo_pack_kv_fp8(bf(3, 2, 2, 1024), dst_pages=ints(3)),
    lambda: sevo.sevo_unpack_kv_fp8(u8(3, 2, TILE + 16)),
    lambda: sevo.sevo_unpack_kv_fp8(u8(3, 2, TILE), bf(3, 2, 2, 2048)),
    lambda: sevo.sevo_unpack_kv_fp8(u8(3, 2, TILE), src_pages=ints(2).long()),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4), u8(5, 2, TILE), ints(2, 90), ints(2)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 64).float(), u8(5, 2, TILE), ints(2, 90), ints(2)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 128), u8(5, 2, TILE), ints(2, 90), ints(2)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 64), u8(5, 2, TILE), ints(3, 90), ints(2)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 64), u8(5, 2, TILE), ints(2, 180)[:, ::2], ints(2)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 64), u8(5, 2, TILE), ints(2, 90), ints(2), q_lens=ints(3)),
    lambda: sevo.sevo_attn_decode_fp8(bf(2, 4, 64), u8(5, 2, TILE), ints(2, 90), ints(2), out=bf(2, 1, 4, 64)),
    lambda: sevo.sevo_attn_decode_fp8(bf(4, 2, 64).transpose(0, 1), u8(5, 2, TILE), ints(2, 90), ints(2)),
    lambda: sevo.sevo_verify_drafts(fp(3, 64), ints(2, 2), fp(2, 3)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 3), fp(2, 3)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 2), fp(2, 2)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 2), fp(2, 3), vocab=65),
    lambda: sevo.sevo_verify_drafts(fp(2, 4, 64)[:, ::3][:, :2], ints(2, 1), fp(2, 2), draft_logits=fp(2, 2, 64)),
    lambda: sevo.sevo_verify_drafts(fp(2, 5, 64)[:, :3], ints(2, 2), fp(2, 3)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 2), fp(2, 3), draft_logits=fp(2, 2, 60)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64).double(), ints(2, 2), fp(2, 3)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 128)[:, :, ::2], ints(2, 2), fp(2, 3)),
    lambda: sevo.sevo_verify_drafts(fp(2, 3, 64), ints(2, 2), fp(2, 3), n_drafts=ints(3)),
])
def test_the_binding_refuses(call, monkeypatch):
    monkeypatch.setattr(sevo, "_call", lambda *a: pytest.fail("reached the library"))
    with pytest.raises(ValueError):
        call()


def test_tensors_on_the_cpu_are_refused():
    for name in ("pack", "unpack", "attn", "verify", "append"):
        with pytest.raises(ValueError, match="CPU"):
            CALLS[name]()
