"""The binding's ``stream`` argument, without a GPU: everything that a call
allocates belongs to the stream that it runs on, so that no other call is given
the same memory while its kernels run."""
import contextlib
import types

import pytest
import torch

from paper_2604_07725_amd import sevo

F8, BF = torch.float8_e4m3fn, torch.bfloat16


def f8(*shape):
    return torch.zeros(shape).to(F8)


def bf(*shape):
    return torch.zeros(shape, dtype=BF)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


LISTS = sevo.MoeLists(4, 2, 3, torch.zeros(1 << 16, dtype=torch.uint8))
SHAPE = types.SimpleNamespace(n_layers=1, hidden=64, vocab=128, top_k=2)
MODEL = types.SimpleNamespace(handle=0, shape=SHAPE,
                              config=types.SimpleNamespace(n_q_heads=2, head_dim=64))
CALLS = {
    "add_rmsnorm_fp8": lambda **k: sevo.sevo_add_rmsnorm_fp8(torch.zeros(4, 256), None, bf(256), 1e-6, **k),
    "quantize_fp8": lambda **k: sevo.sevo_quantize_fp8(bf(4, 256), **k),
    "pack_weight_fp8": lambda **k: sevo.sevo_pack_weight_fp8(f8(64, 128), **k),
    "linear_fp8": lambda **k: sevo.sevo_linear_fp8(f8(4, 256), torch.zeros(2, 4), f8(64, 256),
                                                   torch.zeros(1, 2), **k),
    "moe_route": lambda **k: sevo.sevo_moe_route(torch.zeros(4, 8), 2, **k),
    "moe_lists": lambda **k: sevo.sevo_moe_lists(ints(4, 2), 3, **k),
    "moe_linear_fp8": lambda **k: sevo.sevo_moe_linear_fp8(f8(4, 256), torch.zeros(2, 4), f8(3, 64, 256),
                                                           torch.zeros(3, 1, 2), LISTS, **k),
    "attn_decode": lambda **k: sevo.sevo_attn_decode(bf(2, 4, 64), bf(3, 2, 2, 1024), ints(2, 3), ints(2), **k),
    "attn_prefill": lambda **k: sevo.sevo_attn_prefill(bf(5, 4, 64), bf(3, 2, 2, 1024), ints(2, 3), ints(3), 3, **k),
    "logprob_sample": lambda **k: sevo.sevo_logprob_sample(torch.zeros(2, 64), 1.0, 1, ints(2), ints(2), **k),
    "group_confidence": lambda **k: sevo.sevo_group_confidence(torch.zeros(4), ints(4), ints(2, 2), **k),
    "embed": lambda **k: sevo.sevo_embed(bf(8, 64), ints(2), **k),
    "rmsnorm": lambda **k: sevo.sevo_rmsnorm(torch.zeros(2, 64), bf(64), 1e-6, **k),
    "add_rmsnorm": lambda **k: sevo.sevo_add_rmsnorm(torch.zeros(2, 64), None, bf(64), 1e-6, **k),
    "linear": lambda **k: sevo.sevo_linear(bf(2, 64), bf(64, 64), **k),
    "pack_weight": lambda **k: sevo.sevo_pack_weight(bf(64, 64), **k),
    "pack_kv": lambda **k: sevo.sevo_pack_kv(bf(2, 2, 16, 64), bf(2, 2, 16, 64), **k),
    "qk_norm_rope_append": lambda **k: sevo.sevo_qk_norm_rope_append(
        MODEL, 0, torch.zeros(2, 256), ints(2), ints(2, 3), bf(3, 2, 2, 1024), **k),
    "decode_step": lambda **k: sevo.sevo_decode_step(MODEL, ints(2), ints(2), ints(2, 3), [bf(3, 2, 2, 1024)],
                                                     ints(2), 1, keep_logits=True, **k),
    "moe_ffn": lambda **k: sevo.sevo_moe_ffn(MODEL, 0, bf(16, 64), 4, **k),
    "hbm_read_probe": lambda **k: sevo.sevo_hbm_read_probe(bf(4096), **k),
}


class Library:
    """Every entry point: a size, or success."""

    def __getattr__(self, name):
        return lambda *a: 4096 if name.endswith("_bytes") else 0


@pytest.fixture
def watched(monkeypatch):
    """Allocations as (stream they are made under, pointer), the stream of each
    launch, and the tensors marked as used by another stream."""
    seen = types.SimpleNamespace(under=None, made=[], launched=[], marked=[])

    def stream_of(handle, device=None):
        return types.SimpleNamespace(cuda_stream=handle, device=device)

    @contextlib.contextmanager
    def under(s):
        before, seen.under = seen.under, s.cuda_stream
        yield
        seen.under = before

    def recording(make):
        def made(*a, **k):
            t = make(*a, **k)
            seen.made.append((seen.under, t.data_ptr()))
            return t
        return made

    monkeypatch.setattr(torch.cuda, "ExternalStream", stream_of)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream_of(7))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: seen.marked.append((t.data_ptr(), s.cuda_stream)), raising=False)
    monkeypatch.setattr(sevo, "lib", Library)
    monkeypatch.setattr(sevo, "_call", lambda name, i, *a: seen.launched.append(seen.under))
    for name in ("sevo_linear_fp8_workspace_bytes", "sevo_moe_lists_bytes"):   # (they keep their answers)
        monkeypatch.setattr(sevo, name, lambda *a: 4096)
    for name in ("empty", "zeros", "empty_like"):
        monkeypatch.setattr(torch, name, recording(getattr(torch, name)))
    return seen


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations_belong_to_the_stream(watched, name):
    out = CALLS[name](stream=1234)
    assert watched.under is None
    made = [p for s, p in watched.made if s == 1234]
    returned = [t.data_ptr() for t in (out if isinstance(out, tuple) else (out,)) if isinstance(t, torch.Tensor)]
    if isinstance(out, sevo.MoeLists):
        returned = [out.buffer.data_ptr()]
    assert returned and all(p in made for p in returned), f"{name}: outputs made on another stream"
    assert all((p, 7) in watched.marked for p in returned), f"{name}: not marked for the current stream"
    if name == "linear_fp8":
        assert len(made) == 2          # the output and the workspace
        assert watched.launched == [1234]


def test_without_a_stream_nothing_is_marked(watched):
    for call in CALLS.values():
        call()
    assert watched.marked == [] and all(s is None for s, _ in watched.made)


def test_a_stream_of_another_device_is_refused(monkeypatch):
    class Stream:
        device = torch.device("cuda:1")
        cuda_stream = 5
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    with pytest.raises(ValueError, match="stream"):
        sevo.sevo_quantize_fp8(bf(4, 256), stream=Stream())
