"""GPU tests of calls of the 8-bit layer that tests/test_gpu_fp8.py does not make:
explicit streams, routers with large biases, entries without an expert, the
accuracy of the 8-bit sums, and a layer around its attention.  Its tolerances and
helpers are those of that file."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import say
from tests.test_gpu_fp8 import BF, F8, check_codes, check_product, gen, normal, quantised, sevo, weights  # noqa: F401

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream that the memory of t belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no segment")


def test_stream_arguments(sevo):
    """Chains on two explicit streams, nothing given and temporaries dropped at once:
    always the bits of the same chain alone, in memory of the chain's stream."""
    g = gen(31)
    m, n_out, k = 64, 1024, 12288
    assert sevo.sevo_linear_fp8_workspace_bytes(m, n_out, k) > 0     # K splits: a workspace of the call's own
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    ins = [normal((m, k), g, 1.0, BF) for _ in range(2)]
    ex = [torch.randint(0, 16, (m, 4), device="cuda", dtype=torch.int32, generator=g) for _ in range(2)]
    mq, ms = weights((16, 256, n_out), g)
    mw = sevo.sevo_pack_weight_fp8(mq)

    def chain(i, stream=None):
        y = sevo.sevo_linear_fp8(*sevo.sevo_quantize_fp8(ins[i], stream=stream), w, ws, stream=stream)
        return y, sevo.sevo_moe_linear_fp8(*sevo.sevo_quantize_fp8(y, stream=stream), mw, ms,
                                           sevo.sevo_moe_lists(ex[i], 16, stream=stream), stream=stream)

    want = [chain(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    handles = (streams[0], streams[1].cuda_stream)                   # a Stream and a raw handle
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(chain(i, handles[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for y, z in got[i]:
            assert torch.equal(y, want[i][0]) and torch.equal(z, want[i][1])
        assert stream_of(got[i][-1][0]) == streams[i].cuda_stream
