"""The 8-bit attention on the lowest scores that fp32 holds."""
import pytest
import torch

from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def sevo(have_gpu):
    from paper_2604_07725_amd import sevo
    sevo.lib()
    return sevo


@pytest.mark.parametrize("width", [20, 300])         # one split a candidate, several
@pytest.mark.parametrize("hq,d,T", [(2, 64, 1), (16, 64, 3), (4, 128, 1), (16, 128, 4)])
def test_equal_scores_near_the_lowest_number(sevo, hq, d, T, width):
    """Every key scores about -2.2e38 (-3.2e38 in base 2; fp32 ends at -3.4e38), but for the last third of
    them, which score 1e37 less and get nothing: an average of the others' values."""
    g = torch.Generator().manual_seed(d + T)
    lens = [T, 40, 319]
    hkv = 2
    table = torch.full((3, width), -1, dtype=torch.int32)
    table[:, :20] = torch.randperm(60, generator=g).view(3, 20).to(torch.int32)
    k = torch.ones(60, hkv, 16, d).to(ref.F8)
    v = (torch.randn(60, hkv, 16, d, generator=g) * 64).to(ref.F8)
    ks, vs = torch.full((60, hkv, 16), 3.0e18), torch.rand(60, hkv, 16, generator=g) / 64
    for i, n in enumerate(lens):
        for u in range(n - n // 3, n):
            ks[table[i, u // 16].long(), :, u % 16] = 3.1e18
    pool = ref.write_pool(k, v, ks, vs)
    q = torch.full((3, T, hq, d), -2.0 ** 69 / d).to(BF)
    scale = 0.125
    low = [2.0 ** 69 * s * scale * 1.4426950408889634 for s in (3.0e18, 3.1e18)]
    assert 3e38 < low[0] < low[1] < 3.4e38
    o = sevo.sevo_attn_decode_fp8(q.to(DEV), pool.to(DEV), table.to(DEV),
                                  torch.tensor(lens, dtype=torch.int32, device=DEV), scale=scale).double().cpu()
    vals = v.double() * vs.double()[..., None]
    for i, n in enumerate(lens):
        at = torch.arange(n)
        rows = vals[table[i, at // 16].long(), :, at % 16]       # [keys, hkv, d]
        for t in range(T):
            seen = n - T + t + 1
            few = min(seen, n - n // 3)
            if few < 1:
                continue
            want = rows[:few].mean(0).repeat_interleave(hq // hkv, 0)
            mass = rows[:few].abs().mean(0).repeat_interleave(hq // hkv, 0)
            # equal probabilities of exactly 1: two bf16 parts of p vs (2^-16), sums of 20 pages' keys in fp32,
            # the division, and bf16's half step
            bound = mass * (2.0 ** -16 + 2 * 330 * 2.0 ** -24) * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
            assert ((o[i, t] - want).abs() <= bound).all(), (i, t)
