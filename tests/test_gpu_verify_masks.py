"""Verification of drafted tokens where both distributions are truncated: whole chunks of the vocabulary
without any probability, at the ends of the uniform numbers, against float64."""
import math

import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_verify import check, gen, sevo  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
LAST = (0.0, 1.0 - 2.0 ** -24, 1.0)


def truncated(v, lo, hi, mask, g, n=6):
    """Target rows [n, 2, v] and draft rows [n, 1, v] with ``mask`` outside [lo, hi), the first half of the
    candidates with a flatter draft row (its sum of exponentials is the larger one), the others with a
    steeper one."""
    z = torch.full((n, 2, v), mask)
    y = torch.full((n, 1, v), mask)
    z[:, :, lo:hi] = torch.randn(n, 2, hi - lo, generator=g) * 2
    y[:, :, lo:hi] = torch.randn(n, 1, hi - lo, generator=g) * 2
    y[:n // 2, :, lo:hi] *= 0.5
    y[n // 2:, :, lo:hi] *= 2.0

    def total(x):
        return torch.exp(x.double() - x.double().amax(-1, keepdim=True)).sum(-1)
    larger = total(y[:, 0]) > total(z[:, 0])
    assert larger[:n // 2].all() and not larger[n // 2:].any()
    return z, y


def refused(z, y, temp):
    """Drafts with more probability under y than under z, and their uniform number: all are refused."""
    p, q = (torch.softmax(x[:, 0].double() / temp, 1) for x in (z, y))
    return (q - p).argmax(1, keepdim=True).to(torch.int32), 1.0 - 2.0 ** -24


@pytest.mark.parametrize("mask", [-math.inf, -1e4, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("v,lo,hi", [
    (6244, 2048, 4400), (6144, 2100, 4000), (4097, 2048, 4096), (2049, 2048, 2049), (5000, 0, 2000),
    (151936, 81920, 81990), (163841, 4096, 163840), (250003, 140000, 249000)])
def test_chunks_masked_in_both_rows(sevo, v, lo, hi, mask):  # noqa: F811
    if hi - lo == 1:      # one entry that holds all of either row: nothing is left of the residual
        z, y = torch.full((6, 2, v), mask), torch.full((6, 1, v), mask)
        z[:, :, lo], y[:, :, lo] = 1.5, torch.arange(6.0)[:, None]
    else:
        z, y = truncated(v, lo, hi, mask, gen(v))
    x, first = refused(z, y, 1.0)
    if hi - lo == 1:
        x, first = torch.full_like(x, lo), 1.0
    for last in LAST:
        u = torch.full((6, 2), last)
        u[:, 0] = first
        tok, lp, taken = check(sevo, z, x, u, 1.0, y)
        assert (taken == 0).all() and (tok[:, 0] >= lo).all() and (tok[:, 0] < hi).all()
        assert lp[:, 0].isfinite().all()
        check(sevo, z, x, u, 1.0)                 # certain drafts
    u = torch.rand(6, 2, generator=gen(1))
    check(sevo, z, x, u, 1.0, y)


def test_a_target_narrower_than_the_draft(sevo):  # noqa: F811
    """The target keeps entries of one chunk, the draft's row all of them, and the reverse."""
    g = gen(3)
    v = 8192
    z = torch.full((4, 2, v), -math.inf)
    z[:, :, 4100:4200] = torch.randn(4, 2, 100, generator=g)
    y = torch.randn(4, 1, v, generator=g) * 3
    for a, b in ((z, y), (torch.cat([y, y], 1), z[:, :1])):
        x, first = refused(a, b, 1.0)
        for last in LAST:
            u = torch.tensor([[first, last]]).repeat(4, 1)
            check(sevo, a, x, u, 1.0, b)


@pytest.mark.parametrize("temp", [2e-3, 1e-3])
def test_small_temperatures_without_masks(sevo, temp):  # noqa: F811
    """Entries hundreds of nats below the largest: no row holds a mask, most entries no share.  (None is put
    between 700 and 760 nats, where shares are subnormal and float64 libraries differ in what they keep.)"""
    g = gen(7)
    n, v = 6, 6200
    z, y = torch.randn(n, 2, v, generator=g) * 2, torch.randn(n, 1, v, generator=g) * 2
    for x in (z, y):
        d = (x.amax(2, keepdim=True) - x) / temp
        x[(d > 690) & (d < 770)] -= 100 * temp
    x, first = refused(z, y, temp)
    for last in LAST:
        u = torch.tensor([[first, last]]).repeat(n, 1)
        check(sevo, z, x, u, temp, y)


def test_shares_near_the_end_of_float64(sevo):  # noqa: F811
    """With the last uniform number 0 the first entry with any share is drawn, however small: 640 to 700
    nats below the largest."""
    v = 6200
    z, y = torch.full((4, 2, v), -math.inf), torch.full((4, 1, v), -math.inf)
    z[:, :, 5000], y[:, :, 5000] = 0.0, 0.0
    z[:, :, 5001], y[:, :, 5001] = 0.0, 1.0
    for i, at in enumerate((640.0, 670.0, 700.0)):
        z[i, 0, 77 + 2048 * i] = -at
    x, first = refused(z, y, 1.0)
    assert (x == 5001).all()
    tok, _, _ = check(sevo, z, x, torch.tensor([[first, 0.0]]).repeat(4, 1), 1.0, y)
    assert tok[:, 0].tolist() == [77, 77 + 2048, 77 + 4096, 5000]
    # behind the mass they are the last ones
    z[:, 0, 6100] = torch.tensor([-640.0, -670.0, -700.0, -math.inf])
    tok, _, _ = check(sevo, z, x, torch.tensor([[first, 1.0]]).repeat(4, 1), 1.0, y)
    assert tok[:, 0].tolist() == [6100, 6100, 6100, 5000]
