"""Verification of drafted tokens on the GPU, against float64."""
import math

import pytest
import torch

from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def sevo(have_gpu):
    from paper_2604_07725_amd import sevo
    sevo.lib()
    return sevo


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows(n, r, v, g, std=2.0):
    z = torch.randn(n, r, v, generator=g) * std
    z.scatter_add_(2, torch.randint(0, v, (n, r, 5), generator=g), torch.full((n, r, 5), 6.0))
    return z


def padded(z):
    """On the GPU with a row stride of the next multiple of 4, NaN behind the rows."""
    n, r, v = z.shape
    out = torch.full((n, r, -(-v // 4) * 4), math.nan, device=DEV)
    out[:, :, :v] = z.to(DEV)
    return out


def check(sevo, z, x, u, temp, y=None, count=None, **kw):
    n, r, v = z.shape
    T = r - 1
    tok, lp, taken = sevo.sevo_verify_drafts(
        padded(z), x.to(DEV), u.to(DEV), temp, draft_logits=None if y is None else padded(y),
        n_drafts=None if count is None else count.to(DEV), vocab=v, **kw)
    tok, lp, taken = tok.cpu(), lp.double().cpu(), taken.cpu()
    for i in range(n):
        m = T if count is None else min(max(int(count[i]), 0), T)
        t, l, a = ref.verify(z[i], None if y is None else y[i], x[i], u[i], m, temp)
        assert int(taken[i]) == a and tok[i].tolist() == t + [-1] * (T - a), i
        l = torch.tensor(l, dtype=torch.float64)
        assert torch.equal(lp[i, :a + 1].isnan(), l.isnan())
        # fp64 until the last rounding, to fp32 (2^-24 of itself)
        assert ((lp[i, :a + 1] - l).abs()[~l.isnan()] <= 2.0 ** -24 * l.abs()[~l.isnan()] + 1e-12).all()
        assert (lp[i, a + 1:] == 0).all()
    return tok, lp, taken


@pytest.mark.parametrize("dist", [False, True])
@pytest.mark.parametrize("n,T,v,temp", [
    (1, 0, 1, 1.0), (1, 1, 1, 1.0), (3, 2, 2, 0.5), (5, 3, 63, 1.0), (4, 4, 4096, 0.7), (3, 2, 4097, 1.0),
    (7, 16, 1001, 1.3), (2, 5, 20483, 0.6), (2, 3, 151936, 1.0), (1, 2, 250003, 1.0), (1, 1, 250003, 0.0), (40, 1, 300, 1.0), (3, 4, 8191, 0.0), (6, 0, 5000, 1.0)])
def test_verify(sevo, n, T, v, temp, dist):
    g = gen(n * T + v)
    z = rows(n, T + 1, v, g)
    y = z[:, :T] + torch.randn(n, T, v, generator=g)
    # drafts as their own distribution gives them, or the target's best
    q = torch.softmax(y.double() / max(temp, 0.5), 2)
    x = (torch.multinomial(q.view(-1, v), 1, generator=g).view(n, T) if T else torch.zeros(n, 0)).to(torch.int32)
    x = torch.where(torch.rand(n, T, generator=g) < 0.5, z[:, :T].argmax(2).to(torch.int32), x)
    count = torch.randint(0, T + 1, (n,), generator=g, dtype=torch.int32)
    u = torch.rand(n, T + 1, generator=g)
    check(sevo, z, x, u, temp, y if dist else None)
    check(sevo, z, x, u, temp, y if dist else None, count)


def test_counts_outside_and_bad_drafts(sevo):
    g = gen(1)
    z = rows(6, 3, 500, g)
    y = rows(6, 2, 500, g)
    x = torch.tensor([[-1, 3], [500, 3], [1, 2], [2 ** 31 - 1, 0], [5, -2 ** 31], [7, 8]], dtype=torch.int32)
    count = torch.tensor([2, 2, -3, 9, 2, 2 ** 31 - 1], dtype=torch.int32)
    u = torch.rand(6, 3, generator=g)
    u[:, 0] = 0
    check(sevo, z, x, u, 1.0, None, count)
    check(sevo, z, x, u, 1.0, y, count)
    check(sevo, z, x, u, 0.0, y, count)


def test_edges_of_the_uniform_numbers(sevo):
    g = gen(2)
    z = rows(4, 2, 5000, g)
    z[:, :, 4990:] = -math.inf               # the last entries have no probability
    z[1, :, :7] = -math.inf
    x = z[:, :1].argmax(2).to(torch.int32)
    for last in (0.0, 1.0 - 2.0 ** -24, 1.0):
        for first in (0.0, 1.0):
            u = torch.full((4, 2), last)
            u[:, 0] = first
            tok, _, _ = check(sevo, z, x, u, 1.0)
            check(sevo, z, x, u, 1.0, z[:, :1])
            assert (tok < 4990).all()


def test_drafts_from_the_target_are_always_taken(sevo):
    g = gen(3)
    z = rows(8, 5, 3001, g)
    p = torch.softmax(z[:, :4].double(), 2).view(-1, 3001)
    x = torch.multinomial(p, 1, generator=g).view(8, 4).to(torch.int32)
    _, _, taken = check(sevo, z, x, torch.rand(8, 5, generator=g), 1.0, z[:, :4])
    assert (taken == 4).all()


def test_nothing_left_of_the_residual(sevo):
    """A rejected draft whose distribution is the target's own, and certain drafts that are."""
    z = torch.zeros(3, 2, 640)
    z[1, 0] = -math.inf
    z[1, 0, 99] = 2.0                        # all of the mass at 99, drafted and refused (u = 1)
    z[2, 0, 5] = math.inf                    # no distribution
    x = torch.tensor([[4], [99], [5]], dtype=torch.int32)
    u = torch.tensor([[1.0, 0.5], [1.0, 0.5], [0.0, 0.5]])
    tok, lp, taken = check(sevo, z, x, u, 1.0, z[:, :1])
    assert taken.tolist() == [0, 0, 0] and tok[1, 0] == 99 and tok[2, 0] == -1
    check(sevo, z, x, u, 1.0)


@pytest.mark.parametrize("temp", [0.0, 1.0])
def test_rows_that_are_no_distribution(sevo, temp):
    g = gen(4)
    z = rows(6, 3, 9000, g)
    z[0, 0, 8999] = math.nan
    z[1, 1] = -math.inf
    z[2, 2, 17] = math.inf
    z[3, :, 100:] = -math.inf
    y = rows(6, 2, 9000, g)
    y[4, 0, 3] = math.nan
    y[5, 1] = -math.inf
    x = z[:, :2].nan_to_num(0, 0).argmax(2).to(torch.int32)
    u = torch.rand(6, 3, generator=g) * 0.01
    tok, _, _ = check(sevo, z, x, u, temp, y)
    assert tok[0, 0] == -1
    check(sevo, z, x, u, temp)


def test_ties_go_to_the_lowest_index(sevo):
    z = torch.zeros(2, 3, 12289)
    z[0, 0, [4095, 4096, 9000]] = 3.0
    z[1, 1, [12288, 8191]] = 1.0
    x = torch.tensor([[4095, 0], [0, 12288]], dtype=torch.int32)
    tok, _, taken = check(sevo, z, x, torch.zeros(2, 3), 0.0)
    assert taken.tolist() == [2, 1] and tok[0].tolist() == [4095, 0, 0] and tok[1].tolist() == [0, 8191, -1]


def test_large_magnitudes(sevo):
    g = gen(5)
    z = rows(3, 3, 700, g) * 1e4
    z[1] *= 1e30
    x = z[:, :2].argmax(2).to(torch.int32)
    check(sevo, z, x, torch.rand(3, 3, generator=g), 1.0, z[:, :2] * 0.5)
    check(sevo, z, x, torch.rand(3, 3, generator=g), 1e-3)


def test_emitted_tokens_follow_the_target(sevo):
    """First emitted tokens over a grid of uniform numbers: each entry's share is its
    target probability.  The drafts take their distribution's shares exactly, the grid has 64 x 64
    points for each, so a share is off by at most its border cells: 2 / 64 for each of the
    two comparisons."""
    v, k = 6, 64
    g = gen(6)
    z, y = torch.randn(1, 2, v, generator=g), torch.randn(1, 1, v, generator=g)
    p, q = torch.softmax(z[0, 0].double(), 0), torch.softmax(y[0, 0].double(), 0)
    grid = (torch.arange(k) + 0.5) / k
    u = torch.stack(torch.meshgrid(grid, grid, indexing="ij"), 2).view(-1, 2)
    share = torch.zeros(v, dtype=torch.float64)
    for x in range(v):
        n = u.shape[0]
        tok, _, _ = sevo.sevo_verify_drafts(padded(z.expand(n, 2, v)), torch.full((n, 1), x, dtype=torch.int32, device=DEV),
                                            u.to(DEV), 1.0, draft_logits=padded(y.expand(n, 1, v)), vocab=v)
        share += q[x] * torch.bincount(tok[:, 0].long().cpu(), minlength=v).double() / n
    assert (share - p).abs().max() <= 4 / k


def test_without_drafts_it_is_a_sample(sevo):
    """T = 0 in several layouts: one row of a wider buffer, a strided batch."""
    g = gen(7)
    buf = torch.randn(4, 1030, generator=g).to(DEV)
    u = torch.rand(4, 1, generator=g).to(DEV)
    none = torch.zeros(4, 0, dtype=torch.int32, device=DEV)
    wide = torch.empty(4, 1032, device=DEV)
    wide[:, :1030] = buf
    a = sevo.sevo_verify_drafts(wide[:, None], none, u, 1.0, vocab=1030)
    for i in range(4):
        b = sevo.sevo_verify_drafts(wide[i:i + 1, None, :1030], none[:1], u[i:i + 1].contiguous(), 1.0)
        assert [int(b[0]), float(b[1])] == [int(a[0][i]), float(a[1][i])]
    with pytest.raises(sevo.SevoError):
        sevo.sevo_verify_drafts(buf[:, None], none, u, 1.0)       # rows 1030 apart: no multiple of 4


@pytest.mark.parametrize("dist", [False, True])
def test_in_graphs_with_other_rows(sevo, dist):
    """Captured once, replayed with other logits, drafts, counts and uniform numbers; two graphs on one
    workspace."""
    g = gen(13)
    n, T, v = 5, 3, 9001
    ws = torch.empty(sevo.sevo_verify_workspace_bytes(n, T, v), dtype=torch.uint8, device=DEV)
    sets = []
    for _ in range(3):
        z, y = rows(n, T + 1, v, g), rows(n, T, v, g)
        x = z[:, :T].argmax(2).to(torch.int32)
        x[0] = torch.randint(0, v, (T,), generator=g).to(torch.int32)
        sets.append([padded(z), padded(y), x.to(DEV), torch.rand(n, T + 1, generator=g).to(DEV),
                     torch.randint(0, T + 2, (n,), generator=g).to(torch.int32).to(DEV)])
    def call(s, **k):
        return sevo.sevo_verify_drafts(s[0], s[2], s[3], 0.9, draft_logits=s[1] if dist else None, n_drafts=s[4], vocab=v, **k)
    want = [[t.clone() for t in call(s)] for s in sets]
    held = [[t.clone() for t in s] for s in sets[:2]]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(s, workspace=ws))
        graphs.append(graph)
    for rep in range(3):
        for k in range(2):
            for t, x in zip(held[k], sets[(rep + k) % 3]):
                t.copy_(x)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[k], want[(rep + k) % 3]))
        assert all(torch.equal(a, b) for a, b in zip(call(sets[rep]), want[rep]))
