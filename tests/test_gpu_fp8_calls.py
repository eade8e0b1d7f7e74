"""GPU tests of calls of the 8-bit layer that tests/test_gpu_fp8.py does not make:
explicit streams, routers with large biases, entries without an expert, the
accuracy of the 8-bit sums, and a layer around its attention.  Its tolerances and
helpers are those of that file."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import say
from tests.test_gpu_fp8 import (BF, F8, TOP, check_codes, check_product, gen, normal, quantised,  # noqa: F401
                                sevo, weights)

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


# ------------------------------------------------------------------ routing
def route64(logits, top_k, score, bias, groups, top_groups, best):
    """(experts, weights) by the definition in float64 (numpy, all tokens at once)."""
    z = logits.astype(np.float64)
    n, E = z.shape
    if score == "sigmoid":
        p = 1 / (1 + np.exp(-z))
    else:
        p = np.exp(z - z.max(1, keepdims=True))
        p = p / p.sum(1, keepdims=True)
    c = p if bias is None else p + bias.astype(np.float64)
    gs = -np.sort(-c.reshape(n, groups, E // groups), axis=2)[:, :, :best].sum(2)
    kept = np.argsort(-gs, axis=1, kind="stable")[:, :top_groups]
    keep = np.zeros((n, groups), bool)
    np.put_along_axis(keep, kept, True, 1)
    c = np.where(np.repeat(keep, E // groups, 1), c, -np.inf)
    ex = np.argsort(-c, axis=1, kind="stable")[:, :top_k]
    w = np.take_along_axis(p, ex, 1)
    return ex, w / (w.sum(1, keepdims=True) + 1e-20)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [3.0, 300.0, 1e4, 1e6, 1e9])
def test_moe_route_large_biases(sevo, score, size):
    """Each group has one expert with a large bias and the rest with its negative:
    the sum of its two best is as small as the scores, and the float32 sum is off by
    the rounding of the biases.  Beside them one group that is switched off by a
    large negative bias.  The three experts with the large bias of the groups kept
    stand apart from all others, so that the groups alone decide."""
    n, E, groups, top_groups, top_k = 3000, 128, 8, 3, 3
    rng = np.random.default_rng(int(size))
    # scores near each other: groups a few float32 steps of the bias apart, and less
    spread = 1.0 if size < 10 else min(1.0, size * (2e-6 if score == "sigmoid" else 5e-5))
    z = (0.3 + rng.normal(0, spread, (n, E))).astype(np.float32)
    bias = np.full(E, -size, np.float32)
    # (each in another place of its lane's eight: no two of them have the same key)
    bias[np.arange(groups) * (E // groups) + [0, 9, 2, 11, 4, 13, 6, 15]] = size
    bias[-E // groups:] = -3 * size
    ex, wt = sevo.sevo_moe_route(torch.from_numpy(z).cuda(), top_k, score, torch.from_numpy(bias).cuda(),
                                 groups, top_groups, 2, True, 1.0)
    rex, rwt = route64(z, top_k, score, bias, groups, top_groups, 2)
    wrong = int((np.sort(ex.cpu().numpy() * groups // E, 1) != np.sort(rex * groups // E, 1)).any(1).sum())
    assert wrong == 0, f"{wrong} of {n} tokens in other groups"
    np.testing.assert_array_equal(ex.cpu().numpy(), rex)
    np.testing.assert_allclose(wt.cpu().numpy(), rwt, rtol=2.0 ** -23)


def test_moe_route_nan_is_last(sevo):
    """A NaN is chosen after every other value, experts that a bias of -inf has
    switched off among them; a group without a value after those with one."""
    nan, inf = float("nan"), float("inf")
    z = torch.tensor([[nan, 0.0, 2.0, 1.0, 0.5, nan, 0.25, -1.0]], device="cuda")
    bias = torch.tensor([0, 0, 0, -inf, 0, 0, 0, 0], device="cuda")
    for top_k, want in ((5, [2, 4, 6, 1, 7]), (6, [2, 4, 6, 1, 7, 3]), (8, [2, 4, 6, 1, 7, 3, 0, 5])):
        ex, wt = sevo.sevo_moe_route(z, top_k, "sigmoid", bias, renormalise=False)
        assert ex[0].tolist() == want, ex[0].tolist()
        assert torch.isnan(wt[0, 6:]).all() and torch.isfinite(wt[0, :6]).all()
    # groups of two: 0's sum is +inf - inf, 1's -inf, 2's and 3's finite
    bias = torch.tensor([inf, -inf, -inf, 0, 0, 0, 0, 0], device="cuda")
    ex, _ = sevo.sevo_moe_route(torch.zeros(1, 8, device="cuda"), 6, "sigmoid", bias, 4, 3, 2, False)
    assert sorted(ex[0].tolist()) == [2, 3, 4, 5, 6, 7]


# ------------------------------------------------------------------ experts
@pytest.mark.parametrize("n,E,top_k,n_out,k", [
    (3, 8, 2, 192, 128), (40, 64, 4, 64, 256), (300, 16, 4, 320, 256), (900, 16, 4, 4160, 128),
    (9000, 16, 8, 192, 128)])
@pytest.mark.parametrize("share", [0.0, 0.3, 1.0])
def test_moe_linear_fp8_unlisted_rows(sevo, n, E, top_k, n_out, k, share):
    """Entries without an expert, as a rank that holds some of the experts has them:
    without ``out`` their rows are zero in memory that was not, all other rows as they
    are with it, and the next norm can add the planes."""
    say(f"unlisted n={n} E={E} top {top_k} {n_out} x {k} share {share}")
    g = gen(n + E)
    ex = torch.randint(0, E, (n, top_k), device="cuda", dtype=torch.int32, generator=g)
    drop = torch.rand((n, top_k), device="cuda", generator=g) < share
    bad = torch.tensor([-1, E, -2 ** 31, 2 ** 31 - 1], device="cuda", dtype=torch.int32)
    ex = torch.where(drop, bad[torch.randint(0, 4, (n, top_k), device="cuda", generator=g)], ex)
    wt = torch.rand((n, top_k), device="cuda", generator=g)
    wq, ws = weights((E, n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    lists = sevo.sevo_moe_lists(ex, E)
    for down in (False, True):
        xq, xs = quantised(normal((n * top_k if down else n, k), g))
        kw = dict(weights=wt) if down else {}
        shape = (top_k, n, n_out) if down else (n * top_k, n_out)
        given = torch.full(shape, float("nan"), dtype=BF, device="cuda")
        sevo.sevo_moe_linear_fp8(xq, xs, w, ws, lists, out=given, **kw)
        rows = drop.t() if down else drop.reshape(-1)
        assert torch.isnan(given[rows]).all() and torch.isfinite(given[~rows]).all()
        dirty = torch.full(shape, float("nan"), dtype=BF, device="cuda")
        at = dirty.data_ptr()
        del dirty
        y = sevo.sevo_moe_linear_fp8(xq, xs, w, ws, lists, **kw)
        say(f"  the same memory: {y.data_ptr() == at}")
        assert (y[rows] == 0).all() and torch.equal(y[~rows], given[~rows])
    parts = torch.nn.functional.pad(y, (0, -n_out % 128)).contiguous()
    x = normal((n, parts.shape[2]), g)
    want = x.clone()
    for p in parts:
        want = want + p.float()
    sevo.sevo_add_rmsnorm_fp8(x, parts, torch.ones(parts.shape[2], dtype=BF, device="cuda"), 1e-6)
    assert torch.equal(x, want)


# ------------------------------------------------------------------ one row
def test_one_row_of_any_buffer(sevo):
    """One token out of buffers whose rows are an odd number of bytes apart."""
    g = gen(12)
    n_out, k, E = 192, 256, 4
    wq, ws = weights((E, n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    xq, xs = quantised(normal((1, k), g))
    x = torch.zeros(3, k + 8, device="cuda").to(F8)
    x[:1, :k] = xq
    out = torch.full((3, n_out + 1), 7.0, dtype=BF, device="cuda")
    sevo.sevo_linear_fp8(x[:1, :k], xs, w[0], ws[0], out=out[:1, :n_out])
    check_product(out[:1, :n_out], xq, xs, wq[0], ws[0])
    assert (out[1:] == 7.0).all() and (out[0, n_out:] == 7.0).all()
    y = sevo.sevo_moe_linear_fp8(x[:1, :k], xs, w, ws,
                                 sevo.sevo_moe_lists(torch.tensor([[2, 1]], device="cuda", dtype=torch.int32), E))
    for j, e in enumerate((2, 1)):
        check_product(y[j:j + 1], xq, xs, wq[e], ws[e])
    rows = normal((3, 2 * k + 3), g, 1.0, BF)
    q, s = sevo.sevo_quantize_fp8(rows[:1, :2 * k], swiglu=True)
    u = rows[:1, :2 * k].double()
    check_codes(q, s, u[:, :k] / (1 + torch.exp(-u[:, :k])) * u[:, k:], rel=64 * 2.0 ** -24)
    z = normal((2, 9), g)
    ex, _ = sevo.sevo_moe_route(z[:1, :8], 3)
    assert ex[0].tolist() == torch.sort(z[0, :8], descending=True)[1][:3].tolist()


# ------------------------------------------------------------------ accuracy of the 8-bit sums
def exponent(v):
    """Exponents of e4m3 values, those of subnormal ones (and 0) as -6."""
    return torch.frexp(v)[1].double().sub(1).clamp_min(-6)


def block_sums(X, W):
    """(exact, as the 8-bit instructions add, sum of magnitudes, largest products of
    the groups of eight) of one block's rows X [m, 128], W [n, 128] (float64)."""
    p = (X[:, None] * W[None]).view(X.shape[0], W.shape[0], 16, 8)
    e = (exponent(X)[:, None] + exponent(W)[None]).view_as(p)
    unit = torch.exp2(torch.where(p == 0, -18.0, e).amax(3, keepdim=True) - 13)
    return (p.sum((2, 3)), (torch.trunc(p / unit) * unit).sum((2, 3)), p.abs().sum((2, 3)),
            (unit * 2.0 ** 13).sum((2, 3)))


def codes_of(kind, rows, k, g):
    v = normal((rows, k), g)
    if kind == "one sign":
        v = v.abs()
    elif kind == "wide":
        v = v * torch.exp(3 * normal((rows, k), g))
    elif kind == "small":                           # most codes subnormal
        v = v * torch.where(torch.rand((rows, k), device="cuda", generator=g) < 0.1, 1.0, 2.0 ** -15)
    return (v / v.abs().amax(1, keepdim=True) * TOP).to(F8)


def cancel(X, W):
    """W with its last 16 columns of each row changed so that the products with the
    same row of X nearly cancel."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(F8).float()
    codes = codes[torch.isfinite(codes)].double()
    x, w = X[:W.shape[0]].double(), W.double()[:X.shape[0]]
    for j in range(x.shape[1] - 16, x.shape[1]):
        rest = (x * w).sum(1) - x[:, j] * w[:, j]
        w[:, j] = codes[(rest[:, None] + x[:, j:j + 1] * codes).abs().argmin(1)]
    W = W.clone()
    W[:w.shape[0]] = w.float().to(F8)
    return W


@pytest.mark.parametrize("kind", ["normal", "one sign", "wide", "small"])
@pytest.mark.parametrize("m,n_out,E", [(5, 64, 0), (64, 256, 0), (2048, 1024, 0), (6, 128, 4), (700, 256, 4)])
def test_sums_of_one_block(sevo, kind, m, n_out, E):
    """What the header says of the inner sums, on one block (its scales 1), sums that
    cancel among them: within the bound of the exact sum, and the sum of the cut
    products to 2^-20 of the magnitudes (sixteen groups and the stages that join
    them, each to about 2^-24 of the largest); fp32 results exact to fp32 rounding."""
    say(f"one block {kind} m={m} n_out={n_out} E={E}")
    g = gen(m + n_out)
    k = 128
    X8 = codes_of(kind, m, k, g)
    W8 = codes_of(kind, max(E, 1) * n_out, k, g).view(max(E, 1), n_out, k)
    W8 = torch.stack([cancel(X8, w) for w in W8])
    w = sevo.sevo_pack_weight_fp8(W8)
    xs = torch.ones(1, m, device="cuda")
    ws = torch.ones(max(E, 1), -(-n_out // 128), 1, device="cuda")
    rows = torch.arange(0, m, max(1, m // 48), device="cuda")
    if E:
        ex = (torch.arange(m, device="cuda") % E).to(torch.int32).view(m, 1)
        out = {BF: sevo.sevo_moe_linear_fp8(X8, xs, w, ws, sevo.sevo_moe_lists(ex, E))}
    else:
        out = {t: sevo.sevo_linear_fp8(X8, xs, w[0], ws[0], out_dtype=t) for t in (BF, torch.float32)}
    worst = 0.0
    for e in range(max(E, 1)):
        r = rows[rows % E == e] if E else rows
        if not r.numel():
            continue
        exact, cut, mag, largest = block_sums(X8[r].double(), W8[e].double())
        for t, y in out.items():
            err = (y[r].double() - exact).abs()
            if t == BF:
                near = (y[r].double() - cut).abs()
                assert (near <= cut.abs() * 2.0 ** -8 + mag * 2.0 ** -20).all(), "not the sum of the cut products"
                assert (err <= exact.abs() * 2.0 ** -8 + 7 * 2.0 ** -13 * largest + mag * 2.0 ** -20).all()
                worst = max(worst, float(((err - exact.abs() * 2.0 ** -8) / mag).max()))
            else:
                assert (err <= mag * 144 * 2.0 ** -24).all()
    say(f"  furthest off: {worst:.1e} of the sum of magnitudes")


# ------------------------------------------------------------------ a layer around its attention
@pytest.mark.parametrize("n", [1, 24, 300])
def test_attention_half_of_a_layer(sevo, n):
    """Norm, fp32 QKV product, QK norm + RoPE + append, paged attention, quantiser, output
    projection, and the norm that adds it: each stage against float64 on what the
    stage before it gave, and in a graph replayed between eager work."""
    import oracle.decoder as od
    from paper_2604_07725_amd import device_inputs as di, synth
    from tests.gpu_helpers import ATTN_REL_TOL, make_population, to_np
    say(f"attention half n={n}")
    hq, hkv, d, H = 8, 2, 128, 512
    shape = synth.ModelShape(1, H, hq, hkv, d, 256, 256)
    pop = make_population(np.random.default_rng(n).integers(0, 200, size=n), shuffle=True, seed=4, extra=1)
    tensors = di.device_weights(shape, 5)
    model = sevo.sevo_init_model(shape, tensors, max_position=256)
    pos = torch.from_numpy(pop.lengths.astype(np.int32)).cuda()
    pt = torch.from_numpy(pop.page_table.astype(np.int32)).cuda()
    pool0 = di.device_pools(shape, 5, pop.n_pages)[0]
    g = gen(n)
    wqkv, wo = weights(((hq + 2 * hkv) * d, H), g), weights((H, hq * d), g)
    pqkv, po = sevo.sevo_pack_weight_fp8(wqkv[0]), sevo.sevo_pack_weight_fp8(wo[0])
    gain = normal((H,), g, 0.1, BF) + 1
    x0 = normal((n, H), g, 2.0)

    def half(x, pool):
        q8, s8 = sevo.sevo_add_rmsnorm_fp8(x, None, gain, 1e-6)
        qkv = sevo.sevo_linear_fp8(q8, s8, pqkv, wqkv[1], out_dtype=torch.float32)
        q = sevo.sevo_qk_norm_rope_append(model, 0, qkv, pos, pt, pool)
        o = sevo.sevo_attn_decode(q, pool, pt, pos + 1)
        a8, sa = sevo.sevo_quantize_fp8(o.view(n, hq * d))
        y = sevo.sevo_linear_fp8(a8, sa, po, wo[1])
        h8, sh = sevo.sevo_add_rmsnorm_fp8(x, y.unsqueeze(0), gain, 1e-6)
        return q8, s8, qkv, q, o, a8, sa, y, h8, sh

    x, pool = x0.clone(), pool0.clone()
    q8, s8, qkv, q, o, a8, sa, y, h8, sh = half(x, pool)
    check_product(qkv, q8, s8, *wqkv)
    # bf16 of values whose angles and norms are in fp32: half a step and 2^-16 of the head's largest
    lw = {k: to_np(v) for k, v in tensors["layers"][0].items() if k in ("q_norm", "k_norm")}
    heads = to_np(qkv).reshape(n, hq + 2 * hkv, d)
    p = pop.lengths.astype(np.int64)[:, None]
    want = od.rope_rotate(od.rms_norm(heads[:, :hq], lw["q_norm"], shape.rms_eps), p, shape.rope_theta)
    big = np.abs(want).max(-1, keepdims=True)
    assert np.all(np.abs(to_np(q) - want) <= np.abs(want) * 2.0 ** -8 + big * 2.0 ** -16)
    kw = od.rope_rotate(od.rms_norm(heads[:, hq:hq + hkv], lw["k_norm"], shape.rms_eps), p, shape.rope_theta)
    hpool = to_np(pool)
    ref = np.empty((n, hq, d))
    for i in range(n):
        K, V = od.gather_kv(hpool, pop.page_table[i], int(pop.lengths[i]) + 1)
        big = np.abs(kw[i]).max(-1, keepdims=True)
        assert np.all(np.abs(K[:, -1] - kw[i]) <= np.abs(kw[i]) * 2.0 ** -8 + big * 2.0 ** -16)
        v = heads[i, hq + hkv:]
        assert np.all(np.abs(V[:, -1] - v) <= np.abs(v) * 2.0 ** -8)
        ref[i] = od.attention_dense(to_np(q[i]), K, V, d ** -0.5)
    err = np.abs(to_np(o) - ref).max((1, 2)) / np.abs(ref).max((1, 2))
    assert err.max() <= ATTN_REL_TOL
    check_codes(a8, sa, o.view(n, hq * d).double(), rel=4 * 2.0 ** -24)
    check_product(y, a8, sa, *wo)
    assert torch.equal(x, x0 + y.float())
    xd = x.double()
    check_codes(h8, sh, xd / (xd.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * gain.double(), rel=64 * 2.0 ** -24)
    # in a graph
    xg, poolg = x0.clone(), pool0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xg.copy_(x0)
        got = half(xg, poolg)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(xg, x) and torch.equal(poolg.view(torch.int16), pool.view(torch.int16))
        for a, b in zip(got, (q8, s8, qkv, q, o, a8, sa, y, h8, sh)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        half(x0.clone(), pool0.clone())                       # eager work between
    torch.cuda.synchronize()
    model.close()


def test_stream_arguments_in_a_graph(sevo):
    """A capture that forks to a stream of its own and joins it: what the calls there
    allocate is the graph's, and every replay gives the eager bits."""
    g = gen(32)
    m, n_out, k = 48, 512, 12288
    assert sevo.sevo_linear_fp8_workspace_bytes(m, n_out, k) > 0
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    x = normal((m, k), g, 1.0, BF)
    side = torch.cuda.Stream()

    def both(s):
        here = torch.cuda.current_stream()
        s.wait_stream(here)
        a = sevo.sevo_linear_fp8(*sevo.sevo_quantize_fp8(x, stream=s), w, ws, stream=s)
        b = sevo.sevo_linear_fp8(*sevo.sevo_quantize_fp8(-x), w, ws)
        here.wait_stream(s)
        return a, b, a.float() + b.float()

    want = [t.clone() for t in both(side)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(side)
    for turn in range(4):
        x.copy_(normal((m, k), gen(turn), 1.0, BF))
        graph.replay()
        torch.cuda.synchronize()
        want = [t.clone() for t in both(side)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn


def test_default_stream_by_its_handle(sevo):
    x = normal((8, 256), gen(2), 1.0, BF)
    want = sevo.sevo_quantize_fp8(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = sevo.sevo_quantize_fp8(x, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])
    assert stream_of(got[0]) == 0
