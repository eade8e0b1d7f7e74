"""GPU tests of the 8-bit layer: norm, quantiser, packed weights, block-scaled
products, routing, the experts' products, and a layer of them together, each
against its definition in float64.

Tolerances count roundings.  e4m3 is off by at most half a step: 2^-4 relative,
2^-10 below its smallest normal value 2^-6.  bf16 2^-8, fp32 2^-24.  A product kept
in fp32 sees at most 128 additions in a block, one per block and a few across
waves and splits; in bf16 mode the 8-bit matrix instruction holds a block's sum
to 2^-15 of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import poisoned, say

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
BF = torch.bfloat16
TOP, LEAST = 448.0, 2.0 ** -64


@pytest.fixture(scope="module")
def sevo():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_07725_amd import sevo
    sevo.lib()
    return sevo


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, g, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, device="cuda", generator=g) * std).to(dtype)


def quantised(y):
    """Row-wise operands of the products: fp32 [m, k] -> codes, scales [k/128, m]."""
    m, k = y.shape
    yb = y.view(m, k // 128, 128)
    s = (yb.abs().amax(2) / TOP).clamp_min(LEAST)
    return (yb / s[:, :, None]).view(m, k).to(F8), s.t().contiguous()


def weights(shape, g):
    """Codes [..., n, k] and scales [..., ceil(n/128), k/128] of N(0, 0.02) weights."""
    *lead, n, k = shape
    w = normal((*lead, -(-n // 128) * 128, k), g, 0.02)
    wb = w.view(*lead, -1, 128, k // 128, 128)
    s = wb.abs().amax((-3, -1)) / TOP
    q = (wb / s[..., :, None, :, None]).view(*lead, -1, k)[..., :n, :].to(F8)
    return q.contiguous(), s.contiguous()


def values(q, s):
    """float64 values of activations."""
    m, k = q.shape
    return (q.float().double().view(m, k // 128, 128) * s.double().t()[:, :, None]).view(m, k)


def weight_values(q, s):
    n, k = q.shape
    return q.float().double() * s.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)


def check_codes(q, s, y, rel=1e-5, label=""):
    """Codes q [m, k] and scales s [k/128, m] of the float64 rows y, computed in
    fp32 to the relative error ``rel``."""
    m, k = y.shape
    yb = y.view(m, k // 128, 128)
    bad = ~torch.isfinite(yb).all(2)                       # blocks with a NaN or an infinity
    ref = (yb.abs().amax(2) / TOP).clamp_min(LEAST)
    st = s.double().t()
    assert torch.equal(torch.isnan(st), bad), f"{label}: NaN scales"
    assert torch.isnan(q.float().view(m, k // 128, 128)[bad]).all(), f"{label}: NaN codes"
    ok = ~bad
    err = ((st - ref).abs() / ref)[ok]
    assert err.numel() == 0 or err.max() <= rel, f"{label}: scales {err.max():.2e}"
    v = (yb / st[:, :, None])[ok]
    c = q.float().double().view(m, k // 128, 128)[ok]
    tol = torch.maximum(v.abs() * 2.0 ** -4, torch.full_like(v, 2.0 ** -10)) * (1 + 1e-6) + \
        v.abs() * rel
    assert ((c - v).abs() <= tol).all(), f"{label}: codes off by {((c - v).abs() / tol).max():.3f} tolerances"


# ------------------------------------------------------------------ packed weights
@pytest.mark.parametrize("shape", [(64, 128), (192, 384), (3, 128, 256)])
def test_pack_weight_layout(sevo, shape):
    g = gen(1)
    src = torch.randint(0, 255, shape, device="cuda", dtype=torch.uint8, generator=g)
    dst = sevo.sevo_pack_weight_fp8(src.view(F8)).view(torch.uint8).cpu().numpy().ravel()
    w = src.cpu().numpy().reshape(-1, shape[-1])
    r, c = np.arange(w.shape[0])[:, None], np.arange(w.shape[1])[None, :]
    off = (((r // 64) * (w.shape[1] // 128) + c // 128) * 4 + (r // 16) % 4) * 2048 + \
        (16 * ((c // 16) % 8) + r % 16) * 16 + c % 16
    np.testing.assert_array_equal(dst[off], w)


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("rows,cols,S,ptype", [
    (1, 128, 0, BF), (3, 256, 1, BF), (1, 4096, 1, BF), (37, 4096, 2, torch.float32),
    (130, 2048, 8, BF), (5, 12288, 16, torch.float32), (2, 8320, 3, BF), (2, 32768, 1, BF),
    (301, 640, 4, torch.float32), (1025, 1024, 5, BF)])
def test_add_rmsnorm_fp8(sevo, rows, cols, S, ptype):
    say(f"norm {rows} x {cols}, {S} partials {ptype}")
    g = gen(rows + cols)
    x = normal((rows, cols), g, 2.0)
    x[:, cols // 3] *= 50.0
    if rows > 2:
        x[1] = 0.0                                  # a zero row: zero codes, the least scale
        x[2, 64:192] *= 1e-30                       # part of a block and of the next one tiny
    parts = normal((S, rows, cols), g, 0.5, ptype) if S else None
    if S and rows > 2:
        parts[:, 1] = 0.0
    gain = normal((cols,), g, 0.1, BF) + 1
    x0 = x.clone()
    nb = torch.full((rows, cols), float("nan"), device="cuda", dtype=BF)
    q, s = sevo.sevo_add_rmsnorm_fp8(x, parts, gain, 1e-6, out_bf16=nb)
    want = x0
    for p in range(S):
        want = want + parts[p].float()              # fp32, in order
    assert torch.equal(x, want)
    xd = want.double()
    y = xd / (xd.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * gain.double()
    # the fp32 sum of squares and its square root: 32 roundings at most per thread and tree
    check_codes(q, s, y, rel=64 * 2.0 ** -24)
    assert ((nb.double() - y).abs() <= y.abs() * (2.0 ** -8 + 64 * 2.0 ** -24)).all()
    # alone, a row gives the same bits
    r = rows // 2
    xr = x0[r:r + 1].clone()
    q1, s1 = sevo.sevo_add_rmsnorm_fp8(xr, None if parts is None else parts[:, r:r + 1].contiguous(),
                                       gain, 1e-6)
    assert torch.equal(q1.view(torch.uint8), q[r:r + 1].view(torch.uint8))
    assert torch.equal(s1[:, 0], s[:, r])


def test_add_rmsnorm_fp8_not_finite(sevo):
    g = gen(5)
    x = normal((4, 512), g)
    x[1, 200] = float("nan")
    x[2, 300] = float("inf")
    gain = torch.ones(512, device="cuda", dtype=BF)
    q, s = sevo.sevo_add_rmsnorm_fp8(x, None, gain, 1e-6)
    assert torch.isfinite(s[:, 0]).all() and torch.isfinite(s[:, 3]).all()
    assert torch.isnan(s[:, 1]).all()               # the NaN reaches the whole row's norm
    assert torch.isnan(s[2, 2]) and torch.isfinite(s[[0, 1, 3], 2]).all()   # inf * 0 in its block
    assert (q[2, :256].float() == 0).all()


# ------------------------------------------------------------------ quantiser
@pytest.mark.parametrize("m,k,swiglu,pad", [(1, 128, False, 0), (64, 4096, False, 0), (3, 640, True, 0),
                                            (129, 12288, True, 16), (4001, 2048, False, 8),
                                            (2053, 4224, True, 0), (1, 25600, True, 0)])
def test_quantize_fp8(sevo, m, k, swiglu, pad):
    say(f"quantise {m} x {k} swiglu {swiglu}")
    g = gen(m + k)
    cols = k * (2 if swiglu else 1)
    x = normal((m, cols + pad), g, 3.0, BF)[:, :cols]
    x[0, :128] = 0.0
    if m > 2:
        x[1, 5] = float("nan")
        x[2, 7] = float("inf")
        x[2, 128:256] *= 1e-20
    q, s = sevo.sevo_quantize_fp8(x, swiglu=swiglu)
    y = x.double()
    rel = 4 * 2.0 ** -24
    if swiglu:
        gate, up = y[:, :k], y[:, k:]
        y = gate / (1 + torch.exp(-gate)) * up
        rel = 64 * 2.0 ** -24                       # exp of |g| up to 14: its argument's rounding
    check_codes(q, s, y, rel=rel)


# ------------------------------------------------------------------ products
def check_product(y, xq, xs, wq, ws, label=""):
    X, W = values(xq, xs), weight_values(wq, ws)
    ref = X @ W.t().contiguous()
    mag = X.abs() @ W.abs().t().contiguous()
    k = X.shape[1]
    if y.dtype == torch.float32:
        tol = mag * (128 + k // 128 + 16) * 2.0 ** -24
    else:
        tol = ref.abs() * 2.0 ** -8 + mag * 2.0 ** -15
    err = (y.double() - ref).abs()
    assert (err <= tol).all(), f"{label}: {(err / tol.clamp_min(1e-300)).max():.2f} tolerances"
    return float((err.norm() / ref.norm().clamp_min(1e-300)))


SHAPES = [(1, 64, 128), (1, 6144, 4096), (2, 256, 1024), (5, 4096, 12288), (16, 6144, 4096),
          (17, 192, 384), (33, 64, 25600), (48, 1088, 640), (64, 4096, 4096), (65, 448, 256),
          (100, 5120, 2048), (128, 64, 128), (129, 320, 1152), (203, 5120, 8192), (255, 2048, 4096),
          (256, 256, 128), (300, 24576, 256), (513, 576, 640), (1000, 4096, 4096), (2049, 1024, 512)]


@pytest.mark.parametrize("m,n_out,k", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_linear_fp8(sevo, m, n_out, k, dtype):
    say(f"product {m} x {n_out} x {k} {dtype}")
    g = gen(m * 7 + n_out + k)
    x = normal((m, k), g)
    x[:, k // 2] *= 30.0
    xq, xs = quantised(x)
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    need = sevo.sevo_linear_fp8_workspace_bytes(m, n_out, k)
    y = sevo.sevo_linear_fp8(xq, xs, w, ws, out_dtype=dtype, workspace=poisoned(need))
    rel = check_product(y, xq, xs, wq, ws, f"{m} x {n_out} x {k}")
    say(f"  rel {rel:.2e}")
    again = sevo.sevo_linear_fp8(xq, xs, w, ws, out_dtype=dtype)
    assert torch.equal(y, again)


@pytest.mark.parametrize("m", [3, 64, 90, 300])
def test_linear_fp8_strides(sevo, m):
    """Rows of x, its scales and the output inside larger buffers: the right rows
    are read, nothing beside the output is written."""
    g = gen(m)
    n_out, k = 192, 384
    xq, xs = quantised(normal((m, k), g))
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    xb = torch.full((m, k + 48), 0x7F, dtype=torch.uint8, device="cuda")
    xb[:, 16:16 + k] = xq.view(torch.uint8)
    sb = torch.full((k // 128, m + 5), float("nan"), device="cuda")
    sb[:, 3:3 + m] = xs
    for dtype in (torch.float32, BF):
        ob = torch.full((m + 2, n_out + 12), 7.0, dtype=dtype, device="cuda")
        sevo.sevo_linear_fp8(xb.view(F8)[:, 16:16 + k], sb[:, 3:3 + m], w, ws, out=ob[:m, 8:8 + n_out]
                             if dtype == BF else ob[:m, 4:4 + n_out])
        c0 = 8 if dtype == BF else 4
        check_product(ob[:m, c0:c0 + n_out], xq, xs, wq, ws)
        ob[:m, c0:c0 + n_out] = 7.0
        assert (ob == 7.0).all()


def test_linear_fp8_shows_nan(sevo):
    g = gen(3)
    for m in (4, 80):
        xq, xs = quantised(normal((m, 256), g))
        wq, ws = weights((128, 256), g)
        w = sevo.sevo_pack_weight_fp8(wq)
        xs[1, 2] = float("nan")
        for dtype in (torch.float32, BF):
            y = sevo.sevo_linear_fp8(xq, xs, w, ws, out_dtype=dtype)
            assert torch.isnan(y[2]).all()
            assert torch.isfinite(y[:2]).all() and torch.isfinite(y[3:]).all()


# ------------------------------------------------------------------ routing
def route_reference(logits, top_k, score, bias, groups, top_groups, best, renorm, scaling):
    """The definition, a token at a time, in float64 (numpy)."""
    n, E = logits.shape
    ex, wt = np.zeros((n, top_k), np.int64), np.zeros((n, top_k))
    each = E // groups
    with np.errstate(all="ignore"):
        for t in range(n):
            z = logits[t].astype(np.float64)
            if score == "sigmoid":
                p = 1 / (1 + np.exp(-z))
            else:
                p = np.exp(z - z.max())
                p = p / p.sum()
            c = p if bias is None else p + bias.astype(np.float64)
            c = np.where(np.isnan(c), -np.inf, c)
            gs = np.array([np.sort(c[j * each:(j + 1) * each])[::-1][:best].sum()
                           for j in range(groups)])
            gs = np.where(np.isnan(gs), -np.inf, gs)
            kept = sorted(range(groups), key=lambda j: (-gs[j], j))[:top_groups]
            cand = [e for e in range(E) if e // each in kept]
            pick = sorted(cand, key=lambda e: (-c[e], e))[:top_k]
            w = p[pick]
            if renorm:
                w = w / (w.sum() + 1e-20)
            ex[t], wt[t] = pick, w * scaling
    return ex, wt


@pytest.mark.parametrize("n,E,top_k,score,biased,groups,top_groups,best,renorm", [
    (1, 1, 1, "softmax", False, 1, 1, 1, True), (3, 7, 3, "sigmoid", False, 1, 1, 1, False),
    (64, 128, 8, "softmax", False, 1, 1, 1, True), (100, 256, 8, "sigmoid", True, 8, 4, 2, True),
    (65, 160, 6, "softmax", False, 8, 3, 1, False), (33, 64, 16, "sigmoid", True, 1, 1, 1, True),
    (5, 192, 4, "softmax", True, 64, 2, 2, True), (300, 256, 1, "sigmoid", True, 4, 1, 2, True),
    (17, 60, 5, "softmax", True, 5, 2, 2, True)])
def test_moe_route(sevo, n, E, top_k, score, biased, groups, top_groups, best, renorm):
    g = gen(n + E)
    ld = E + 3
    buf = normal((n, ld), g, 2.0)
    buf[:, E:] = float("nan")
    logits = buf[:, :E]
    bias = normal((E,), g, 0.3) if biased else None
    if n > 2:
        logits[1] = 0.5                             # every expert ties: the lowest indices
        logits[2] = torch.round(logits[2])          # many ties
    ex, wt = sevo.sevo_moe_route(logits, top_k, score, bias, groups, top_groups, best, renorm, 2.5)
    rex, rwt = route_reference(logits.cpu().numpy(), top_k, score,
                               None if bias is None else bias.cpu().numpy(), groups, top_groups,
                               best, renorm, 2.5)
    np.testing.assert_array_equal(ex.cpu().numpy(), rex)
    np.testing.assert_allclose(wt.cpu().numpy(), rwt, rtol=2.0 ** -23, atol=1e-44)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_moe_route_hard_values(sevo, score):
    """Saturated scores that tie in fp32 but not in float64, infinities, NaN,
    experts switched off by a bias of -inf."""
    E, k = 96, 4
    z = np.full((7, E), -3.0, np.float32)
    z[0, 10:20] = np.linspace(30, 31, 10)           # sigmoids of 1 - 1e-13
    z[1, :] = -200.0
    z[1, 5], z[1, 90] = -199.0, -198.5
    z[2, 3] = np.inf
    z[3, 3] = np.nan
    z[4] = np.nan
    z[5] = -np.inf
    z[6, :] = np.arange(E)[::-1] * 1e-6
    bias = np.zeros(E, np.float32)
    bias[19] = bias[18] = -np.inf
    for b in (None, bias):
        for groups, top_groups, best in ((1, 1, 1), (8, 2, 2)):
            ex, wt = sevo.sevo_moe_route(torch.from_numpy(z).cuda(), k, score,
                                         None if b is None else torch.from_numpy(b).cuda(), groups,
                                         top_groups, best, True, 1.0)
            rex, rwt = route_reference(z, k, score, b, groups, top_groups, best, True, 1.0)
            np.testing.assert_array_equal(ex.cpu().numpy(), rex)
            np.testing.assert_allclose(wt.cpu().numpy(), rwt, rtol=2.0 ** -23, atol=1e-44)


# ------------------------------------------------------------------ experts
def routing(n, E, top_k, g, how):
    z = normal((n, E), g, 1.5)
    if how == "skewed":
        z[:, 0] += 20.0                             # one expert takes every token
        z[:, E // 2:] -= 50.0                       # half of them none
    w, ex = torch.topk(z, top_k)
    return ex.to(torch.int32), torch.softmax(w, 1)


@pytest.mark.parametrize("n,E,top_k,n_out,k,how", [
    (1, 8, 2, 128, 128, "even"), (1, 64, 1, 64, 256, "even"), (37, 64, 4, 256, 128, "even"),
    (64, 128, 8, 1536, 2048, "even"), (64, 128, 8, 2048, 768, "even"), (300, 16, 3, 320, 384, "skewed"),
    (700, 4, 2, 192, 640, "even"), (1500, 64, 8, 256, 256, "skewed"), (5, 3, 3, 64, 128, "even"),
    (2500, 16, 4, 512, 384, "even"), (600, 1, 1, 576, 512, "even")])
def test_moe_linear_fp8(sevo, n, E, top_k, n_out, k, how):
    say(f"experts n={n} E={E} top {top_k} {n_out} x {k} {how}")
    g = gen(n + E + k)
    ex, wt = routing(n, E, top_k, g, how)
    if n > 20:
        ex[3, 0] = -1                               # entries without an expert
        ex[7, top_k - 1] = E
    wq, ws = weights((E, n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    lists = sevo.sevo_moe_lists(ex, E, buffer=poisoned(sevo.sevo_moe_lists_bytes(n, top_k, E)))
    flat = ex.reshape(-1)
    ok = (flat >= 0) & (flat < E)
    for down in (False, True):
        rows = n * top_k if down else n
        xq, xs = quantised(normal((rows, k), g))
        shape = (top_k, n, n_out) if down else (n * top_k, n_out)
        out = torch.full(shape, 7.0, dtype=BF, device="cuda")
        y = sevo.sevo_moe_linear_fp8(xq, xs, w, ws, lists, weights=wt if down else None, out=out)
        y = y.transpose(0, 1).reshape(n * top_k, n_out) if down else y
        assert (y[~ok] == 7.0).all()
        X = values(xq, xs)
        for e in range(E):
            i = torch.nonzero(flat == e).squeeze(1)
            if not i.numel():
                continue
            W = weight_values(wq[e], ws[e])
            Xe = X[i if down else i // top_k]
            ref, mag = Xe @ W.t().contiguous(), Xe.abs() @ W.abs().t().contiguous()
            if down:
                p = wt.reshape(-1)[i].double().unsqueeze(1)
                ref, mag = ref * p, mag * p
            err = (y[i].double() - ref).abs()
            tol = ref.abs() * 2.0 ** -8 + mag * 2.0 ** -15
            assert (err <= tol).all(), f"expert {e} down {down}"


def test_moe_lists_none(sevo):
    """No entry has an expert: nothing is written."""
    ex = torch.full((70, 2), -1, dtype=torch.int32, device="cuda")
    wq, ws = weights((4, 64, 128), gen(1))
    xq, xs = quantised(normal((70, 128), gen(2)))
    lists = sevo.sevo_moe_lists(ex, 4)
    out = torch.full((140, 64), 7.0, dtype=BF, device="cuda")
    sevo.sevo_moe_linear_fp8(xq, xs, sevo.sevo_pack_weight_fp8(wq), ws, lists, out=out)
    assert (out == 7.0).all()


# ------------------------------------------------------------------ together
def dense_ffn(sevo, x, parts, gain, w, out):
    """x += parts; FFN of the normed rows in 8 bits; out: bf16 partial of the next norm."""
    q, s = sevo.sevo_add_rmsnorm_fp8(x, parts, gain, 1e-6)
    gu = sevo.sevo_linear_fp8(q, s, *w["gate_up"])
    a, sa = sevo.sevo_quantize_fp8(gu, swiglu=True)
    sevo.sevo_linear_fp8(a, sa, *w["down"], out=out)
    return q, s, gu, a, sa


@pytest.mark.parametrize("m", [1, 16, 100, 600])
def test_dense_ffn(sevo, m):
    """Norm, gate/up, SwiGLU, down, each stage against float64 on what the stage
    before it gave, and a captured graph replayed between eager work."""
    g = gen(m)
    H, F = 512, 1152
    say(f"dense FFN m={m}")
    ref, w = {}, {}
    for name, shape in (("gate_up", (2 * F, H)), ("down", (H, F))):
        ref[name] = weights(shape, g)
        w[name] = (sevo.sevo_pack_weight_fp8(ref[name][0]), ref[name][1])
    x0 = normal((m, H), g, 2.0)
    parts = normal((1, m, H), g, 0.5, BF)
    gain = normal((H,), g, 0.1, BF) + 1
    x = x0.clone()
    out = torch.empty(1, m, H, dtype=BF, device="cuda")
    q, s, gu, a, sa = dense_ffn(sevo, x, parts, gain, w, out[0])
    xd = (x0 + parts[0].float()).double()
    check_codes(q, s, xd / (xd.pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * gain.double(),
                rel=64 * 2.0 ** -24)
    check_product(gu, q, s, *ref["gate_up"])
    u = gu.double()
    check_codes(a, sa, u[:, :F] / (1 + torch.exp(-u[:, :F])) * u[:, F:], rel=64 * 2.0 ** -24)
    check_product(out[0], a, sa, *ref["down"])
    # the same in a graph, on the bits of the eager run
    want = out.clone()
    stream = torch.cuda.Stream()
    xg = x0.clone()
    outg = torch.empty_like(out)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dense_ffn(sevo, xg, parts, gain, w, outg[0])
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xg.copy_(x0)
        dense_ffn(sevo, xg, parts, gain, w, outg[0])
    for _ in range(3):
        outg.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outg, want) and torch.equal(xg, x)
        dense_ffn(sevo, x0.clone(), parts, gain, w, torch.empty_like(out)[0])   # eager between


@pytest.mark.parametrize("n", [1, 40, 700])
def test_moe_ffn(sevo, n):
    """Norm, router, routing, lists, gate/up, SwiGLU, down, and the next norm that
    adds the slots."""
    from paper_2604_07725_amd import sevo as binding
    g = gen(n)
    H, F, E, top = 256, 128, 64, 4
    wg, wd = weights((E, 2 * F, H), g), weights((E, H, F), g)
    pg, pd = sevo.sevo_pack_weight_fp8(wg[0]), sevo.sevo_pack_weight_fp8(wd[0])
    router = binding.sevo_pack_weight(normal((E, H), g, 0.1, BF))
    bias = normal((E,), g, 0.02)
    gain = normal((H,), g, 0.1, BF) + 1
    x = normal((n, H), g, 2.0)

    def layer(x):
        nb = torch.empty(n, H, dtype=BF, device="cuda")
        q, s = sevo.sevo_add_rmsnorm_fp8(x, None, gain, 1e-6, out_bf16=nb)
        logits = binding.sevo_linear(nb, router)
        ex, wt = sevo.sevo_moe_route(logits, top, "sigmoid", bias, 8, 4, 2, True, 1.5)
        lists = sevo.sevo_moe_lists(ex, E)
        gu = sevo.sevo_moe_linear_fp8(q, s, pg, wg[1], lists)
        a, sa = sevo.sevo_quantize_fp8(gu, swiglu=True)
        part = sevo.sevo_moe_linear_fp8(a, sa, pd, wd[1], lists, weights=wt)
        x0 = x.clone()
        q2, s2 = sevo.sevo_add_rmsnorm_fp8(x, part, gain, 1e-6)
        return x0, q, s, ex, wt, part, q2, s2

    x0, q, s, ex, wt, part, q2, s2 = layer(x)
    X = values(q, s)
    ffn = torch.zeros(n, H, dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero(ex == e, as_tuple=True)
        if t.numel():
            u = X[t] @ weight_values(wg[0][e], wg[1][e]).t().contiguous()
            y = u[:, :F] / (1 + torch.exp(-u[:, :F])) * u[:, F:]
            ffn.index_add_(0, t, (y @ weight_values(wd[0][e], wd[1][e]).t().contiguous()) *
                           wt[t, j].double().unsqueeze(1))
    got = (x.double() - x0.double())
    # bf16 gate/up and partials (2^-8 each) and 8-bit SwiGLU rows (2^-4 an element,
    # independent: about 2^-4 / sqrt(3) of the norm)
    rel = float((got - ffn).norm() / ffn.norm())
    say(f"moe FFN n={n} rel {rel:.3e}")
    assert rel <= 2.0 ** -4
    want = x0
    for p in range(top):
        want = want + part[p].float()
    assert torch.equal(x, want)
    # twice on the same inputs: the same bits
    again = layer(x0.clone())
    for p, r in zip(again[1:], (q, s, ex, wt, part, q2, s2)):
        assert torch.equal(p.view(torch.uint8) if p.dtype == F8 else p,
                           r.view(torch.uint8) if r.dtype == F8 else r)


def test_two_streams(sevo):
    """Calls on two streams at once, each with its own outputs."""
    g = gen(9)
    m, n_out, k = 48, 1024, 2048
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    ins = [quantised(normal((m, k), g)) for _ in range(2)]
    want = [sevo.sevo_linear_fp8(q, s, w, ws) for q, s in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    need = max(sevo.sevo_linear_fp8_workspace_bytes(m, n_out, k), 256)
    wss = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty(m, n_out, dtype=BF, device="cuda") for _ in range(2)]
    for _ in range(20):
        for i in range(2):
            sevo.sevo_linear_fp8(*ins[i], w, ws, out=outs[i], workspace=wss[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i])


# ------------------------------------------------------------------ other calls
@pytest.mark.parametrize("m,n_out,k", [(2100, 8256, 384), (1500, 20544, 128), (700, 16448, 256),
                                       (40, 16960, 256), (4700, 4160, 1024)])
@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_linear_fp8_more_tiles_than_cus(sevo, m, n_out, k, dtype):
    """A workgroup takes several tiles: the next one's loads run under the stores of
    the last, whole tiles and cut ones in turn."""
    say(f"tiles {m} x {n_out} x {k} {dtype}")
    g = gen(m + k)
    xq, xs = quantised(normal((m, k), g))
    wq, ws = weights((n_out, k), g)
    out = torch.full((m + 1, n_out), 7.0, dtype=dtype, device="cuda")
    y = sevo.sevo_linear_fp8(xq, xs, sevo.sevo_pack_weight_fp8(wq), ws, out=out[:m])
    check_product(y, xq, xs, wq, ws)
    assert (out[m] == 7.0).all()


def test_linear_fp8_far_rows(sevo):
    """Output rows 2^23 bytes and more apart, the last ones past 2^31 bytes."""
    g = gen(5)
    m, n_out, k, ld = 300, 320, 256, (1 << 22) + 4
    xq, xs = quantised(normal((m, k), g))
    wq, ws = weights((n_out, k), g)
    out = torch.empty(m, ld, dtype=BF, device="cuda")[:, :n_out]
    sevo.sevo_linear_fp8(xq, xs, sevo.sevo_pack_weight_fp8(wq), ws, out=out)
    check_product(out.contiguous(), xq, xs, wq, ws)


def check_experts(y, xq, xs, wq, ws, flat, top_k, wt, down):
    """Rows [entries, n_out] of the experts' products against float64."""
    X = values(xq, xs)
    for e in range(wq.shape[0]):
        i = torch.nonzero(flat == e).squeeze(1)
        if not i.numel():
            continue
        W = weight_values(wq[e], ws[e])
        Xe = X[i if down else i // top_k]
        ref, mag = Xe @ W.t().contiguous(), Xe.abs() @ W.abs().t().contiguous()
        if down:
            p = wt.reshape(-1)[i].double().unsqueeze(1)
            ref, mag = ref * p, mag * p
        err = (y[i].double() - ref).abs()
        assert (err <= ref.abs() * 2.0 ** -8 + mag * 2.0 ** -15).all(), f"expert {e} down {down}"


@pytest.mark.parametrize("n,E,top_k,n_out,k", [
    (20, 16, 2, 192, 256), (100, 16, 3, 320, 384), (250, 12, 2, 448, 256), (400, 8, 3, 192, 128),
    (900, 6, 2, 576, 384), (9000, 16, 8, 192, 128), (3, 256, 16, 64, 128), (1, 2, 2, 128, 128)])
def test_moe_linear_fp8_inside_buffers(sevo, n, E, top_k, n_out, k):
    """Every tile height, n_out no multiple of 128, rows and scales inside larger
    buffers, a token that has the same expert twice; 72000 entries (lists in more
    than one launch)."""
    say(f"experts in buffers n={n} E={E} top {top_k} {n_out} x {k}")
    g = gen(n + E + k)
    ex, wt = routing(n, E, top_k, g, "even")
    if n > 10:
        ex[5] = ex[5, 0]
        ex[n - 1, 0] = 1 << 30
    wq, ws = weights((E, n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    lists = sevo.sevo_moe_lists(ex, E, buffer=poisoned(sevo.sevo_moe_lists_bytes(n, top_k, E)))
    flat = ex.reshape(-1)
    for down in (False, True):
        rows = n * top_k if down else n
        xq, xs = quantised(normal((rows, k), g))
        xb = torch.full((rows, k + 32), 0x7F, dtype=torch.uint8, device="cuda")
        xb[:, 16:16 + k] = xq.view(torch.uint8)
        sb = torch.full((k // 128, rows + 7), float("nan"), device="cuda")
        sb[:, 2:2 + rows] = xs
        out = torch.full((top_k, n, n_out) if down else (n * top_k, n_out), 7.0, dtype=BF, device="cuda")
        y = sevo.sevo_moe_linear_fp8(xb.view(F8)[:, 16:16 + k], sb[:, 2:2 + rows], w, ws, lists,
                                     weights=wt if down else None, out=out)
        y = y.transpose(0, 1).reshape(n * top_k, n_out) if down else y
        assert (y[flat >= E] == 7.0).all()
        check_experts(y, xq, xs, wq, ws, flat, top_k, wt, down)


@pytest.mark.parametrize("n,E,top_k,score,biased", [
    (4099, 256, 16, "sigmoid", True), (2050, 128, 8, "softmax", False), (1027, 250, 11, "softmax", True)])
def test_moe_route_near_ties(sevo, n, E, top_k, score, biased):
    """Logits a few fp32 steps apart, where fp32 scores cannot tell which is larger."""
    g = gen(E)
    steps = torch.randint(0, 40, (n, E), device="cuda", generator=g).float()
    logits = 0.7 + steps * 2.0 ** -23
    logits[: n // 2] += normal((n // 2, 1), g)
    bias = torch.randint(0, 3, (E,), device="cuda", generator=g).float() * 2.0 ** -22 if biased else None
    ex, wt = sevo.sevo_moe_route(logits, top_k, score, bias, renormalise=True)
    z = logits.double().cpu().numpy()
    p = 1 / (1 + np.exp(-z)) if score == "sigmoid" else np.exp(z - z.max(1, keepdims=True))
    if score == "softmax":
        p = p / p.sum(1, keepdims=True)
    c = p if bias is None else p + bias.double().cpu().numpy()
    got = ex.cpu().numpy()
    # exp in float64 is within a step of its value on either side: choices whose values
    # are that near may stand either way, and are equal up to it
    rank = np.sort(c, 1)[:, ::-1][:, :top_k]
    mine = np.take_along_axis(c, got, 1)
    assert np.abs(mine - rank).max() <= 8 * 2.0 ** -53
    assert all(len(set(r)) == top_k for r in got)
    w = np.take_along_axis(p, got, 1)
    np.testing.assert_allclose(wt.cpu().numpy(), w / w.sum(1, keepdims=True), rtol=2.0 ** -23)


def test_graphs(sevo):
    """Two layers' chains captured in two graphs, replayed in turn with eager calls
    between: every replay gives the eager bits."""
    H, F, E, top, n = 512, 256, 32, 4, 96
    g = gen(77)
    wg, wd, wo = weights((E, 2 * F, H), g), weights((E, H, F), g), weights((H, 4 * H), g)
    pg, pd, po = (sevo.sevo_pack_weight_fp8(w[0]) for w in (wg, wd, wo))
    gain = normal((H,), g, 0.1, BF) + 1

    def layer(s):
        a, sa = sevo.sevo_quantize_fp8(s["attn"])
        o = sevo.sevo_linear_fp8(a, sa, po, wo[1])
        x = s["x"].clone()
        q, qs = sevo.sevo_add_rmsnorm_fp8(x, o.unsqueeze(0), gain, 1e-6)
        ex, wt = sevo.sevo_moe_route(s["logits"], top, "sigmoid", None, 4, 2, 1)
        lists = sevo.sevo_moe_lists(ex, E)
        gu = sevo.sevo_moe_linear_fp8(q, qs, pg, wg[1], lists)
        d, ds = sevo.sevo_quantize_fp8(gu, swiglu=True)
        part = sevo.sevo_moe_linear_fp8(d, ds, pd, wd[1], lists, weights=wt)
        y, ys = sevo.sevo_add_rmsnorm_fp8(x, part, gain, 1e-6)
        f = sevo.sevo_linear_fp8(a, sa, po, wo[1], out_dtype=torch.float32)
        return x, y.view(torch.uint8), ys, ex, wt, f

    def fill(s, seed):
        h = gen(seed)
        s["x"].copy_(normal((n, H), h))
        s["attn"].copy_(normal((n, 4 * H), h, 1.0, BF))
        s["logits"].copy_(normal((n, E), h, 1.5))

    states, graphs, outs = [], [], []
    for i in range(2):
        s = {"x": torch.empty(n, H, device="cuda"), "attn": torch.empty(n, 4 * H, dtype=BF, device="cuda"),
             "logits": torch.empty(n, E, device="cuda")}
        fill(s, i)
        layer(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer(s)
        states.append(s), graphs.append(graph), outs.append(out)
    for turn in range(4):
        for i in range(2):
            fill(states[i], 100 * turn + i)
        want = [[t.clone() for t in layer(s)] for s in states]
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            for got, ref in zip(outs[i], want[i]):
                assert torch.equal(got, ref), f"turn {turn}, graph {i}"


def test_other_stream_order(sevo):
    """A chain on a stream of its own, its inputs made there too, the current stream
    busy with other work."""
    g = gen(8)
    n_out, k = 256, 1024
    wq, ws = weights((n_out, k), g)
    w = sevo.sevo_pack_weight_fp8(wq)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for m in (1, 30, 200):
        with torch.cuda.stream(side):
            x = normal((m, k), gen(m), 1.0, BF)
            q, s = sevo.sevo_quantize_fp8(x)
            y = sevo.sevo_linear_fp8(q, s, w, ws)
        busy = torch.randn(2048, 2048, device="cuda") @ torch.randn(2048, 2048, device="cuda")
        side.synchronize()
        check_product(y, q, s, wq, ws)
        assert torch.isfinite(busy).all()


@pytest.mark.parametrize("rows,cols,S,ptype", [(8300, 2048, 8, BF), (4100, 4096, 5, torch.float32),
                                               (9000, 4096, 3, BF)])
def test_add_rmsnorm_fp8_larger_than_the_cache(sevo, rows, cols, S, ptype):
    """More data than the last-level cache holds: the bits of calls on fewer rows."""
    say(f"norm {rows} x {cols}, {S} partials {ptype}")
    g = gen(S)
    x = normal((rows, cols), g, 2.0)
    parts = torch.randn(S, rows, cols, device="cuda", generator=g).to(ptype)
    gain = normal((cols,), g, 0.1, BF) + 1
    want = []
    for r0 in range(0, rows, 1024):
        xp = x[r0:r0 + 1024].clone()
        q, s = sevo.sevo_add_rmsnorm_fp8(xp, parts[:, r0:r0 + 1024].contiguous(), gain, 1e-6)
        want.append((xp, q.view(torch.uint8), s))
    q, s = sevo.sevo_add_rmsnorm_fp8(x, parts, gain, 1e-6)
    assert torch.equal(x, torch.cat([w[0] for w in want]))
    assert torch.equal(q.view(torch.uint8), torch.cat([w[1] for w in want]))
    assert torch.equal(s, torch.cat([w[2] for w in want], 1))


@pytest.mark.parametrize("m,n_out,k", [(33, 5120, 25600), (64, 10240, 5120), (81, 8192, 2048), (128, 6144, 4096),
                                       (192, 4096, 4096), (203, 2048, 768), (256, 512, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_linear_fp8_middle_rows(sevo, m, n_out, k, dtype):
    """Row counts between a few and many, with one to four M tiles of 64 rows, the last
    one cut."""
    say(f"middle {m} x {n_out} x {k} {dtype}")
    g = gen(m + n_out)
    xq, xs = quantised(normal((m, k), g))
    wq, ws = weights((n_out, k), g)
    out = torch.full((m + 2, n_out), 7.0, dtype=dtype, device="cuda")
    y = sevo.sevo_linear_fp8(xq, xs, sevo.sevo_pack_weight_fp8(wq), ws, out=out[:m])
    check_product(y, xq, xs, wq, ws)
    assert (out[m:] == 7.0).all()


def test_mixed_calls_on_four_streams(sevo):
    """Products of every kind, routings and quantisers at once, in changing company:
    always the bits of the same call alone."""
    g = gen(21)
    jobs = []
    for m, n_out, k, dtype in ((700, 4096, 1024, BF), (64, 4096, 4096, BF), (2100, 2048, 768, BF),
                               (203, 5120, 2048, torch.float32), (16, 6144, 4096, torch.float32)):
        q, s = quantised(normal((m, k), g))
        wq, ws = weights((n_out, k), g)
        w = sevo.sevo_pack_weight_fp8(wq)
        jobs.append(lambda q=q, s=s, w=w, ws=ws, d=dtype: sevo.sevo_linear_fp8(q, s, w, ws, out_dtype=d))
    for n, E, top, n_out, k in ((900, 16, 4, 512, 384), (64, 64, 8, 768, 512), (300, 16, 4, 512, 512)):
        ex, _ = routing(n, E, top, g, "even")
        wq, ws = weights((E, n_out, k), g)
        w = sevo.sevo_pack_weight_fp8(wq)
        q, s = quantised(normal((n, k), g))
        jobs.append(lambda ex=ex, E=E, q=q, s=s, w=w, ws=ws:
                    sevo.sevo_moe_linear_fp8(q, s, w, ws, sevo.sevo_moe_lists(ex, E)))
    logits, rows = normal((3000, 256), g, 1.5), normal((2000, 4096), g, 1.0, BF)
    jobs.append(lambda: sevo.sevo_moe_route(logits, 8, "sigmoid", None, 8, 4, 2)[1])
    jobs.append(lambda: sevo.sevo_quantize_fp8(rows)[0].view(torch.uint8))
    want = [f() for f in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    rng = np.random.default_rng(4)
    for turn in range(12):
        got = []
        for stream in streams:
            with torch.cuda.stream(stream):
                for j in rng.integers(0, len(jobs), 5):
                    got.append((j, jobs[j]()))
        torch.cuda.synchronize()
        for j, t in got:
            assert torch.equal(t, want[j]), f"turn {turn}, call {j}"
