"""The 8-bit cache on the GPU: append, pages to 8 bits and back, attention, and the run of them
together, against float64."""
import math
import types

import numpy as np
import pytest
import torch

from tests import kv8_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def sevo(have_gpu):
    from paper_2604_07725_amd import sevo
    sevo.lib()
    return sevo


def gen(seed):
    return torch.Generator().manual_seed(seed)


def model(sevo, hq, hkv, d, qk_norm=True, max_position=512, seed=0, theta=1e4):
    from paper_2604_07725_amd import synth
    g = gen(seed)
    shape = synth.ModelShape(1, 128, hq, hkv, d, 128, 64, rope_theta=theta, rms_eps=1e-6, qk_norm=qk_norm)
    w = torch.zeros((hq + 2 * hkv) * d * 128, dtype=BF, device=DEV)
    gq, gk = ((1 + 0.2 * torch.randn(d, generator=g)).to(BF).to(DEV) for _ in range(2))
    layer = {k: w for k in ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate_up", "w_down")}
    return sevo.sevo_init_model(shape, {"embed": w, "lm_head": w, "final_norm": w,
                                        "layers": [{**layer, "q_norm": gq, "k_norm": gk}]}, max_position)


def rope_rows(m, qkv, positions):
    """float64 q [n, hq, d], k, v [n, hkv, d] after norm and RoPE."""
    c = m.config
    hq, hkv, d = c.n_q_heads, c.n_kv_heads, c.head_dim
    x = qkv.double().cpu().view(-1, hq + 2 * hkv, d)
    layer = m.tensors["layers"][0]
    out = []
    for part, gain in ((x[:, :hq], layer["q_norm"]), (x[:, hq:hq + hkv], layer["k_norm"])):
        if c.qk_norm:
            part = part / (part.pow(2).mean(2, keepdim=True) + 1e-6).sqrt() * gain.double().cpu()
        w = float(np.float32(c.rope_theta)) ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
        a = positions.double().cpu()[:, None, None] * w
        lo, hi = part[..., :d // 2], part[..., d // 2:]
        out.append(torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], 2))
    return out[0], out[1], x[:, hq + hkv:]


# A value after norm and RoPE: the norm's sum of d squares (d 2^-24), its root, division, two factors
# and the rotation's two products (about 10 roundings), cos and sin to 2^-24 of 1: relative to the pair's
# larger value.
def value_tol(d):
    return (d / 2 + 16) * 2.0 ** -24


def check_block(codes, scale, y, tol):
    """codes, scales of blocks y [.., d] float64 that the kernel knows to tol of the block's largest."""
    s = (y.abs().amax(-1) / 448).clamp_min(2.0 ** -64)
    assert (scale - s).abs().max() <= ((tol + 4 * 2.0 ** -24) * s).max()
    assert ((scale - s).abs() <= (tol + 4 * 2.0 ** -24) * s).all()
    # a code is off by half a step: 2^-4 of itself, 2^-10 below the smallest normal (2^-6), and by what
    # the value itself is off by (tol and 4 roundings of at most 448)
    x = y / s[..., None]
    assert ((codes - x).abs() <= x.abs() * 2.0 ** -4 + 2.0 ** -10 + 448 * (2 * tol + 8 * 2.0 ** -24)).all()
    # and nowhere nearer to another code than that uncertainty
    near = x.clamp(-448, 448).to(torch.float32).to(F8).double()
    step = torch.maximum(2.0 ** (torch.floor(torch.log2(x.abs().clamp_min(1e-30))) - 3), torch.tensor(2.0 ** -9, dtype=torch.float64))
    tie = ((codes - x).abs() - step / 2).abs() <= 448 * (2 * tol + 8 * 2.0 ** -24)
    assert ((codes == near) | tie).all()


@pytest.mark.parametrize("hq,hkv,d,qk_norm,n", [
    (4, 2, 64, True, 4), (8, 2, 64, False, 33), (32, 8, 128, True, 5), (64, 8, 128, True, 17),
    (8, 1, 128, False, 1), (2, 2, 128, True, 600), (8, 8, 64, True, 530), (32, 4, 128, True, 513)])
def test_append(sevo, hq, hkv, d, qk_norm, n):
    g = gen(n)
    m = model(sevo, hq, hkv, d, qk_norm, max_position=700)
    cand, max_pages = 3, 44
    pages = cand * max_pages + 2
    table = torch.randperm(pages, generator=g)[:cand * max_pages].view(cand, max_pages).to(torch.int32)
    at = torch.randperm(cand * 600, generator=g)[:n]
    rows, positions = (at // 600).to(torch.int32), (at % 600).to(torch.int32)
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g) * 2
    pool = torch.full((pages, hkv, 32 * d + 128), 0xA5, dtype=torch.uint8)
    dev = pool.to(DEV)
    q = sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv.to(DEV), positions.to(DEV), table.to(DEV), dev, rows=rows.to(DEV))
    rq, rk, rv = rope_rows(m, qkv, positions)
    tol = value_tol(d)
    pair = torch.maximum(rq[..., :d // 2].abs(), rq[..., d // 2:].abs()).repeat(1, 1, 2)
    assert ((q.double().cpu() - rq).abs() <= rq.abs() * 2.0 ** -8 + 4 * tol * pair).all()
    k, v, ks, vs = ref.read_pool(dev, d)
    page, slot = table[rows.long(), positions.long() // 16].long(), positions.long() % 16
    check_block(k[page, :, slot], ks[page, :, slot], rk, 2 * tol)
    check_block(v[page, :, slot], vs[page, :, slot], rv, 0.0)
    # every other slot as it was
    k0, v0, ks0, vs0 = ref.read_pool(pool, d)
    for now, was in ((k, k0), (v, v0), (ks, ks0), (vs, vs0)):
        same = (now == was).flatten(3).all(3) if now.dim() == 4 else now == was
        left = torch.ones(pages, hkv, 16, dtype=torch.bool)
        left[page, :, slot] = False
        assert same[left].all()
    m.close()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (32, 8, 128), (64, 8, 128)])
def test_append_many_tokens_as_few(sevo, hq, hkv, d):
    """A prefill's call and a step's give the same bits."""
    g = gen(5)
    n = 1037
    m = model(sevo, hq, hkv, d, max_position=n)
    table = torch.randperm(-(-n // 16), generator=g).view(1, -1).to(torch.int32).to(DEV)
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g).to(DEV)
    pos, rows = torch.arange(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    a, b = (torch.zeros(table.shape[1], hkv, 32 * d + 128, dtype=torch.uint8, device=DEV) for _ in range(2))
    qa = sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv, pos, table, a, rows=rows)
    qb = torch.cat([sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv[i:i + 256].contiguous(), pos[i:i + 256].contiguous(),
                                                      table, b, rows=rows[i:i + 256].contiguous())
                    for i in range(0, n, 256)])
    assert torch.equal(qa, qb) and torch.equal(a, b)
    m.close()


def test_append_leaves_out_what_has_no_place(sevo):
    g = gen(1)
    hq, hkv, d = 4, 2, 64
    m = model(sevo, hq, hkv, d, max_position=60)
    table = torch.tensor([[0, 7, 2, 3], [4, -1, 1, 5]], dtype=torch.int32)      # six pages: 7 and -1 are none
    positions = torch.tensor([-1, 60, 20, 25, 33, 3, 5, 5], dtype=torch.int32)
    rows = torch.tensor([0, 0, 0, 1, 0, 2, -1, 1], dtype=torch.int32)
    qkv = torch.randn(8, (hq + 2 * hkv) * d, generator=g)
    pool = torch.full((6, hkv, 32 * d + 128), 0x11, dtype=torch.uint8, device=DEV)
    q = sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv.to(DEV), positions.to(DEV), table.to(DEV), pool, rows=rows.to(DEV)).cpu()
    assert (q[:2] == 0).all()
    rq = rope_rows(m, qkv, positions)[0]
    assert (q[2:].double() - rq[2:]).abs().max() < 2.0 ** -6
    _, _, ks, vs = ref.read_pool(pool, d)
    was = torch.full((4,), 0x11, dtype=torch.uint8).view(torch.float32).double()
    changed = ((ks != was) | (vs != was)).any(1).nonzero().tolist()
    assert changed == [[2, 1], [4, 5]]           # (row 0, 33) and (row 1, 5)
    # without rows: token i is row i's
    pool.fill_(0x11)
    sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv[:2].contiguous().to(DEV), positions[6:].to(DEV), table.to(DEV), pool)
    _, _, ks, _ = ref.read_pool(pool, d)
    assert (ks != was).any(1).nonzero().tolist() == [[0, 5], [4, 5]]
    m.close()


@pytest.mark.parametrize("rows", [False, True])
def test_append_of_no_tokens(sevo, rows):
    m = model(sevo, 4, 2, 64, max_position=60)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    table = torch.zeros(2 if rows else 0, 3, dtype=torch.int32, device=DEV)
    pool = torch.full((3, 2, 32 * 64 + 128), 0x11, dtype=torch.uint8, device=DEV)
    q = sevo.sevo_qk_norm_rope_append_fp8(m, 0, torch.empty(0, 8 * 64, device=DEV), ids, table, pool,
                                          rows=ids if rows else None)
    assert q.shape == (0, 4, 64) and (pool == 0x11).all()
    m.close()


def test_append_nan_infinity_and_zeros(sevo):
    hq, hkv, d = 4, 2, 128
    m = model(sevo, hq, hkv, d, qk_norm=False)
    qkv = torch.zeros(1, (hq + 2 * hkv) * d)
    x = qkv.view(hq + 2 * hkv, d)
    x[hq, 5], x[hq + 3, 70] = math.nan, math.inf      # K of head 0, V of head 1
    x[hq + 1] = 2.0
    pool = torch.full((1, hkv, 32 * d + 128), 0xA5, dtype=torch.uint8, device=DEV)
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv.to(DEV), zero, zero[None], pool)
    k, v, ks, vs = ref.read_pool(pool, d)
    assert math.isnan(ks[0, 0, 0]) and math.isnan(vs[0, 1, 0])
    assert (k[0, 0, 0] == 0).all() and (v[0, 1, 0] == 0).all() and (v[0, 0, 0] == 0).all()
    # (the scale 2 / 448 is no fp32 number: 2 times the rounded 1 / 448, two roundings of 2^-24 at most)
    assert vs[0, 0, 0] == 2.0 ** -64 and ((k[0, 1, 0] * ks[0, 1, 0] - 2.0).abs() <= 2 * 2.0 ** -23).all()
    m.close()


# ------------------------------------------------------------------ pages
def bf_tiles(k, v):
    """[pages, hkv, 16, d] values -> the bf16 pool [pages, hkv, 2, 16 d]."""
    p, h, _, d = k.shape
    kt = k.view(p, h, 16, d // 32, 32).transpose(2, 3).reshape(p, h, -1)
    return torch.stack([kt, v.transpose(2, 3).reshape(p, h, -1)], 2).to(BF)


@pytest.mark.parametrize("hkv,d,count", [(1, 64, 1), (2, 64, 5), (3, 64, 7), (1, 128, 1), (4, 128, 33), (8, 128, 6)])
def test_pack_pages(sevo, hkv, d, count):
    g = gen(count)
    pages = count + 3
    k, v = (torch.randn(pages, hkv, 16, d, generator=g).to(BF) for _ in range(2))
    k[0, 0, 3] = 0
    v[1, 0, 2] *= 1e30
    pool = bf_tiles(k, v).to(DEV)
    src = torch.randperm(pages, generator=g)[:count].to(torch.int32)
    out = sevo.sevo_pack_kv_fp8(pool, src_pages=src.to(DEV))
    kc, vc, ks, vs = ref.read_pool(out, d)
    check_block(kc, ks, k[src.long()].double(), 0.0)
    check_block(vc, vs, v[src.long()].double(), 0.0)
    # into a pool, at places of their own; all pages in order
    dst = torch.randperm(pages, generator=g)[:count].to(torch.int32)
    into = torch.full((pages, hkv, 32 * d + 128), 0x5A, dtype=torch.uint8, device=DEV)
    assert sevo.sevo_pack_kv_fp8(pool, into, src.to(DEV), dst.to(DEV)) is into
    assert torch.equal(into[dst.long().to(DEV)], out)
    rest = torch.ones(pages, dtype=torch.bool)
    rest[dst.long()] = False
    assert (into[rest.to(DEV)] == 0x5A).all()
    assert torch.equal(sevo.sevo_pack_kv_fp8(pool)[src.long().to(DEV)], out)


@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 64), (1, 128), (4, 128)])
def test_unpack_pages(sevo, hkv, d):
    g = gen(d)
    pages = 9
    codes = torch.arange(pages * hkv * 16 * d, dtype=torch.int64) * 37 % 256
    codes[codes % 128 == 127] = 0                      # the NaN codes
    codes = codes.to(torch.uint8).view(F8).view(pages, hkv, 16, d)
    ks, vs = (torch.rand(pages, hkv, 16, generator=g) + 0.5 for _ in range(2))
    ks[1, 0, 2] = math.nan
    pool = ref.write_pool(codes, codes, ks, vs).to(DEV)
    src = torch.randperm(pages, generator=g)[:5].to(torch.int32)
    out = sevo.sevo_unpack_kv_fp8(pool, src_pages=src.to(DEV)).cpu()
    full = sevo.sevo_unpack_kv_fp8(pool).cpu()
    want = bf_tiles(codes.float() * ks[..., None], codes.float() * vs[..., None])
    assert torch.equal(full.view(torch.int16)[~full.isnan()], want.view(torch.int16)[~want.isnan()])
    assert torch.equal(full.isnan(), want.isnan()) and full.isnan().any()
    assert torch.equal(out.view(torch.int16), full[src.long()].view(torch.int16))


@pytest.mark.parametrize("d", [64, 128])
def test_pages_outside_the_pools(sevo, d):
    g = gen(3)
    pool = torch.randn(4, 2, 2, 16 * d, generator=g).to(BF).to(DEV)
    src = torch.tensor([1, 4, -1, 2, 0], dtype=torch.int32, device=DEV)
    dst = torch.tensor([0, 1, 2, 6, -5], dtype=torch.int32, device=DEV)
    into = torch.full((6, 2, 32 * d + 128), 0x5A, dtype=torch.uint8, device=DEV)
    sevo.sevo_pack_kv_fp8(pool, into, src, dst)
    assert torch.equal(into[0], sevo.sevo_pack_kv_fp8(pool)[1])
    assert (into[1:3] == 0).all() and (into[3:] == 0x5A).all()
    back = torch.full((6, 2, 2, 16 * d), 7.0, dtype=BF, device=DEV)
    sevo.sevo_unpack_kv_fp8(into[:4].contiguous(), back, src, dst)
    assert (back[0] == 0).all() and (back[1:3] == 0).all() and (back[3:] == 7).all()


def test_pack_nan_and_infinity(sevo):
    k = torch.ones(1, 1, 16, 128)
    v = torch.ones(1, 1, 16, 128)
    k[0, 0, 4, 100], v[0, 0, 9, 3] = math.inf, math.nan
    kc, vc, ks, vs = ref.read_pool(sevo.sevo_pack_kv_fp8(bf_tiles(k, v).to(DEV)), 128)
    assert ks[0, 0].isnan().nonzero().tolist() == [[4]] and vs[0, 0].isnan().nonzero().tolist() == [[9]]
    assert (kc[0, 0, 4] == 0).all() and (vc[0, 0, 9] == 0).all()
    assert (kc[0, 0, 5] == 448).all() and (vc[0, 0, 8] == 448).all()


# ------------------------------------------------------------------ attention
def cache(lens, hkv, d, seed, extra=1, max_pages=None):
    g = gen(seed)
    need = [(x + 15) // 16 for x in lens]
    pages = sum(need) + extra
    pool = ref.random_pool(pages, hkv, d, g)
    ids = torch.randperm(pages, generator=g)[:sum(need)].to(torch.int32)
    width = max_pages or max(max(need), 1)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for i, x in enumerate(need):
        table[i, :x] = ids[at:at + x]
        at += x
    return pool, table, g


def check_attention(sevo, pool, table, lens, q, m=None, **kw):
    n, T, hq, d = q.shape
    length = torch.tensor(lens, dtype=torch.int32)
    mm = torch.tensor(m, dtype=torch.int32) if m is not None else torch.full((n,), T, dtype=torch.int32)
    scale = kw.pop("scale", d ** -0.5)
    o = sevo.sevo_attn_decode_fp8(q.to(DEV), pool.to(DEV), table.to(DEV), length.to(DEV),
                                  q_lens=mm.to(DEV) if m is not None else None, scale=scale, **kw)
    want, mass, big = ref.attention(q, pool, table, length, mm.clamp(0, T), scale)
    bound = ref.attention_bound(want, mass, big, d, max(lens))
    err = (o.double().cpu() - want).abs()
    assert (err <= bound).all(), f"worst {float((err / bound).max()):.2f} of the bound"
    return o


@pytest.mark.parametrize("hq,hkv,d,T", [
    (4, 2, 64, 1), (3, 3, 64, 1), (8, 1, 64, 3), (10, 2, 64, 5), (8, 2, 128, 1), (8, 1, 128, 1), (6, 2, 128, 1),
    (16, 1, 128, 1), (16, 2, 128, 4), (4, 1, 128, 8), (8, 1, 128, 8), (16, 1, 128, 5), (8, 1, 128, 16), (2, 2, 128, 16)])
def test_attention(sevo, hq, hkv, d, T):
    lens = [T, 16, T + 15, 33, 47, 300, 700]
    pool, table, g = cache(lens, hkv, d, seed=hq + T)
    q = torch.randn(len(lens), T, hq, d, generator=g).to(BF)
    check_attention(sevo, pool, table, lens, q)
    # a page table that may hold long contexts: candidates in several splits
    wide = torch.full((len(lens), 300), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    check_attention(sevo, pool, wide, lens, q)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_empty_and_short(sevo, d):
    """Lengths 0 and 1, new tokens fewer than the rows, none, or more than the keys."""
    lens = [0, 1, 1, 2, 16, 17, 40, 5]
    m = [0, 1, 3, 2, 0, 3, 1, 9]
    pool, table, g = cache(lens, 2, d, seed=4)
    q = torch.randn(8, 3, 4, d, generator=g).to(BF)
    o = check_attention(sevo, pool, table, lens, q, m)
    for i, x in enumerate(m):
        assert (o[i, min(x, 3):] == 0).all()
    assert (o[0] == 0).all() and (o[2, :2] == 0).all()       # the first two of three new tokens over one key
    # with an output of its own the spare rows stay
    out = torch.full_like(o, 3.0)
    check = sevo.sevo_attn_decode_fp8(q.to(DEV), pool.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                                      q_lens=torch.tensor(m, dtype=torch.int32, device=DEV), out=out)
    assert check is out
    for i, x in enumerate(m):
        x = min(x, 3)
        assert torch.equal(out[i, :x], o[i, :x]) and (out[i, x:] == 3).all()


@pytest.mark.parametrize("T,hkv,G", [(1, 2, 4), (5, 1, 8)])
def test_attention_split_and_joined(sevo, T, hkv, G):
    """One long candidate among short ones: many splits, some of them of a page; the spare rows of a
    joined candidate; the same bits on every call."""
    lens = [3000, 7, 1025, 512, 2049]
    m = [T, T, max(1, T - 2), T, 1]
    pool, table, g = cache(lens, hkv, 128, seed=7, max_pages=400)
    q = torch.randn(5, T, hkv * G, 128, generator=g).to(BF)
    a = check_attention(sevo, pool, table, lens, q, m)
    b = check_attention(sevo, pool, table, lens, q, m)
    assert torch.equal(a, b)
    for i, x in enumerate(m):
        assert (a[i, x:] == 0).all()


def test_attention_many_candidates(sevo):
    """More candidates than a workgroup's threads, most of them short."""
    g = gen(9)
    lens = [int(x) for x in torch.randint(0, 40, (300,), generator=g)]
    lens[257] = 900
    pool, table, g = cache(lens, 1, 64, seed=9)
    q = torch.randn(300, 1, 2, 64, generator=g).to(BF)
    o = check_attention(sevo, pool, table, lens, q)
    # a wider page table: splits, and their join
    wide = torch.full((300, 200), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    far = check_attention(sevo, pool, wide, lens, q)
    assert (far.float() - o.float()).abs().max() <= 2.0 ** -6 * o.abs().max()


@pytest.mark.parametrize("hq,hkv,d,T", [(8, 8, 128, 1), (16, 8, 128, 9), (32, 8, 128, 9), (64, 8, 64, 7)])
def test_attention_many_short_candidates(sevo, hq, hkv, d, T):
    """More workgroups than the chip has units, one per candidate and head."""
    g = gen(hq + T)
    lens = [int(x) for x in torch.randint(1, 130, (40,), generator=g)]
    pool, table, g = cache(lens, hkv, d, seed=T)
    q = torch.randn(40, T, hq, d, generator=g).to(BF)
    check_attention(sevo, pool, table, lens, q, [min(T, x) for x in lens])


@pytest.mark.parametrize("width", [40, 300])
def test_attention_in_graphs_with_other_lengths(sevo, width):
    """Captured with some lengths, replayed with others, pages and queries too; two graphs on one
    workspace, one after the other."""
    hkv, d, T = 2, 128, 3
    pool, table, g = cache([640] * 4, hkv, d, seed=11, max_pages=width)
    pool = pool.to(DEV)
    need = max(16, sevo.sevo_attn_fp8_workspace_bytes(4, T, 8, hkv, d, width))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    sets = []
    for lens in ([640, 3, 0, 97], [16, 620, 320, 1], [0, 0, 0, 640]):
        sets.append([torch.randn(4, T, 8, d, generator=g).to(BF).to(DEV), table[torch.randperm(4, generator=g)].to(DEV),
                     torch.tensor(lens, dtype=torch.int32, device=DEV),
                     torch.tensor([min(T, x) for x in lens], dtype=torch.int32, device=DEV)])
    call = lambda x, **k: sevo.sevo_attn_decode_fp8(x[0], pool, x[1], x[2], q_lens=x[3], **k)
    want = [call(x).clone() for x in sets]
    held = [[t.clone() for t in x] for x in sets[:2]]
    outs = [torch.zeros_like(want[0]) for _ in held]
    torch.cuda.synchronize()
    graphs = []
    for x, o in zip(held, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(x, out=o, workspace=ws)
        graphs.append(graph)
    for rep in range(3):
        for k in range(2):
            x = sets[(rep + k) % 3]
            for t, v in zip(held[k], x):
                t.copy_(v)
            outs[k].zero_()                            # (rows past the new tokens stay as they were)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(outs[k], want[(rep + k) % 3])
        assert torch.equal(call(sets[rep]), want[rep])


def test_attention_on_two_streams_at_once(sevo):
    pool, table, g = cache([3000, 40, 1500], 2, 128, seed=12, max_pages=400)
    pool, table = pool.to(DEV), table.to(DEV)
    lens = torch.tensor([3000, 40, 1500], dtype=torch.int32, device=DEV)
    qs = [torch.randn(3, 8, 128, generator=g).to(BF).to(DEV) for _ in range(2)]
    want = [sevo.sevo_attn_decode_fp8(q, pool, table, lens).clone() for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[sevo.sevo_attn_decode_fp8(q, pool, table, lens, stream=s) for _ in range(20)] for q, s in zip(qs, streams)]
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        assert all(torch.equal(x, w) for x in o)


@pytest.mark.parametrize("d,T", [(64, 1), (128, 1), (128, 4)])
def test_attention_garbage_and_bad_pages(sevo, d, T):
    """What lies behind the last key, or in pages outside the pool, does not enter."""
    lens = [T + 5, 37, 64, 600]
    pool, table, g = cache(lens, 2, d, seed=d, max_pages=100 if T > 1 else None)
    q = torch.randn(4, T, 8, d, generator=g).to(BF)
    table[3, 4], table[3, 20], table[2, 1] = 10 ** 6, -7, pool.shape[0]
    clean = check_attention(sevo, pool, table, lens, q)
    k, v, ks, vs = (x.clone() for x in ref.read_pool(pool, d))
    k, v, ks, vs = k.float(), v.float(), ks.float(), vs.float()
    for i, n in enumerate(lens):
        page = int(table[i, (n - 1) // 16])
        s = n % 16
        if s and 0 <= page < pool.shape[0]:
            for x in (k, v, ks, vs):
                x[page, :, s:] = math.nan
    dirty = ref.write_pool(k.to(F8), v.to(F8), ks, vs)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o = sevo.sevo_attn_decode_fp8(q.to(DEV), dirty.to(DEV), table.to(DEV), lens_d)
    assert torch.equal(o, clean)


def test_attention_nan_tokens_stay_theirs(sevo):
    """A new token whose key and value are NaN: earlier rows do not see it, later ones do."""
    hq, hkv, d, T = 4, 1, 128, 4
    m = model(sevo, hq, hkv, d, qk_norm=False, max_position=64)
    g = gen(2)
    qkv = torch.randn(40 + T, (hq + 2 * hkv) * d, generator=g)
    qkv[42].view(-1, d)[hq:] = math.nan                     # keys 40 .. 43 are the new ones
    table = torch.arange(3, dtype=torch.int32, device=DEV)[None]
    pool = torch.full((3, hkv, 32 * d + 128), 255, dtype=torch.uint8, device=DEV)
    pos = torch.arange(40 + T, dtype=torch.int32, device=DEV)
    q = sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv.to(DEV), pos, table, pool, rows=torch.zeros_like(pos))
    lens = torch.tensor([44], dtype=torch.int32, device=DEV)
    o = sevo.sevo_attn_decode_fp8(q[None, 40:].contiguous(), pool, table, lens)
    assert not o[0, :2].isnan().any() and o[0, 2:].isnan().all()
    sub = sevo.sevo_attn_decode_fp8(q[None, 40:42].contiguous(), pool, table, lens - 2)
    assert torch.equal(sub[0], o[0, :2])
    m.close()


def test_attention_extreme_scores(sevo):
    """Scores of hundreds in either sign, and a single key that takes everything."""
    lens, d = [50, 333], 128
    pool, table, g = cache(lens, 2, d, seed=11)
    q = torch.randn(2, 1, 8, d, generator=g).to(BF) * 30
    check_attention(sevo, pool, table, lens, q, scale=1.0)
    check_attention(sevo, pool, table, lens, -q, scale=1e-6)


def test_attention_large_pool(sevo):
    """Pages beyond 4 GiB of the pool: the same bits as near its start."""
    hkv, d = 8, 128
    lens = [100, 2000]
    pool, table, g = cache(lens, hkv, d, seed=13, extra=0)
    q = torch.randn(2, 2, 32, d, generator=g).to(BF).to(DEV)
    tile = hkv * (32 * d + 128)
    far = (9 << 30) // tile
    big = torch.empty(far + pool.shape[0], hkv, 32 * d + 128, dtype=torch.uint8, device=DEV)
    big[far:] = pool.to(DEV)
    lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    near = sevo.sevo_attn_decode_fp8(q, pool.to(DEV), table.to(DEV), lens)
    moved = torch.where(table >= 0, table + far, table)
    assert torch.equal(sevo.sevo_attn_decode_fp8(q, big, moved.to(DEV), lens), near)
    # and through the other operators
    ids = torch.arange(far, far + pool.shape[0], dtype=torch.int32, device=DEV)
    values = sevo.sevo_unpack_kv_fp8(big, src_pages=ids)
    assert torch.equal(values, sevo.sevo_unpack_kv_fp8(pool.to(DEV)))
    big[far:] = 0
    sevo.sevo_pack_kv_fp8(values, big, dst_pages=ids)
    assert torch.equal(big[far:], sevo.sevo_pack_kv_fp8(values))


# ------------------------------------------------------------------ the run of them
class Run:
    """Candidates on an 8-bit cache whose prompts a bf16 prefill left, decoding with drafts."""

    def __init__(self, sevo, hq, hkv, d, n, T, vocab, seed):
        self.sevo, self.T = sevo, T
        g = gen(seed)
        self.m = model(sevo, hq, hkv, d, max_position=400)
        self.lens = torch.randint(20, 90, (n,), generator=g, dtype=torch.int32)
        width = (int(self.lens.max()) + 3 * (T + 1) + 15) // 16
        pages = n * width
        self.table = torch.randperm(pages, generator=g).view(n, width).to(torch.int32).to(DEV)
        k, v = (torch.randn(pages, hkv, 16, d, generator=g).to(BF) for _ in range(2))
        self.bf_pool = bf_tiles(k, v).to(DEV)
        self.pool = sevo.sevo_pack_kv_fp8(self.bf_pool)
        self.qkv = torch.randn(n * (T + 1), (hq + 2 * hkv) * d, generator=g).to(DEV)
        w = (torch.randn(vocab, hq * d, generator=g) * 0.25).to(BF).to(DEV)
        self.w = sevo.sevo_pack_weight(w)
        self.w_plain = w.double().cpu()
        self.drafts = torch.randint(0, vocab, (n, T), generator=g, dtype=torch.int32).to(DEV)
        self.draft_logits = (torch.randn(n, T, vocab, generator=g) * 2).to(DEV)
        self.u = torch.rand(n, T + 1, generator=g).to(DEV)
        self.rows = torch.arange(n, dtype=torch.int32).repeat_interleave(T + 1).to(DEV)
        self.lens = self.lens.to(DEV)
        self.positions = (self.lens[:, None] + torch.arange(T + 1, dtype=torch.int32, device=DEV)).reshape(-1).contiguous()
        self.total = self.lens + T + 1

    def step(self, pool):
        n, T = self.drafts.shape
        q = self.sevo.sevo_qk_norm_rope_append_fp8(self.m, 0, self.qkv, self.positions, self.table, pool, rows=self.rows)
        o = self.sevo.sevo_attn_decode_fp8(q.view(n, T + 1, *q.shape[1:]), pool, self.table, self.total)
        logits = self.sevo.sevo_linear(o.view(n * (T + 1), -1), self.w)
        return (q, o, logits) + self.sevo.sevo_verify_drafts(logits.view(n, T + 1, -1), self.drafts, self.u, 0.8,
                                                             draft_logits=self.draft_logits)


@pytest.mark.parametrize("hq,hkv,d,n,T", [(4, 2, 64, 5, 3), (32, 4, 128, 3, 4), (8, 2, 128, 2, 0)])
def test_a_step_with_drafts(sevo, hq, hkv, d, n, T):
    r = Run(sevo, hq, hkv, d, n, T, 448, seed=T)
    before = r.pool.clone()
    q, o, logits, tokens, lps, taken = r.step(r.pool)
    # the cache holds the prompt as it was, and the new tokens' blocks
    rq, rk, rv = rope_rows(r.m, r.qkv, r.positions)
    tol = value_tol(d)
    k, v, ks, vs = ref.read_pool(r.pool, d)
    pos = r.positions.cpu().long()
    page, slot = r.table.cpu()[r.rows.cpu().long(), pos // 16].long(), pos % 16
    check_block(k[page, :, slot], ks[page, :, slot], rk, 2 * tol)
    check_block(v[page, :, slot], vs[page, :, slot], rv, 0.0)
    lens = [int(x) for x in r.total]
    want, mass, big = ref.attention(q.view(n, T + 1, hq, d).cpu(), r.pool.cpu(), r.table.cpu(), lens, [T + 1] * n, d ** -0.5)
    assert ((o.double().cpu() - want).abs() <= ref.attention_bound(want, mass, big, d, max(lens))).all()
    # the products of bf16 values in fp32: K additions of terms whose magnitudes sum to at most this
    x = o.double().cpu().view(n * (T + 1), -1)
    near = (logits.double().cpu() - x @ r.w_plain.t()).abs()
    assert (near <= (hq * d + 4) * 2.0 ** -24 * (x.abs() @ r.w_plain.abs().t())).all()
    z = logits.view(n, T + 1, -1).cpu()
    for i in range(n):
        t, lp, a = ref.verify(z[i], r.draft_logits[i].cpu(), r.drafts[i].cpu(), r.u[i].cpu(), T, 0.8)
        assert tokens[i].tolist() == t + [-1] * (T - a) and int(taken[i]) == a
        assert (lps[i, :a + 1].double().cpu() - torch.tensor(lp)).abs().max() <= 2.0 ** -20
    # token by token: the same keys, so the same attention within its bound
    if T:
        pool = before.clone()
        for t in range(T + 1):
            at = torch.arange(n, device=DEV) * (T + 1) + t
            q1 = sevo.sevo_qk_norm_rope_append_fp8(r.m, 0, r.qkv[at].contiguous(), r.positions[at].contiguous(), r.table, pool)
            assert torch.equal(q1, q[at])
            o1 = sevo.sevo_attn_decode_fp8(q1, pool, r.table, (r.lens + t + 1).contiguous())
            bound = ref.attention_bound(want, mass, big, d, max(lens))[:, t]
            assert ((o1.double().cpu() - want[:, t]).abs() <= bound).all()
        assert torch.equal(pool, r.pool)
    # read back, the prefill's attention runs over it
    full = sevo.sevo_unpack_kv_fp8(r.pool)
    starts = (torch.arange(n + 1, dtype=torch.int32) * (T + 1)).to(DEV)
    op = sevo.sevo_attn_prefill(q, full, r.table, starts, T + 1, start_pos=r.lens)
    # the cache's values rounded to bf16 (half a step of 2^-7) in the scores, and again in V; P in bf16
    rel = torch.expm1(2 * 2.0 ** -8 * big + 1e-3) + 3 * 2.0 ** -8
    assert ((op.view(n, T + 1, hq, d).double().cpu() - want).abs() <= mass * rel + want.abs() * 2.0 ** -8).all()
    r.m.close()


def test_a_step_with_drafts_in_a_graph(sevo):
    """Two captured steps that share the allocator's memory, replayed between eager ones."""
    runs = [Run(sevo, 8, 2, 128, 3, 2, 448, seed=s) for s in (1, 2)]
    eager = []
    for r in runs:
        eager.append([t.clone() for t in r.step(r.pool)] + [r.pool.clone()])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(r.step(r.pool))
        graphs.append(g)
    for rep in range(3):
        for r, g, out, want in zip(runs, graphs, outs, eager):
            r.pool.view(-1)[:] = 0xFF if rep == 1 else r.pool.view(-1)
            if rep == 1:                       # a cache that was spoiled meanwhile: packed again, then the step
                r.pool.copy_(sevo.sevo_pack_kv_fp8(r.bf_pool))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(r.pool, want[-1])
            assert all(torch.equal(a, b) for a, b in zip(r.step(r.pool), want))
    for r in runs:
        r.m.close()


def test_stream_arguments(sevo):
    """Each call on a stream of its own beside work on the current one."""
    r = Run(sevo, 8, 2, 128, 3, 2, 448, seed=3)
    want = [t.clone() for t in r.step(r.pool)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for rep in range(3):
        for s in streams:
            o = sevo.sevo_attn_decode_fp8(want[0].view(3, 3, 8, 128), r.pool, r.table, r.total, stream=s)
            tok = sevo.sevo_verify_drafts(want[2].view(3, 3, -1), r.drafts, r.u, 0.8, draft_logits=r.draft_logits,
                                          stream=s.cuda_stream)
            p8 = sevo.sevo_pack_kv_fp8(r.bf_pool, stream=s)
            s.synchronize()
            assert torch.equal(o, want[1]) and torch.equal(tok[0], want[3]) and torch.equal(tok[1], want[4])
            assert torch.equal(sevo.sevo_unpack_kv_fp8(p8, stream=s).isnan(), torch.zeros_like(r.bf_pool, dtype=torch.bool))
    r.m.close()
