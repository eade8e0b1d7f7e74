"""The 8-bit cache's operators at sizes that take their other paths: contexts in more splits than a join
takes at once, splits in several rounds of workgroups, waves with more pages than they hold the ids of, calls
larger than the last-level cache, more tiles than a launch has waves."""
import math

import pytest
import torch

from tests import kv8_ref as ref
from tests.test_gpu_kv8 import bf_tiles, gen, model, sevo  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def bytes_pool(pages, hkv, d, g):
    """A pool of random codes (no NaN) on g's device, K's scales near 2^-9, those of V spread over a
    factor of 16, so that every page counts."""
    pool = torch.randint(0, 256, (pages, hkv, 32 * d + 128), generator=g, dtype=torch.uint8, device=g.device)
    codes = pool[:, :, :32 * d]
    codes[(codes & 0x7F) == 0x7F] = 0
    u = torch.rand(pages, hkv, 32, generator=g, device=g.device)
    scales = torch.where(torch.arange(32, device=g.device) < 16, (1 + u) * 2.0 ** -9, 2.0 ** (4 * u - 8))
    pool[:, :, 32 * d:] = scales.view(torch.uint8)
    return pool


def attention(q, pool, table, length, m, scale, heads):
    """float64 attention of one candidate's q [T, hq, d] on ``pool``'s device, for the kv heads in ``heads``:
    o, sum p |v|, largest sum |q k| scale, each [T, len(heads), G, ..].  A key counts by its page and slot, however
    often the table holds the page."""
    T, hq, d = q.shape
    G = hq // pool.shape[1]
    ids = table.long()
    ids = torch.where((ids >= 0) & (ids < pool.shape[0]), ids, -1)
    at = torch.arange(length, device=pool.device)
    slot = ids[at // 16] * 16 + at % 16
    o, mass, big = [], [], []
    for c in heads:
        part = pool[:, c:c + 1]
        k, v, ks, vs = (x.to(pool.device) for x in ref.read_pool(part, d))
        K = (k * ks[..., None]).reshape(-1, d)
        V = (v * vs[..., None]).reshape(-1, d)
        for t in range(T):
            seen = slot[:max(0, length - m + t + 1)]
            count = torch.bincount(seen[seen >= 0], minlength=K.shape[0]).double()
            qh = q[t, c * G:(c + 1) * G].double().to(pool.device)
            z = torch.mm(K, qh.t().contiguous()) * scale                     # [slots, G]
            z = torch.where(count[:, None] > 0, z, -math.inf)
            w = count[:, None] * torch.exp(z - z.amax(0))
            w = (w / w.sum(0)).t().contiguous()
            o.append(torch.mm(w, V))
            mass.append(torch.mm(w, V.abs()))
            b = torch.mm(K.abs(), qh.abs().t().contiguous()) * scale
            big.append(torch.where(count[:, None] > 0, b, 0.0).amax(0)[:, None])
    return [torch.stack(x).view(len(heads), T, G, -1).transpose(0, 1) for x in (o, mass, big)]


# name: query heads, kv heads, head dim, new tokens, keys of the candidates, pages of the pool, splits of the longest
# candidate, pages of a split, waves that take a split's pages, kv heads that are compared
CASES = {
    # a chunk of more than 16 pages; four waves join 94 splits, 24 each
    "one_64k": (8, 8, 128, 1, [65537], 4097, 94, 44, 4, range(8)),
    # four waves join 274 splits: two turns of 64 each
    "one_70k": (4, 1, 64, 3, [70001], 4376, 274, 16, 4, [0]),
    # one wave joins 69 splits: nine batches of eight, two turns of 64
    "one_of_64": (2, 1, 64, 1, [1100 * 16 - 5] + [9] * 63, 1163, 69, 16, 4, [0]),
    # the most pages that go in one round, and what goes in several
    "round_full": (64, 64, 64, 1, [11 * 192 * 16], 60, 11, 192, 4, [0, 1, 31, 63]),
    "rounds": (64, 64, 64, 1, [11 * 192 * 16 + 1], 60, 23, 96, 4, [0, 1, 31, 63]),
    "rounds_128": (64, 32, 128, 2, [71234], 70, 47, 96, 4, [0, 17, 31]),
    # 75 and 69 pairs of pages a wave
    "ids_64": (2048, 2048, 64, 1, [9600 - 3], 40, 1, 600, 4, [0, 1, 1000, 2047]),
    "ids_128": (1024, 1024, 128, 1, [1100 * 16 - 20], 40, 2, 550, 4, [0, 3, 600, 1023]),
}


def make(name, device):
    hq, hkv, d, T, lens, pages, splits, chunk, waves, heads = CASES[name]
    g = torch.Generator(device=device).manual_seed(sum(map(ord, name)))
    pool = bytes_pool(pages, hkv, d, g)
    width = max(-(-x // 16) for x in lens)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=device)
    need = sum(-(-x // 16) for x in lens)
    ids = (torch.randperm(pages, generator=g, device=device) if need <= pages
           else torch.randint(0, pages, (need,), generator=g, device=device)).to(torch.int32)
    at = 0
    for i, x in enumerate(lens):
        table[i, :-(-x // 16)] = ids[at:at - (-x // 16)]
        at -= -x // 16
    q = (torch.randn(len(lens), T, hq, d, generator=g, device=device) * 0.6).to(BF)
    return pool, table, q


@pytest.mark.parametrize("name", list(CASES))
def test_attention_of_long_contexts(sevo, name):  # noqa: F811
    hq, hkv, d, T, lens, pages, splits, chunk, waves, heads = CASES[name]
    pool, table, q = make(name, DEV)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    scale = d ** -0.5
    got = sevo.sevo_attn_decode_fp8(q, pool, table, length)
    G = hq // hkv
    for i in ([0] if len(lens) == 1 else [0, 1, len(lens) - 1]):
        o, mass, big = attention(q[i], pool, table[i], lens[i], T, scale, heads)
        # the longest chain of fp32 additions: a wave's keys of a split, the waves, the splits
        chain = (chunk + 2) * 16 // waves + waves + splits + 64
        bound = ref.attention_bound(o, mass, big, d, chain)
        x = got[i].view(T, hkv, G, d)[:, list(heads)].double()
        assert ((x - o).abs() <= bound).all(), (i, float(((x - o).abs() / bound).max()))
    for _ in range(3):
        assert torch.equal(sevo.sevo_attn_decode_fp8(q, pool, table, length), got)


@pytest.mark.parametrize("hq,hkv,d,n", [(64, 8, 128, 4601), (64, 8, 64, 9103)])
def test_append_beyond_the_caches(sevo, hq, hkv, d, n):  # noqa: F811
    """A call of more than 256 MiB gives the bits of calls of a seventh."""
    assert n * d * (6 * hq + 10 * hkv) > 256 << 20
    g = torch.Generator(device=DEV).manual_seed(d)
    m = model(sevo, hq, hkv, d, max_position=n)
    table = torch.randperm(-(-n // 16), generator=g, device=DEV).view(1, -1).to(torch.int32)
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g, device=DEV)
    pos, rows = torch.arange(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    a, b = (torch.zeros(table.shape[1], hkv, 32 * d + 128, dtype=torch.uint8, device=DEV) for _ in range(2))
    qa = sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv, pos, table, a, rows=rows)
    step = -(-n // 7)
    qb = torch.cat([sevo.sevo_qk_norm_rope_append_fp8(m, 0, qkv[i:i + step], pos[i:i + step], table, b,
                                                      rows=rows[i:i + step]) for i in range(0, n, step)])
    assert torch.equal(qa, qb) and torch.equal(a, b) and bool(a.any())
    m.close()


@pytest.mark.parametrize("hkv,d,pages", [(8, 128, 2703), (8, 64, 5351)])
def test_pages_beyond_the_caches(sevo, hkv, d, pages):  # noqa: F811
    assert pages * hkv * (96 * d + 128) > 256 << 20
    g = torch.Generator(device=DEV).manual_seed(d)
    pool = torch.randn(pages, hkv, 2, 16 * d, generator=g, device=DEV).to(BF)
    src = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    packed = sevo.sevo_pack_kv_fp8(pool, src_pages=src)
    few = [src[i:i + 500].contiguous() for i in range(0, pages, 500)]
    assert torch.equal(packed, torch.cat([sevo.sevo_pack_kv_fp8(pool, src_pages=x) for x in few]))
    back = sevo.sevo_unpack_kv_fp8(packed, src_pages=src)
    assert torch.equal(back, torch.cat([sevo.sevo_unpack_kv_fp8(packed, src_pages=x) for x in few]))


@pytest.mark.parametrize("to8", [True, False])
@pytest.mark.parametrize("hkv,d", [(8, 128), (7, 64)])
def test_more_tiles_than_a_launch_has_waves(sevo, hkv, d, to8):  # noqa: F811
    """Entries past 65536 workgroups' tiles; most of them have no destination."""
    count = 65536 * 4 * (2 if to8 and d == 64 else 1) // hkv + 103
    g = torch.Generator(device=DEV).manual_seed(d)
    plain = torch.randn(6, hkv, 2, 16 * d, generator=g, device=DEV).to(BF)
    pool = plain if to8 else sevo.sevo_pack_kv_fp8(plain)
    call = sevo.sevo_pack_kv_fp8 if to8 else sevo.sevo_unpack_kv_fp8
    want = call(pool)
    src = torch.randint(0, 6, (count,), generator=g, device=DEV, dtype=torch.int32)
    at = torch.cat([torch.arange(0, 5), torch.arange(count // 2, count // 2 + 5), torch.arange(count - 120, count)]).to(DEV)
    dst = torch.full((count,), -1, dtype=torch.int32, device=DEV)
    dst[at] = torch.randperm(len(at), generator=g, device=DEV).to(torch.int32)
    into = torch.zeros(len(at), *want.shape[1:], dtype=want.dtype, device=DEV)
    call(pool, into, src, dst)
    assert torch.equal(into[dst[at].long()], want[src[at].long()])
