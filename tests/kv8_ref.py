"""Plain float64 forms of the 8-bit cache's operators and of the verification, for the tests."""
import math

import torch

PAGE = 16
F8 = torch.float8_e4m3fn


def k_offsets(d):
    """[16, d]: where the code of K's (slot, dim) is, from the layout's formula."""
    s, e = torch.meshgrid(torch.arange(16), torch.arange(d), indexing="ij")
    return (e // 64) * 1024 + s * 64 + e % 64


def v_offsets(d):
    s, e = torch.meshgrid(torch.arange(16), torch.arange(d), indexing="ij")
    return (e // 64) * 1024 + (s // 4) * 256 + (e % 16) * 16 + ((e // 16) % 4) * 4 + s % 4


def read_pool(pool, d):
    """uint8 [pages, hkv, 32 d + 128] (CPU) -> K and V codes float64 [pages, hkv, 16, d], scales
    float64 [pages, hkv, 16]."""
    pool = pool.cpu()
    out = []
    for base, at in ((0, k_offsets(d)), (16 * d, v_offsets(d))):
        out.append(pool[:, :, base:base + 16 * d].contiguous()[:, :, at].view(F8).double())
    sc = pool[:, :, 32 * d:].contiguous().view(torch.float32).double()
    return out[0], out[1], sc[:, :, :16], sc[:, :, 16:]


def write_pool(k, v, ks, vs):
    """The reverse, from e4m3 codes [pages, hkv, 16, d] and fp32 scales."""
    pages, hkv, _, d = k.shape
    pool = torch.zeros(pages, hkv, 32 * d + 128, dtype=torch.uint8)
    for base, at, c in ((0, k_offsets(d), k), (16 * d, v_offsets(d), v)):
        part = torch.zeros(pages, hkv, 16 * d, dtype=torch.uint8)
        part[:, :, at.reshape(-1)] = c.reshape(pages, hkv, -1).view(torch.uint8)
        pool[:, :, base:base + 16 * d] = part
    pool[:, :, 32 * d:] = torch.cat([ks, vs], 2).float().contiguous().view(torch.uint8)
    return pool


def random_pool(pages, hkv, d, g, loud=3.0):
    """A pool whose slots hold unit-normal values, some dims of K larger."""
    amp = torch.ones(d)
    amp[torch.randint(0, d, (3,), generator=g)] = loud
    parts = []
    for a in (amp, torch.ones(d)):
        y = torch.randn(pages, hkv, 16, d, generator=g) * a
        s = y.abs().amax(3) / 448
        parts.append(((y / s[..., None]).to(F8), s))
    return write_pool(parts[0][0], parts[1][0], parts[0][1], parts[1][1])


def attention(q, pool, table, lens, m, scale):
    """float64 attention of q [n, T, hq, d] over the pool (CPU): (o, the bound of its error's
    terms: sum p |v| per element, the largest sum |q k| scale per row)."""
    n, T, hq, d = q.shape
    hkv = pool.shape[1]
    kc, vc, ks, vs = read_pool(pool, d)
    K, V = kc * ks[..., None], vc * vs[..., None]
    o = torch.zeros(n, T, hq, d, dtype=torch.float64)
    mass, big = torch.zeros_like(o), torch.zeros(n, T, hq, 1, dtype=torch.float64)
    q = q.double().cpu()
    for i in range(n):
        length = int(lens[i])
        ids = table[i, :(length + 15) // 16].tolist()
        where = [(p, t, u) for u in range(length) for p, t in [(ids[u // 16], u % 16)] if 0 <= p < pool.shape[0]]
        for t in range(int(m[i])):
            seen = [(p, s) for p, s, u in where if u < length - int(m[i]) + t + 1]
            if not seen:
                continue
            p, s = torch.tensor([x[0] for x in seen]), torch.tensor([x[1] for x in seen])
            for j in range(hq):
                c = j // (hq // hkv)
                k, v = K[p, c, s], V[p, c, s]
                w = torch.softmax(k @ q[i, t, j] * scale, 0)
                o[i, t, j] = w @ v
                mass[i, t, j] = w @ v.abs()
                big[i, t, j, 0] = (k.abs() @ q[i, t, j].abs()).max() * scale
    return o, mass, big


def attention_bound(o, mass, big, d, keys):
    """How far the kernel's bf16 output may be: a score is off by at most e = (d + 4) 2^-24 of the sum of
    its terms' magnitudes (the products are exact, d additions in fp32, the factors scale and ks), a
    probability by e^(2 e) - 1 (its own and the sum's) and 2^-16 (two bf16 parts, half a step of 2^-7 each)
    and 8 2^-24 (exp2, rescaling), the sums over the keys by keys 2^-24 of their terms;
    the result is rounded to bf16 (half a step of 2^-7)."""
    rel = torch.expm1(2 * (d + 4) * 2.0 ** -24 * big) + 2.0 ** -16 + 8 * 2.0 ** -24 + 2 * keys * 2.0 ** -24
    return mass * rel * (1 + 2.0 ** -8) + o.abs() * 2.0 ** -8 + 1e-38


def verify(z, y, x, u, count, temp):
    """One candidate in float64: (emitted tokens, their log-probabilities, accepted)."""
    z = z.double()
    logp = torch.log_softmax(z / (temp or 1.0), 1)

    def valid(r):
        return bool(torch.isfinite(r).any()) and not bool((torch.isnan(r) | (r == math.inf)).any())

    tokens, lps, a = [], [], 0
    while a < count:
        t = int(x[a])
        if not (0 <= t < z.shape[1]) or not valid(z[a]):
            break
        if temp == 0:
            ok = t == int((z[a] == z[a].max()).nonzero()[0])
        else:
            # (p and q by the same function: those of equal rows are equal)
            q = 1.0 if y is None else float(torch.softmax(y[a].double() / temp, 0)[t])
            ok = float(u[a]) * q < float(torch.softmax(z[a] / temp, 0)[t])
        if not ok:
            break
        tokens.append(t)
        lps.append(float(logp[a, t]))
        a += 1
    if not valid(z[a]):
        return tokens + [-1], lps + [math.nan], a
    if temp == 0:
        t = int((z[a] == z[a].max()).nonzero()[0])
    else:
        # (by the same function as the drafts': of equal rows nothing is left, not even a rounding)
        p = torch.softmax(z[a] / temp, 0)
        r = p
        if a < count:
            if y is not None:
                r = (p - torch.softmax(y[a].double() / temp, 0)).clamp_min(0)
            elif 0 <= int(x[a]) < p.numel():
                r = p.clone()
                r[int(x[a])] = 0
            if not float(r.sum()) > 0:
                r = p
        c = torch.cumsum(r, 0)
        over = (c > float(u[-1]) * c[-1]).nonzero()
        t = int(over[0]) if len(over) else int((r > 0).nonzero()[-1])
    return tokens + [t], lps + [float(logp[a, t])], a
