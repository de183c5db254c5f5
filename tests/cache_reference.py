"""Plain float64 forms of the operators around the 8-bit paged cache, one sequence, page and head at a time (any device)."""
import math

import torch

E4M3_MAX = 448.0


def exponent(top):
    """The least e >= -117 with top <= 448 * 2^e."""
    if top == 0:
        return -117
    e = math.frexp(top)[1] - 10
    while top > math.ldexp(E4M3_MAX, e):
        e += 1
    return max(e, -117)


def append(x, cache, exp, table, cu, lens):
    """x [T, Hkv, d] float64 into cache (float8 [pages, Hkv, page, d]) and exp (uint8), in place."""
    page = cache.shape[2]
    for s in range(len(lens)):
        first, n = cu[s], cu[s + 1] - cu[s]
        at = lens[s] - n
        while at < lens[s]:
            p, r0 = int(table[s][at // page]), at % page
            r1 = min(page, r0 + lens[s] - at)
            for h in range(cache.shape[1]):
                rows = x[first:first + r1 - r0, h]
                finite = rows[torch.isfinite(rows)]
                e = exponent(float(finite.abs().max()) if finite.numel() else 0.0)
                if r0:
                    was = int(exp[p, h]) - 127
                    if was < e:
                        cache[p, h, :r0] = (cache[p, h, :r0].double() * 2.0 ** (was - e)).to(cache.dtype)
                    e = max(e, was)
                q = torch.where(torch.isfinite(rows), rows * 2.0 ** -e, math.nan)
                cache[p, h, r0:r1] = q.to(cache.dtype)
                exp[p, h] = e + 127
            first, at = first + r1 - r0, at + r1 - r0


def values(cache, exp, ids, m, h):
    page = cache.shape[2]
    x = torch.cat([cache[i, h].double() * 2.0 ** (int(exp[i, h]) - 127) for i in ids])
    return x[:m]


def attention(Q, k_cache, v_cache, k_exp, v_exp, table, cu, lens, scale, causal, dropped=()):
    """O, lse and two measures of how far rounding may take them: sum of w |v| a feature, and the largest sum of |q k scale|.
    dropped: (sequence, page place) pairs whose tokens take no part."""
    T, Hq, d = Q.shape
    Hkv, page = k_cache.shape[1], k_cache.shape[2]
    G = Hq // Hkv
    O = torch.full((T, Hq, d), math.nan, dtype=torch.float64, device=Q.device)
    A, lse, B = torch.zeros_like(O), O[..., 0].clone(), O[..., 0].clone()
    for s in range(len(lens)):
        n, m = cu[s + 1] - cu[s], lens[s]
        if n == 0:
            continue
        ids = [int(i) for i in table[s][:-(-m // page)]]
        gone = {p for (t, p) in dropped if t == s}
        safe = [0 if p in gone else i for p, i in enumerate(ids)]
        at = torch.arange(m, device=Q.device)
        seen = torch.ones(n, m, dtype=torch.bool, device=Q.device)
        if causal:
            seen &= at[None] <= torch.arange(n, device=Q.device)[:, None] + m - n
        for p in gone:
            seen[:, p * page:(p + 1) * page] = False
        for h in range(Hkv):
            k, v = values(k_cache, k_exp, safe, m, h), values(v_cache, v_exp, safe, m, h)
            for g in range(h * G, (h + 1) * G):
                q = Q[cu[s]:cu[s + 1], g].double()
                x = (q @ k.T * scale).masked_fill(~seen, -math.inf)
                lse[cu[s]:cu[s + 1], g] = torch.logsumexp(x, 1)
                w = torch.nan_to_num(torch.softmax(x, 1), nan=0.0) if not seen.any(1).all() else torch.softmax(x, 1)
                O[cu[s]:cu[s + 1], g] = w @ v
                A[cu[s]:cu[s + 1], g] = w @ v.abs()
                B[cu[s]:cu[s + 1], g] = (q.abs() @ k.abs().T).max(1).values * abs(scale)
    return O, lse, A, B


def check_attention(O, lse, ref, d, what=""):
    """O within the rounding of the result (bf16: half a step, 2^-8), of the weights (half precision: 2^-11 each of sum w |v|; as much
    again for sums and exponentials in fp32) and, through the weights, of the logits (d products summed in fp32); lse likewise."""
    R, L, A, B = ref
    rows = ~torch.isnan(R[..., 0])
    logits = d * 2.0 ** -24 * B
    tol = 2.0 ** -8 * R.abs() + (2.0 ** -10 + 2 * logits[..., None]) * A + 1e-30
    err = (O.double() - R).abs()
    assert torch.isfinite(O[rows].float()).all(), what
    bad = (err > tol) & rows[..., None]
    assert not bad.any(), (what, int(bad.sum()), float((err / tol)[rows].max()))
    if lse is not None:
        live = rows & torch.isfinite(L)
        assert ((lse.double() - L).abs()[live] <= (logits + 2.0 ** -18 * (1 + L.abs()))[live]).all(), (what, float((lse.double() - L).abs()[live].max()))
        assert (lse[rows & ~live] == -math.inf).all(), what


def make_cache(gen, lens, Hkv, page, d, device, spare=3, exps=(112, 124), max_pages=None):
    """Random pages in random order; every page and head with a scale of its own."""
    counts = [-(-m // page) for m in lens]
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max_pages or max(max(counts), 1)), -7, dtype=torch.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    cache = [(torch.randn(pages, Hkv, page, d, generator=gen) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).to(device) for _ in range(2)]
    exp = [torch.randint(*exps, (pages, Hkv), generator=gen).to(torch.uint8).to(device) for _ in range(2)]
    return cache[0], cache[1], exp[0], exp[1], table.to(device)


def offsets(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return cu
