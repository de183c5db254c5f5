"""The operators of serving and training decoders, as they are measured: rotary positions, the 8-bit paged cache of keys and
values, and attention over it.

Every case names a `kind`:

  rope        flat_attn_rope_fwd, or flat_attn_rope_bwd where "backward" is set, on queries and keys: packed tokens ("packed": slices
              of a fused projection [T, (Hq + 2 Hkv) d]) or dense [B, H, N, d]
  append      flat_attn_cache_append: the keys and values of new tokens into pages of e4m3 values with a scale 2^e a page and head
  attention   flat_attn_cache_fwd: packed queries over that cache; one token a sequence, a few, or chunks of prompts

Plain forms, in 32 bits (angles in 64):

  rope        y = a (x1 cos t - x2 sin t, x2 cos t + x1 sin t) for the pairs (x1, x2) of the first r features, t = position * f_i
  append      e = the least with max|x| <= 448 * 2^e over the page's tokens, not below what older tokens in it had; q = e4m3(x / 2^e)
  attention   O = softmax(scale Q K^T) V with K = 2^(ek - 127) k, V = 2^(ev - 127) v; query i of n sees the keys j <= i + len - n
"""
import math
import random

import torch

own = False

PLAIN, LINEAR, BASE, PARTS = 0, 1, 2, 3       # how the frequencies are scaled for contexts longer than trained on


def listed():
    return [
        # One decode step of a small batch: the smallest call; launches and host time count.  Far positions.
        {"name": "rope_step", "kind": "rope", "packed": True, "tokens": 32, "Hq": 32, "Hkv": 8, "d": 128, "r": 128, "far": 100000},
        # The prompts of a batch at the library's d = 64, neighbouring features paired, half of each head rotated.
        {"name": "rope_prompt_part", "kind": "rope", "B": 4, "N": 4096, "Hq": 16, "Hkv": 16, "d": 64, "r": 32, "interleaved": True},
        # The backward pass of a training step, frequencies scaled by parts.
        {"name": "rope_train_bwd", "kind": "rope", "B": 8, "N": 2048, "Hq": 16, "Hkv": 16, "d": 128, "r": 128, "scaling": PARTS,
         "backward": True},
        # fp32 tensors at a length that no tile divides, a quarter of each head.
        {"name": "rope_fp32_odd", "kind": "rope", "B": 3, "N": 1001, "Hq": 12, "Hkv": 12, "d": 64, "r": 16, "fp32": True, "scaling": LINEAR},
        # One new token for each of many sequences.
        {"name": "append_step", "kind": "append", "seqs": 64, "Hkv": 8, "d": 128, "page": 64, "old": 4000, "new": 1, "mix": 1},
        # Prompts of different lengths behind cached prefixes, in small pages.
        {"name": "append_prompts", "kind": "append", "seqs": 6, "Hkv": 8, "d": 128, "page": 16, "old": 500, "new": 3000, "mix": 2},
        # One sequence, one token: latency.
        {"name": "cache_one_2k", "kind": "attention", "seqs": 1, "Hq": 32, "Hkv": 8, "d": 128, "page": 64, "shortest": 2000, "longest": 2000,
         "new": 1, "mix": 1},
        # A batch of sequences of very different lengths, one token each: the ordinary serving step.
        {"name": "cache_batch_16k", "kind": "attention", "seqs": 64, "Hq": 32, "Hkv": 8, "d": 128, "page": 64, "shortest": 1000,
         "longest": 16384, "new": 1, "mix": 3},
        # As many key heads as query heads, d = 64, small pages.
        {"name": "cache_heads_d64", "kind": "attention", "seqs": 16, "Hq": 16, "Hkv": 16, "d": 64, "page": 16, "shortest": 2048,
         "longest": 8192, "new": 1, "mix": 4},
        # Four drafted tokens a sequence, long contexts, odd numbers of heads a group.
        {"name": "cache_drafts_32k", "kind": "attention", "seqs": 12, "Hq": 28, "Hkv": 4, "d": 128, "page": 32, "shortest": 4000,
         "longest": 32768, "new": 4, "mix": 5},
        # A chunk of a long prompt behind 28K cached tokens: the largest call.
        {"name": "cache_chunk_32k", "kind": "attention", "seqs": 1, "Hq": 32, "Hkv": 8, "d": 128, "page": 128, "shortest": 32768,
         "longest": 32768, "new": 4096, "mix": 6},
        # Two prompts among decoding sequences in one call.
        {"name": "cache_mixed", "kind": "attention", "seqs": 34, "Hq": 16, "Hkv": 4, "d": 64, "page": 64, "shortest": 300,
         "longest": 8000, "new": 1000, "prompts": 2, "mix": 7},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "append", "attention", "attention", "attention"))
    if kind == "rope":
        d = rng.choice((16, 32, 64, 128))
        G = rng.choice((1, 1, 2, 4, 8))
        Hkv = rng.choice((1, 2, 4, 8, 12))
        r = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)))
        case = {"kind": kind, "Hq": G * Hkv, "Hkv": Hkv, "d": d, "r": r, "interleaved": rng.random() < 0.5, "scaling": rng.randrange(4),
                "backward": rng.random() < 0.4, "fp32": rng.random() < 0.25, "far": rng.choice((0, 0, _log(rng, 10, 1000000)))}
        if rng.random() < 0.5:
            case.update(packed=True, tokens=_log(rng, 1, 16384))
        else:
            case.update(B=_log(rng, 1, 16), N=_log(rng, 1, 8192))
        while work(case)["bytes"] > 4e8:
            for key in ("tokens", "B", "N"):
                if case.get(key, 0) > 1:
                    case[key] //= 2
                    break
        return case
    d, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    if kind == "append":
        case = {"kind": kind, "seqs": _log(rng, 1, 128), "Hkv": rng.choice((1, 2, 4, 8, 16)), "d": d, "page": page,
                "old": rng.choice((0, _log(rng, 1, 8192))), "new": rng.choice((1, 1, _log(rng, 2, 4096))), "mix": rng.randrange(1000)}
        while work(case)["bytes"] > 3e8:
            case["seqs"] = max(1, case["seqs"] // 2)
            case["new"] = max(1, case["new"] - case["new"] // 4)
        return case
    use = rng.choice(("step", "step", "drafts", "chunk", "mixed"))
    Hkv, G = rng.choice((1, 2, 4, 8, 16)), rng.choice((1, 1, 2, 3, 4, 4, 5, 7, 8, 16))
    longest = _log(rng, 64, 65536)
    case = {"kind": kind, "seqs": _log(rng, 1, 96), "Hq": G * Hkv, "Hkv": Hkv, "d": d, "page": page,
            "shortest": _log(rng, 1, longest), "longest": longest, "new": 1, "mix": rng.randrange(1000)}
    if use == "drafts":
        case["new"] = rng.randint(2, 8)
    if use == "chunk":
        case.update(new=_log(rng, 16, 4096), seqs=_log(rng, 1, 8))
    if use == "mixed":
        case.update(new=_log(rng, 16, 2048), prompts=rng.randint(1, 4))
    while work(case)["flops"] > 1e12 or work(case)["bytes"] > 1.5e9:
        if case["seqs"] > 1:
            case["seqs"] //= 2
        elif case["Hkv"] > 1:
            case["Hkv"] //= 2
            case["Hq"] //= 2
        else:
            case["longest"] //= 2
            case["shortest"] = min(case["shortest"], case["longest"])
    return case


def _lengths(case):
    """New tokens and lengths with them, sequence by sequence."""
    rng = random.Random(case["mix"])
    if case["kind"] == "append":
        new = [case["new"] if case["new"] < 3 else _log(rng, max(1, case["new"] // 4), case["new"]) for _ in range(case["seqs"])]
        return new, [n + rng.randint(case["old"] // 2, case["old"]) for n in new]
    lens = [_log(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"])]
    new = [min(n, case["new"]) for n in lens]
    if "prompts" in case:
        new = [n if i < case["prompts"] else 1 for i, n in enumerate(new)]
    return new, lens


def work(case):
    d, Hkv = case["d"], case["Hkv"]
    if case["kind"] == "rope":
        size, tokens = 4 if case.get("fp32") else 2, case["tokens"] if case.get("packed") else case["B"] * case["N"]
        heads = case["Hq"] + Hkv
        return {"bytes": 2 * size * tokens * heads * d + 4 * tokens, "flops": 3 * tokens * heads * case["r"]}
    new, lens = _lengths(case)
    if case["kind"] == "append":
        return {"bytes": (4 + 2) * sum(new) * Hkv * d, "flops": 4 * sum(new) * Hkv * d}
    seen = sum(n * m - n * (n - 1) // 2 for n, m in zip(new, lens))
    pages = sum(-(-m // case["page"]) for m in lens)
    return {"bytes": 2 * sum(lens) * Hkv * d + 2 * pages * Hkv + 4 * sum(new) * case["Hq"] * d, "flops": 4 * d * case["Hq"] * seen}


# ---------------------------------------------------------------- inputs

FACTOR, ORIGINAL, BASE_FREQUENCY, LOW, HIGH = 8.0, 4096, 10000.0, 1.0, 32.0


def _frequencies(case):
    """Radians a token, and what the rotated features are multiplied by."""
    r, scaling = case["r"], case.get("scaling", PLAIN)
    base = BASE_FREQUENCY
    if scaling == BASE and r > 2:
        base *= FACTOR ** (r / (r - 2))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if scaling == LINEAR:
        f = f / FACTOR
    if scaling == PARTS:                    # whole turns over the original context: kept; less than one: divided
        kept = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = (1 - kept) * f / FACTOR + kept * f
        return f.cuda(), 0.1 * math.log(FACTOR) + 1
    return f.cuda(), 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, Hkv, d = case["kind"], case["Hkv"], case["d"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, device="cuda", generator=gen, dtype=torch.float32).to(dtype)

    if kind == "rope":
        Hq, dtype = case["Hq"], torch.float32 if case.get("fp32") else torch.bfloat16
        far = case.get("far", 0)
        if case.get("packed"):              # one token of each sequence, anywhere in it
            tokens = case["tokens"]
            fused = normal(tokens, (Hq + 2 * Hkv) * d, dtype=dtype)
            Q, K = fused[:, :Hq * d].view(tokens, Hq, d), fused[:, Hq * d:(Hq + Hkv) * d].view(tokens, Hkv, d)
            positions = torch.randint(0, far + 8192, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
        else:
            Q, K = normal(case["B"], Hq, case["N"], d, dtype=dtype), normal(case["B"], Hkv, case["N"], d, dtype=dtype)
            positions = torch.arange(far, far + case["N"], device="cuda", dtype=torch.int32)
        s = {"kind": kind, "Q": Q, "K": K, "positions": positions, "interleaved": bool(case.get("interleaved")), "r": case["r"],
             "backward": bool(case.get("backward"))}
        s["f"], s["a"] = _frequencies(case)
        s["Qr"], s["Kr"] = torch.empty(Q.shape, dtype=dtype, device="cuda"), torch.empty(K.shape, dtype=dtype, device="cuda")
        if own:
            from paper_2107_06419_b200 import api
            s["table"], s["amplitude"] = api.flat_attn_rope_table(case["r"], BASE_FREQUENCY, scaling=case.get("scaling", PLAIN), factor=FACTOR,
                                                                  original_len=ORIGINAL, low=LOW, high=HIGH)
        return s

    new, lens = _lengths(case)
    page, S = case["page"], len(lens)
    counts = [-(-m // page) for m in lens]
    num_pages = sum(counts) + max(4, sum(counts) // 16)
    order = torch.randperm(num_pages, device="cuda", generator=gen, dtype=torch.int32)
    table = torch.zeros(S, max(counts), dtype=torch.int32)
    host_order, at = order.cpu(), 0
    for i, n in enumerate(counts):
        table[i, :n] = host_order[at:at + n]
        at += n
    s = {"kind": kind, "page": page, "new": new, "lens": lens, "table": table.cuda(),
         "cu": torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda(),
         "seq_lens": torch.tensor(lens, dtype=torch.int32).cuda()}
    # Cached values as a program has them: each page and head with its own spread, the largest value near the top of the type's range
    for name in ("k", "v"):
        cache = torch.empty(num_pages, Hkv, page, d, dtype=torch.float8_e4m3fn, device="cuda")
        for first in range(0, num_pages, 2048):
            some = cache[first:first + 2048]
            some.copy_((torch.randn(some.shape, device="cuda", generator=gen) * 80).clamp(-448, 448))
        s[name + "_cache"] = cache
        s[name + "_exp"] = torch.randint(118, 123, (num_pages, Hkv), device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8)
    T = sum(new)
    if kind == "append":                    # keys come from the rotation, values as a slice of the projections
        s["K"] = normal(T, Hkv, d)
        s["V"] = normal(T, 2 * Hkv * d)[:, Hkv * d:].view(T, Hkv, d)
        s["most"] = max(new)
        return s
    s["Q"] = normal(T, case["Hq"], d)
    s["O"] = torch.empty_like(s["Q"])
    s["scale"], s["most"] = d ** -0.5, max(new)
    if own:
        from paper_2107_06419_b200 import api
        s["workspace"] = torch.zeros(api.flat_attn_cache_workspace_bytes(case["Hq"], Hkv, d), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- one pass

def _rotate(x, s):
    x1, x2 = (x[..., 0:s["r"]:2], x[..., 1:s["r"]:2]) if s["interleaved"] else (x[..., :s["r"] // 2], x[..., s["r"] // 2:s["r"]])
    angles = s["positions"].double()[:, None] * s["f"]
    cos, sin = (s["a"] * torch.cos(angles)).float(), (s["a"] * torch.sin(angles)).float()
    if x.dim() == 3:
        cos, sin = cos[:, None], sin[:, None]
    if s["backward"]:
        sin = -sin
    x1, x2 = x1.float(), x2.float()
    y = x.float().clone() if s["r"] < x.shape[-1] else torch.empty(x.shape, dtype=torch.float32, device=x.device)
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    if s["interleaved"]:
        y[..., 0:s["r"]:2], y[..., 1:s["r"]:2] = y1, y2
    else:
        y[..., :s["r"] // 2], y[..., s["r"] // 2:s["r"]] = y1, y2
    return y.to(x.dtype)


def _append(x, cache, exp, s):
    """The new tokens' rows x [T, Hkv, d] into the cache."""
    page, first = s["page"], 0
    for i, (n, m) in enumerate(zip(s["new"], s["lens"])):
        start, p0, p1 = m - n, (m - n) // page, -(-m // page)
        ids = s["table"][i, p0:p1].long()
        old = start - p0 * page                                            # older tokens in the first of these pages
        rows = torch.zeros((p1 - p0) * page, *x.shape[1:], dtype=torch.float32, device=x.device)
        rows[old:old + n] = x[first:first + n].float()
        rows = rows.view(p1 - p0, page, *x.shape[1:]).transpose(1, 2)      # [pages, Hkv, page, d]
        top = rows.abs().amax((2, 3))
        mantissa, e = torch.frexp(top)                                     # top = mantissa 2^e, mantissa in [0.5, 1); 448 = 0.875 * 2^9
        e = torch.where(top > 0, e - 9 + (mantissa > 0.875), -117).clamp(-117, 120).int() + 127
        if old:
            e[0] = torch.maximum(e[0], exp[ids[0]].int())
            earlier = cache[ids[0]][:, :old].float() * torch.exp2((exp[ids[0]].int() - e[0]).float())[:, None, None]
        codes = (rows * torch.exp2((127 - e).float())[:, :, None, None]).to(cache.dtype)
        at = torch.arange(start, m, device=x.device)
        cache.view(torch.uint8)[ids[at // page - p0], :, at % page] = codes.view(torch.uint8)[at // page - p0, :, at % page]
        if old:
            cache.view(torch.uint8)[ids[0], :, :old] = earlier.to(cache.dtype).view(torch.uint8)
        exp[ids] = e.to(torch.uint8)
        first += n


def _values(cache, exp, ids, m):
    """The first m tokens of the pages `ids`: [Hkv, m, d]."""
    x = cache[ids].float() * torch.exp2(exp[ids].float() - 127)[:, :, None, None]
    return x.transpose(0, 1).flatten(1, 2)[:, :m]


def _attend(s):
    Q, O, Hkv, page, first = s["Q"], s["O"], s["k_cache"].shape[1], s["page"], 0
    G = Q.shape[1] // Hkv
    for i, (n, m) in enumerate(zip(s["new"], s["lens"])):
        ids = s["table"][i, :-(-m // page)].long()
        k, v = _values(s["k_cache"], s["k_exp"], ids, m), _values(s["v_cache"], s["v_exp"], ids, m)
        q = Q[first:first + n].float().view(n, Hkv, G, -1)
        hidden = torch.arange(m, device=Q.device)[None, :] > torch.arange(n, device=Q.device)[:, None] + (m - n)
        for h in range(Hkv):
            x = (q[:, h].flatten(0, 1) @ k[h].T) * s["scale"]              # [n G, m]
            if n > 1:
                x.view(n, G, m).masked_fill_(hidden[:, None], float("-inf"))
            x = torch.exp(x - x.amax(1, keepdim=True))
            O[first:first + n, h * G:(h + 1) * G] = ((x @ v[h]) / x.sum(1, keepdim=True)).view(n, G, -1).to(O.dtype)
        first += n


def run(s):
    kind = s["kind"]
    if own:
        from paper_2107_06419_b200 import api
        if kind == "rope":
            rotate = api.flat_attn_rope_bwd if s["backward"] else api.flat_attn_rope_fwd
            rotate(s["Q"], s["K"], s["table"], s["Qr"], s["Kr"], positions=s["positions"], interleaved=s["interleaved"],
                   amplitude=s["amplitude"])
            return {"Q": s["Qr"], "K": s["Kr"]}
        if kind == "append":
            api.flat_attn_cache_append(s["K"], s["V"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["table"], s["cu"],
                                       s["seq_lens"], s["most"])
            return {name: s[name] for name in ("k_cache", "v_cache", "k_exp", "v_exp")}
        return api.flat_attn_cache_fwd(s["Q"], s["O"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"], s["table"], s["cu"],
                                       s["seq_lens"], s["most"], s["scale"], s["workspace"], causal=True)
    if kind == "rope":
        return {"Q": _rotate(s["Q"], s), "K": _rotate(s["K"], s)}
    if kind == "append":
        _append(s["K"], s["k_cache"], s["k_exp"], s)
        _append(s["V"], s["v_cache"], s["v_exp"], s)
        return {name: s[name] for name in ("k_cache", "v_cache", "k_exp", "v_exp")}
    _attend(s)
    return s["O"]


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        turn = torch.polar(torch.full((1,), float(s["a"]), dtype=torch.float64, device="cuda"),
                           (s["positions"].double()[:, None] * s["f"]) * (-1 if s["backward"] else 1))

        def rotated(x):
            y = x.double().clone()
            part = y[..., :case["r"]]
            pairs = part.unflatten(-1, (-1, 2)) if s["interleaved"] else part.unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_complex(pairs.contiguous()) * (turn[:, None] if x.dim() == 3 else turn)
            z = torch.view_as_real(z)
            y[..., :case["r"]] = (z if s["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            return y
        return {"Q": rotated(s["Q"]), "K": rotated(s["K"])}
    page, table = case["page"], s["table"].cpu()
    if case["kind"] == "append":
        if sum(s["new"]) // page + len(s["new"]) > 8000:                   # (page by page: too long)
            return None
        for name in ("k", "v"):
            cache, exp, x = s[name + "_cache"], s[name + "_exp"], s[name.upper()].double()
            scales, first = exp.cpu().tolist(), 0
            for i, (n, m) in enumerate(zip(s["new"], s["lens"])):
                at = m - n
                while at < m:                                              # page by page
                    p, r0 = int(table[i, at // page]), at % page
                    r1 = min(page, r0 + m - at)
                    rows = x[first:first + r1 - r0].transpose(0, 1)        # [Hkv, tokens, d]
                    tops = rows.abs().amax((1, 2)).tolist()
                    for h, top in enumerate(tops):
                        e = -117
                        if top > 0:
                            e = max(-117, math.frexp(top)[1] - 10)
                            while top > 448 * 2.0 ** e:
                                e += 1
                        was = scales[p][h] - 127
                        if r0 and was < e:
                            cache[p, h, :r0] = (cache[p, h, :r0].double() * 2.0 ** (was - e)).to(cache.dtype)
                        scales[p][h] = (max(e, was) if r0 else e) + 127
                    down = 2.0 ** (127 - torch.tensor(scales[p], dtype=torch.float64, device="cuda"))
                    cache[p, :, r0:r1] = (rows * down[:, None, None]).to(cache.dtype)
                    at, first = at + r1 - r0, first + r1 - r0
            s[name + "_exp"] = torch.tensor(scales, dtype=torch.uint8, device="cuda")
        return {name: s[name] for name in ("k_cache", "v_cache", "k_exp", "v_exp")}
    Hkv, G, out, first = case["Hkv"], case["Hq"] // case["Hkv"], torch.empty(s["Q"].shape, dtype=torch.float64, device="cuda"), 0
    for i, (n, m) in enumerate(zip(s["new"], s["lens"])):
        at = torch.arange(m, device="cuda")
        ids = s["table"][i].long()[at // page]
        for h in range(Hkv):
            k, v = (s[c + "_cache"][ids, h, at % page].double() * torch.pow(2.0, s[c + "_exp"][ids, h].double() - 127)[:, None] for c in "kv")
            for r in range(0, n, 512):                                     # queries, a few at a time
                few = slice(first + r, first + min(n, r + 512))
                q = s["Q"][few, h * G:(h + 1) * G].double()
                logits = torch.einsum("tgc,jc->tgj", q, k) * s["scale"]
                last = torch.arange(r, min(n, r + 512), device="cuda") + m - n
                logits = logits.masked_fill((at > last[:, None])[:, None], -math.inf)
                out[few, h * G:(h + 1) * G] = torch.einsum("tgj,jc->tgc", torch.softmax(logits, -1), v)
        first += n
    return out
