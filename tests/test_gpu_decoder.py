"""Rotary positions, the 8-bit paged cache and its attention between the library's projections, as a decoder uses them; and the rotation
around the attention and its backward pass, as training uses it."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2107_06419_b200 import api as _api
    return _api


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def half_step(x):
    return 2.0 ** -8 * x.abs()


@pytest.mark.parametrize("d,page,interleaved", [(64, 16, False), (128, 64, True)])
def test_prompts_then_tokens(api, d, page, interleaved):
    """Two prompts at once, then one token a sequence, five times: what each step's attention gives is what the plain form gives for the
    rotated queries and the cache's values at hand, and the cache is what the plain form makes of the rotated keys."""
    gen = torch.Generator().manual_seed(d)
    Hq, Hkv, Dm, S, T = 8, 2, 256, 2, 256                # T: rows of the projections (a multiple of 128); the last ones are padding
    heads = Hq + 2 * Hkv
    W = (torch.randn(-(-heads * d // 256) * 256, Dm, generator=gen) * Dm ** -0.5).to(torch.bfloat16).cuda()
    Wo = (torch.randn(Dm, Hq * d, generator=gen) * (Hq * d) ** -0.5).to(torch.bfloat16).cuda()
    table, amplitude = api.flat_attn_rope_table(d, scaling=api.FLAT_ROPE_BASE, factor=4.0)
    prompts = [150, 77]
    most = max(prompts) + 8
    max_pages, pages = -(-most // page), 2 * -(-most // page) + 3
    k = torch.zeros(pages, Hkv, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v, ke = k.clone(), torch.zeros(pages, Hkv, dtype=torch.uint8, device="cuda")
    ve = ke.clone()
    order = torch.randperm(pages, generator=gen).to(torch.int32)
    pages_of = order[:2 * max_pages].view(2, max_pages).cuda()
    want = [t.clone() for t in (k, v, ke, ve)]
    work = torch.zeros(api.flat_attn_cache_workspace_bytes(Hq, Hkv, d), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = [0, 0]
    for step in range(6):
        new = prompts if step == 0 else [1, 1]
        lens = [a + b for a, b in zip(lens, new)]
        cu, used = ref.offsets(new), sum(new)
        X = torch.randn(T, Dm, generator=gen).to(torch.bfloat16).cuda()
        Y = torch.empty(T, W.shape[0], dtype=torch.bfloat16, device="cuda")
        api.flat_fc_fwd(X, W, Y)
        Q, K, V = (Y[:, a * d:b * d].view(T, b - a, d) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, heads)))
        at = torch.zeros(T, dtype=torch.int32)
        at[:used] = torch.cat([torch.arange(m - n, m) for n, m in zip(new, lens)])
        rotated_q = torch.empty(T, Hq, d, dtype=torch.bfloat16, device="cuda")
        api.flat_attn_rope_fwd(Q, K, table, rotated_q, K, positions=at.cuda(), interleaved=interleaved, amplitude=amplitude)
        args = (k, v, ke, ve, pages_of, ints(cu), ints(lens))
        api.flat_attn_cache_append(K, V, *args, max(new), status=status)
        O = torch.zeros(1, Hq, T, d, dtype=torch.bfloat16, device="cuda")        # (head-major, as the output projection reads it)
        api.flat_attn_cache_fwd(rotated_q, O[0].transpose(0, 1), *args, max(new), d ** -0.5, work, causal=True, status=status)
        out = torch.empty(1, T, Dm, dtype=torch.bfloat16, device="cuda")
        api.flat_out_proj_fwd(O, Wo, out)
        torch.cuda.synchronize()
        assert int(status) == 0
        ref.append(K[:used].double(), want[0], want[2], pages_of.tolist(), cu, lens)
        ref.append(V[:used].double(), want[1], want[3], pages_of.tolist(), cu, lens)
        for got, w in zip((k, v, ke, ve), want):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8)), step
        o = O[0].transpose(0, 1)
        ref.check_attention(o[:used], None, ref.attention(rotated_q[:used], *want, pages_of.tolist(), cu, lens, d ** -0.5, True), d, str(step))
        assert (o[used:] == 0).all()
        flat = o.reshape(T, Hq * d).double()
        y = flat @ Wo.double().T
        tol = half_step(y) + Hq * d * 2.0 ** -24 * (flat.abs() @ Wo.double().abs().T) + 1e-6
        assert ((out[0].double() - y).abs() <= tol).all()


@pytest.mark.parametrize("new,lens", [([300, 1, 1, 70], [1000, 2000, 64, 70]), ([1, 400, 1], [5, 400, 3000])])
def test_a_prompt_at_once_is_its_tokens_one_by_one(api, new, lens):
    """The rows of a mixed batch, which two kernels share, against calls of one query a sequence: both within rounding of the same values."""
    gen = torch.Generator().manual_seed(2)
    Hkv, G, d, page = 2, 4, 64, 32
    cu = ref.offsets(new)
    cache = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    Q = torch.randn(cu[-1], G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O, work = torch.empty_like(Q), torch.zeros(api.flat_attn_cache_workspace_bytes(G * Hkv, Hkv, d), dtype=torch.uint8, device="cuda")
    api.flat_attn_cache_fwd(Q, O, *cache, ints(cu), ints(lens), max(new), 0.125, work, causal=True)
    one = torch.empty_like(Q)
    for i in range(max(new)):
        live = [s for s in range(len(new)) if i < new[s]]
        q = torch.stack([Q[cu[s] + i] for s in live])
        o = torch.empty_like(q)
        table = torch.stack([cache[4][s] for s in live])
        api.flat_attn_cache_fwd(q, o, *cache[:4], table, ints(list(range(len(live) + 1))), ints([lens[s] - new[s] + i + 1 for s in live]), 1, 0.125, work)
        for j, s in enumerate(live):
            one[cu[s] + i] = o[j]
    torch.cuda.synchronize()
    want = ref.attention(Q, *cache, cu, lens, 0.125, True)
    ref.check_attention(O, None, want, d)
    ref.check_attention(one, None, want, d)


def test_mixed_batch_in_a_graph_between_other_calls(api):
    """The two kernels of a mixed call run side by side; what was before is done when they begin, and both are done when what follows begins."""
    gen = torch.Generator().manual_seed(4)
    Hkv, G, d, page, new, lens = 4, 4, 128, 64, [700, 1, 1, 30, 1], [2000, 9000, 40, 333, 5000]
    cu, T = ref.offsets(new), sum(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    base = torch.randn(T, G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    rope, _ = api.flat_attn_rope_table(d)
    at = torch.zeros(T, dtype=torch.int32, device="cuda")
    work = torch.zeros(api.flat_attn_cache_workspace_bytes(G * Hkv, Hkv, d), dtype=torch.uint8, device="cuda")
    Q, O, out = torch.empty_like(base), torch.empty_like(base), torch.empty_like(base)
    dcu, dlens = ints(cu), ints(lens)

    def step():
        api.flat_attn_rope_fwd(base, None, rope, Q, None, positions=at)              # writes the queries
        api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, dcu, dlens, max(new), 0.1, work, causal=True)
        api.flat_attn_rope_fwd(O, None, rope, out, None, positions=at)               # reads the outputs (angles of 0: a copy)
        O.zero_()
    step()
    torch.cuda.synchronize()
    assert api.flat_attn_last_launch_count() == 1 and torch.equal(Q, base)
    first = out.clone()
    ref.check_attention(first, None, ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True), d)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(5):
            step()
    for _ in range(10):
        Q.zero_()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_many_empty_sequences_around_long_ones(api):
    """A batch padded to a fixed number of sequences: those without tokens own nothing, whatever their table holds."""
    gen = torch.Generator().manual_seed(5)
    Hkv, G, d, page, S = 4, 2, 64, 16, 700
    lens, new = [0] * S, [0] * S
    for s, m in ((3, 9000), (4, 1), (350, 2500), (699, 77)):
        lens[s], new[s] = m, 1
    cu = ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    for s in range(S):
        if not new[s]:
            table[s] = 1 << 28
    lens_given = list(lens)
    lens_given[10] = 40                                  # cached tokens, none of them new
    Q = torch.randn(6, G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O, status = torch.full_like(Q, 3.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    work = torch.zeros(api.flat_attn_cache_workspace_bytes(G * Hkv, Hkv, d), dtype=torch.uint8, device="cuda")
    K = torch.randn(6, Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    want = [t.clone() for t in (k, v, ke, ve)]
    ref.append(K.double(), want[0], want[2], table.tolist(), cu, lens)
    ref.append(K.double(), want[1], want[3], table.tolist(), cu, lens)
    for most in (1, 5):                                  # (the form for one token, and the other)
        api.flat_attn_cache_append(K, K, k, v, ke, ve, table, ints(cu), ints(lens_given), most, status=status)
        torch.cuda.synchronize()
        for got, w in zip((k, v, ke, ve), want):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
    for most in (1, 6):
        api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens_given), most, 0.1, work, causal=True, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0 and (O[4:] == 3.0).all()
        ref.check_attention(O[:4], None, ref.attention(Q[:4], k, v, ke, ve, table, cu, lens, 0.1, True), d)


@pytest.mark.parametrize("d", [64, 128])
def test_training_with_rotated_queries_and_keys(api, d):
    """Gradients through rotation, attention and back: the library's chain against float64 autograd of the plain formulas."""
    torch.manual_seed(d)
    B, H, N = 2, 2, 200
    Q, K, V, dO = (torch.randn(B, H, N, d, device="cuda").to(torch.bfloat16) for _ in range(4))
    table, a = api.flat_attn_rope_table(d, scaling=api.FLAT_ROPE_PARTS, factor=2.0, original_len=128)
    Qr, Kr = torch.empty_like(Q), torch.empty_like(K)
    scale = d ** -0.5
    api.flat_attn_rope_fwd(Q, K, table, Qr, Kr, amplitude=a)
    O, lse, delta = torch.empty_like(Q), torch.empty(B, H, N, device="cuda"), torch.empty(B, H, N, device="cuda")
    api.flat_attn_fwd_ex(Qr, Kr, V, O, scale, causal=True, lse=lse)
    dQr, dKr, dV = (torch.empty_like(Q) for _ in range(3))
    api.flat_attn_bwd_ex(Qr, Kr, V, O, dO, lse, dQr, dKr, dV, delta, scale, causal=True)
    dQ, dK = torch.empty_like(Q), torch.empty_like(K)
    api.flat_attn_rope_bwd(dQr, dKr, table, dQ, dK, amplitude=a)
    torch.cuda.synchronize()
    f = torch.tensor([10000.0 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
    keep = ((128 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    t = torch.arange(N, device="cuda", dtype=torch.float64)[:, None] * ((1 - keep) * f / 2 + keep * f)
    c, s = a * torch.cos(t), a * torch.sin(t)

    def rotate(x):
        one, two = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([one * c - two * s, two * c + one * s], -1)
    q, k, v = (x.double().requires_grad_() for x in (Q, K, V))
    logits = rotate(q) @ rotate(k).transpose(-1, -2) * scale
    logits = logits.masked_fill(torch.ones(N, N, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    (torch.softmax(logits, -1) @ v).backward(dO.double())
    # (bounds of the library's backward pass, tests/test_gpu_bwd.py: 2e-2 of the largest gradient)
    for got, want in ((dQ, q.grad), (dK, k.grad), (dV, v.grad)):
        assert float((got.double() - want).abs().max()) <= 2e-2 * float(want.abs().max())
