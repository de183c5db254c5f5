"""The 8-bit paged cache: appending to it and attention over it, against plain float64 forms."""
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


def workspace(api, Hq, Hkv, d):
    return torch.zeros(api.flat_attn_cache_workspace_bytes(Hq, Hkv, d), dtype=torch.uint8, device="cuda")


def attend(api, gen, new, lens, G, Hkv, page, d, causal=True, pad=0, scale=None, exps=(112, 124), what=""):
    cu = ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda", exps=exps)
    T = cu[-1] + pad
    Q = torch.randn(T, G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O = torch.full_like(Q, 7.0)
    lse = torch.full((T, G * Hkv), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = d ** -0.5 if scale is None else scale
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), max(max(new), 1), scale, workspace(api, G * Hkv, Hkv, d),
                            causal=causal, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert (O[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all()       # rows behind the last sequence
    want = ref.attention(Q[:cu[-1]], k, v, ke, ve, table, cu, lens, scale, causal)
    ref.check_attention(O[:cu[-1]], lse[:cu[-1]], want, d, what)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("G,Hkv", [(1, 3), (4, 2), (7, 1), (16, 1), (20, 1)])
def test_one_token(api, d, page, G, Hkv):
    gen = torch.Generator().manual_seed(d + page + G)
    lens = [1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 511, 700, 1025]
    attend(api, gen, [1] * len(lens), lens, G, Hkv, page, d, pad=2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("new,lens", [([2, 0, 5, 1], [2, 9, 300, 77]), ([4] * 5, [4, 5, 64, 130, 1000]), ([33, 1], [40, 260]),
                                      ([130, 0, 257], [130, 0, 400]), ([600], [611]), ([1, 300, 1, 1, 64], [500, 300, 7, 129, 640])])
@pytest.mark.parametrize("G,Hkv,page", [(1, 2, 16), (3, 2, 32), (8, 1, 64), (4, 2, 128)])
def test_several_tokens(api, d, causal, new, lens, G, Hkv, page):
    gen = torch.Generator().manual_seed(sum(lens) + G)
    attend(api, gen, new, lens, G, Hkv, page, d, causal=causal, pad=1)


@pytest.mark.parametrize("d,G,Hkv,page", [(128, 4, 8, 64), (64, 1, 16, 16), (128, 8, 1, 16), (64, 5, 2, 128)])
@pytest.mark.parametrize("seqs,longest", [(1, 20000), (3, 9000), (40, 1500), (200, 60)])
def test_long_and_many(api, d, G, Hkv, page, seqs, longest):
    gen = torch.Generator().manual_seed(seqs)
    lens = [1 + int(x) for x in torch.randint(0, longest, (seqs,), generator=gen)]
    lens[0] = longest
    attend(api, gen, [1] * seqs, lens, G, Hkv, page, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 5, 200])
def test_scales_far_apart(api, d, new):
    """Pages of all zeros with the least scale, pages 2^40 apart."""
    gen = torch.Generator().manual_seed(5)
    lens, cu, Hkv, G, page = [700, 300], ref.offsets([new, new]), 2, 2, 16
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    ve.copy_(torch.randint(90, 131, ve.shape, generator=gen).to(torch.uint8))
    ke.copy_(torch.randint(95, 121, ke.shape, generator=gen).to(torch.uint8))
    for p in table[0, :9:2].tolist():
        v.view(torch.uint8)[p] = 0
        ve[p] = 10
        k.view(torch.uint8)[p, 0] = 0
        ke[p, 0] = 10
    T = cu[-1]
    Q = torch.randn(T, G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    Q[0] = 0                                             # a row without a direction: all weights alike
    Q[T - 1] *= 2.0 ** -60
    Q[T // 2, 0] *= 2.0 ** 10
    O, lse = torch.empty_like(Q), torch.empty(T, G * Hkv, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), new, 0.1, workspace(api, G * Hkv, Hkv, d), causal=True, lse=lse)
    torch.cuda.synchronize()
    want = ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True)
    ref.check_attention(O, lse, want, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 150])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales_of_the_logits(api, d, new, scale):
    gen = torch.Generator().manual_seed(6)
    attend(api, gen, [new, new], [600, 301], 2, 2, 32, d, scale=scale, exps=(116, 121))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 6, 140])
def test_nan_behind_the_length_and_unused_pages(api, d, new):
    gen = torch.Generator().manual_seed(7)
    lens, Hkv, G, page = [new, 333, 160], 2, 4, 64
    cu = ref.offsets([new] * 3)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    used = torch.zeros(k.shape[0], page, dtype=torch.bool)
    for s, m in enumerate(lens):
        for j in range(m):
            used[int(table[s, j // page]), j % page] = True
    hidden = ~used[:, None, :, None].cuda().expand(k.shape)
    for c in (k, v):
        c.view(torch.uint8)[hidden] = 0x7F
    for e in (ke, ve):
        e[~used.any(1).cuda()] = 255
    Q = torch.randn(cu[-1], G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O = torch.empty_like(Q)
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), new, 0.1, workspace(api, G * Hkv, Hkv, d), causal=True)
    torch.cuda.synchronize()
    ref.check_attention(O, None, ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True), d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 140])
def test_bad_pages_and_lengths(api, d, new):
    """Page indexes out of range leave their tokens out, offsets and lengths that do not fit leave the sequence out; both are said."""
    gen = torch.Generator().manual_seed(8)
    lens, Hkv, G, page = [400, 333, 160, new], 1, 4, 32
    cu = ref.offsets([new] * 4)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    table[1, 2], table[1, 5], table[3, :] = k.shape[0], -1, 1 << 30
    Q = torch.randn(cu[-1], G, d, generator=gen).to(torch.bfloat16).cuda()
    O, lse = torch.empty_like(Q), torch.empty(cu[-1], G, device="cuda")
    status, w = torch.zeros(1, dtype=torch.int32, device="cuda"), workspace(api, G, Hkv, d)
    args = (k, v, ke, ve, table, ints(cu))
    api.flat_attn_cache_fwd(Q, O, *args, ints(lens), new, 0.1, w, causal=True, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == api.FLAT_CACHE_BAD_PAGE
    dropped = [(1, 2), (1, 5)] + [(3, p) for p in range(-(-new // page))]
    want = ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True, dropped)
    ref.check_attention(O, lse, want, d)
    assert (O[cu[3]:] == 0).all()
    table[1, 2], table[1, 5] = table[0, 0], table[0, 1]
    table[3, :] = table[0, 0]
    for bad in ([400, new - 1, 160, new], [400, 333, table.shape[1] * page + 1, new], [-5, 333, 160, new]):
        status.zero_()
        O.fill_(3.0)
        api.flat_attn_cache_fwd(Q, O, *args, ints(bad), new, 0.1, w, causal=True, status=status)
        torch.cuda.synchronize()
        assert int(status) == api.FLAT_CACHE_BAD_LENGTH
        out = [s for s in range(4) if bad[s] != lens[s]][0]
        assert (O[cu[out]:cu[out + 1]] == 3.0).all()
        rest = torch.cat([O[:cu[out]], O[cu[out + 1]:]])
        assert torch.isfinite(rest.float()).all() and (rest != 3.0).any()
    for bad in ([0, new, 2 * new, 3 * new, 4 * new + 1], [0, new, new - 1, 3 * new, 4 * new], [-1, new, 2 * new, 3 * new, 4 * new]):
        status.zero_()
        api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(bad), ints(lens), 2 * new + 2 if 2 * new + 2 <= 4 * new else 4 * new, 0.1, w, causal=True, status=status)
        torch.cuda.synchronize()
        assert int(status) == api.FLAT_CACHE_BAD_LENGTH
    assert int(w[:4096].sum()) == 0                      # the counters are left as they were found


@pytest.mark.parametrize("new", [1, 100])
def test_strided_queries_and_outputs(api, new):
    """Slices of a fused projection, and head-major tensors of the projections seen as tokens."""
    gen = torch.Generator().manual_seed(9)
    Hkv, G, d, page, lens = 2, 3, 64, 16, [300, 120, 1000]
    cu, T, Hq = ref.offsets([new] * 3), 3 * new, 6
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    fused = torch.randn(T, (Hq + 2 * Hkv) * d, generator=gen).to(torch.bfloat16).cuda()
    Q = fused[:, :Hq * d].view(T, Hq, d)
    heads = torch.zeros(1, Hq, T, d, dtype=torch.bfloat16, device="cuda")
    O = heads[0].transpose(0, 1)
    w = workspace(api, Hq, Hkv, d)
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), new, 0.125, w, causal=True)
    plain = torch.empty(T, Hq, d, dtype=torch.bfloat16, device="cuda")
    api.flat_attn_cache_fwd(Q.contiguous(), plain, k, v, ke, ve, table, ints(cu), ints(lens), new, 0.125, w, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(O, plain)
    ref.check_attention(O, None, ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.125, True), d)


@pytest.mark.parametrize("new", [1, 96])
def test_same_bits_again_on_other_streams_and_in_graphs(api, new):
    gen = torch.Generator().manual_seed(10)
    Hkv, G, d, page, lens = 2, 4, 128, 64, [5000, 130, 2222]
    cu, T, Hq = ref.offsets([new] * 3), 3 * new, 8
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    Q = torch.randn(T, Hq, d, generator=gen).to(torch.bfloat16).cuda()
    w, args = workspace(api, Hq, Hkv, d), (k, v, ke, ve, table, ints(cu), ints(lens), new, 0.1)
    first = torch.empty_like(Q)
    api.flat_attn_cache_fwd(Q, first, *args, w, causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other, w2 = torch.empty_like(Q), workspace(api, Hq, Hkv, d)
    torch.cuda.synchronize()
    here = torch.empty_like(Q)
    for _ in range(20):                                  # two calls at once, a workspace each
        with torch.cuda.stream(side):
            api.flat_attn_cache_fwd(Q, other, *args, w2, causal=True)
        api.flat_attn_cache_fwd(Q, here, *args, w, causal=True, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(first, other) and torch.equal(first, here)
    graphs, outs = [], []
    for _ in range(2):                                   # two graphs with one workspace, one after the other
        o = torch.empty_like(Q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.flat_attn_cache_fwd(Q, o, *args, w, causal=True)
        graphs.append(g)
        outs.append(o)
    for _ in range(3):
        for g, o in zip(graphs, outs):
            o.zero_()
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


def test_offsets_beyond_32_bits(api):
    """A cache of 5 GB: pages whose bytes lie behind 2^32."""
    gen = torch.Generator().manual_seed(11)
    Hkv, G, d, page = 8, 2, 128, 128
    pages = 40000
    k = torch.zeros(pages, Hkv, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(pages, Hkv, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ke = torch.full((pages, Hkv), 120, dtype=torch.uint8, device="cuda")
    ve = ke.clone()
    lens, new = [300, 200], [200, 1]
    table = torch.tensor([[pages - 1, 3, pages - 5], [pages - 2, 0, 0]], dtype=torch.int32, device="cuda")
    cu = ref.offsets(new)
    for p in (pages - 1, 3, pages - 5, pages - 2, 0):
        for c in (k, v):
            c[p] = (torch.randn(Hkv, page, d, generator=gen) * 50).to(torch.float8_e4m3fn).cuda()
    x = [torch.randn(cu[-1], Hkv, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    some = sorted({pages - 1, 3, pages - 5, pages - 2, 0})
    small = {p: i for i, p in enumerate(some)}
    want = [c[some].clone() for c in (k, v)] + [e[some].clone() for e in (ke, ve)]
    small_table = [[small[int(p)] for p in row] for row in table.tolist()]
    for i in range(2):
        ref.append(x[i].double(), want[i], want[2 + i], small_table, cu, lens)
    api.flat_attn_cache_append(x[0], x[1], k, v, ke, ve, table, ints(cu), ints(lens), 200)
    torch.cuda.synchronize()
    for got, c in zip((k, v, ke, ve), want):
        assert torch.equal(got[some].view(torch.uint8), c.view(torch.uint8))
    Q = torch.randn(cu[-1], G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O = torch.empty_like(Q)
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), 200, 0.1, workspace(api, G * Hkv, Hkv, d), causal=True)
    torch.cuda.synchronize()
    ref.check_attention(O, None, ref.attention(Q, *want, small_table, cu, lens, 0.1, True), d)


# ---------------------------------------------------------------- appending

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("new,lens", [([1, 1, 1, 1], [1, 16, 100, 129]), ([5, 0, 1], [5, 70, 131]), ([150, 17, 1, 300], [150, 33, 64, 777])])
def test_append(api, d, page, new, lens):
    gen = torch.Generator().manual_seed(page + d + sum(new))
    Hkv, cu = 3, ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda", exps=(114, 121))
    T = cu[-1] + 2
    x = torch.randn(T, Hkv, d, generator=gen)
    x *= torch.exp2(torch.randint(-6, 7, (T, Hkv, 1), generator=gen).float())
    K = x.to(torch.bfloat16).cuda()
    V = torch.zeros(T, 2 * Hkv * d, dtype=torch.bfloat16, device="cuda")[:, Hkv * d:].view(T, Hkv, d)
    V.copy_(x.flip(0))
    K[0, 0] = 0                                          # a head of zeros
    K[cu[-1] - 1, 1, 3], V[cu[-1] - 1, 2, 5], V[0, 1, 0] = math.inf, math.nan, -math.inf
    K[0, 2, :8] = torch.tensor([448, -448, 449, 464, 480, 2.0 ** -30, -2.0 ** -8, 1.75]).to(torch.bfloat16).cuda()
    want = [t.clone() for t in (k, v, ke, ve)]
    ref.append(K.double(), want[0], want[2], table.tolist(), cu, lens)
    ref.append(V.double(), want[1], want[3], table.tolist(), cu, lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(2):                                   # (a second time: the same tokens to the same places)
        api.flat_attn_cache_append(K, V, k, v, ke, ve, table, ints(cu), ints(lens), max(new), status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        assert torch.equal(ke, want[2]) and torch.equal(ve, want[3])
        for got, w in ((k, want[0]), (v, want[1])):
            nan = torch.isnan(w.float())
            assert torch.equal(torch.isnan(got.float()), nan)
            assert torch.equal(got.view(torch.uint8)[~nan], w.view(torch.uint8)[~nan])


def test_append_token_by_token(api):
    """A page filled one token at a time, its scale growing: what earlier tokens have become is what the definition says."""
    gen = torch.Generator().manual_seed(3)
    Hkv, page, d = 2, 64, 128
    k, v, ke, ve, table = ref.make_cache(gen, [page], Hkv, page, d, "cuda")
    want = [t.clone() for t in (k, v, ke, ve)]
    for m in range(1, page + 1):
        x = (torch.randn(1, Hkv, d, generator=gen) * 2.0 ** (m / 4)).to(torch.bfloat16).cuda()
        api.flat_attn_cache_append(x, x * 2, k, v, ke, ve, table, ints([0, 1]), ints([m]), 1)
        ref.append(x.double(), want[0], want[2], table.tolist(), [0, 1], [m])
        ref.append(x.double() * 2, want[1], want[3], table.tolist(), [0, 1], [m])
    torch.cuda.synchronize()
    for got, w in zip((k, v, ke, ve), want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


def test_append_bad_tables_and_captured(api):
    gen = torch.Generator().manual_seed(4)
    Hkv, page, d, lens, new = 2, 16, 64, [40, 30, 20], [20, 20, 20]
    cu = ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    K = torch.randn(60, Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    before = [t.clone() for t in (k, v, ke, ve)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t, c, m, code in ((torch.full_like(table, -1), cu, lens, api.FLAT_CACHE_BAD_PAGE), (torch.full_like(table, k.shape[0]), cu, lens, api.FLAT_CACHE_BAD_PAGE),
                          (table, cu, [19, 19, 10000], api.FLAT_CACHE_BAD_LENGTH), (table, [60, 40, 20, 0], lens, api.FLAT_CACHE_BAD_LENGTH),
                          (table, [0, 0, 0, 61], lens, api.FLAT_CACHE_BAD_LENGTH)):
        status.zero_()
        api.flat_attn_cache_append(K, K, k, v, ke, ve, t, ints(c), ints(m), 20, status=status)
        torch.cuda.synchronize()
        assert int(status) == code
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((k, v, ke, ve), before))
    ref.append(K.double(), before[0], before[2], table.tolist(), cu, lens)
    ref.append(K.double(), before[1], before[3], table.tolist(), cu, lens)
    dc, dm = ints(cu), ints(lens)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.flat_attn_cache_append(K, K, k, v, ke, ve, table, dc, dm, 20)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((k, v, ke, ve), before))


@pytest.mark.parametrize("most", [2 ** 32 + 1, 2 ** 31, 4, 0, -1, -2 ** 32 + 1])
def test_counts_out_of_range(api, most):
    """More new tokens a sequence than there are, or fewer than one, in 32 bits and beyond."""
    gen = torch.Generator().manual_seed(12)
    k, v, ke, ve, table = ref.make_cache(gen, [40], 2, 16, 64, "cuda")
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    args = (k, v, ke, ve, table, ints([0, 3]), ints([40]))
    for call in (lambda: api.flat_attn_cache_append(x, x, *args, most),
                 lambda: api.flat_attn_cache_fwd(x, torch.empty_like(x), *args, most, 0.1, workspace(api, 2, 2, 64))):
        with pytest.raises(api.FlatAttnError) as e:
            call()
        assert e.value.code == 2


@pytest.mark.parametrize("page", [16, 128])
def test_append_at_the_greatest_length(api, page):
    """A sequence of 2^30 tokens and room for as many new ones as a call may have (one token's memory, seen many times)."""
    d, longest, n = 64, 1 << 30, 5
    pages, total = longest // page, 2 ** 31 - 1
    gen = torch.Generator().manual_seed(13)
    k, v, ke, ve, _ = ref.make_cache(gen, [2 * page], 1, page, d, "cuda", spare=0)
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    x = torch.randn(1, 1, d, generator=gen).to(torch.bfloat16).cuda()
    many = x.expand(total, 1, d)
    want = [t.clone() for t in (k, v, ke, ve)]
    for i in range(2):                                   # (what the page holds at its end, as a sequence of one page)
        ref.append(x.double().expand(n, 1, d), want[i], want[2 + i], [[1]], [0, n], [page])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.flat_attn_cache_append(many, many, k, v, ke, ve, table, ints([0, n]), ints([longest]), total, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for got, w in zip((k, v, ke, ve), want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.parametrize("new,longest,least_parts", [(1, 1 << 30, 400), (70, 1 << 26, 16)])
def test_attention_over_one_page_many_times(api, new, longest, least_parts):
    """A very long sequence whose table names one page again and again: the output is that page's, the log-sum its own and log(times)."""
    d, page, sms = 64, 16, torch.cuda.get_device_properties(0).multi_processor_count
    gen = torch.Generator().manual_seed(14)
    k, v, ke, ve, _ = ref.make_cache(gen, [page], 1, page, d, "cuda", spare=0, exps=(114, 116))
    table = torch.zeros(1, longest // page, dtype=torch.int32, device="cuda")
    Q = torch.randn(new, 1, d, generator=gen).to(torch.bfloat16).cuda()
    O, lse = torch.empty_like(Q), torch.empty(new, 1, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints([0, new]), ints([longest]), new, 0.125, workspace(api, 1, 1, d), causal=False, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    R, L, A, B = ref.attention(Q, k, v, ke, ve, [[0]], [0, new], [page], 0.125, False)
    # Beside what check_attention counts, the roundings of long sums in fp32: a warp of a part adds up n weights a lane, half a step
    # (2^-24 of the sum) each, and its outputs sixteen keys at a time, where the product may cut off a whole step (2^-23).  Parts of at least
    # 1 / least_parts of the sequence; one token: four warps a part, an eighth of a warp's keys a lane; 70: a thread a row, 64 keys at a time.
    least_parts = min(least_parts, 2 * sms)
    keys = longest / least_parts / (4 if new == 1 else 1)
    weights, outputs = keys / (8 if new == 1 else 64) * 2.0 ** -24, keys / 16 * 2.0 ** -23
    logits = d * 2.0 ** -24 * B
    assert ((lse.double() - (L + math.log(longest // page))).abs() <= logits + 2.0 ** -18 * (1 + 20) + weights).all()
    assert ((O.double() - R).abs() <= 2.0 ** -8 * R.abs() + (2.0 ** -10 + 2 * logits[..., None] + weights + outputs) * A).all()
