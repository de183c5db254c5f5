"""The 8-bit paged cache where calls meet (one workspace, many sequences) and where its values are at the ends of their range."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2107_06419_b200 import api as _api
    return _api


@pytest.fixture(scope="module")
def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def workspace(api, Hq, Hkv, d):
    return torch.zeros(api.flat_attn_cache_workspace_bytes(Hq, Hkv, d), dtype=torch.uint8, device="cuda")


def check_call(api, gen, w, new, lens, G, Hkv, page, d, times=1):
    """Causal attention with the workspace `w`, against the plain form."""
    cu = ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    Q = torch.randn(cu[-1], G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    want = ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(times):
        O, lse = torch.full_like(Q, 7.0), torch.full((cu[-1], G * Hkv), 7.0, device="cuda")
        api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), max(new), 0.1, w, causal=True, lse=lse, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        ref.check_attention(O, lse, want, d)


def test_one_workspace_for_both_head_sizes(api, sms):
    """A workspace of the larger size serves calls of either, one after the other: single tokens of d = 128 whose items are dealt to single
    warps and split (their parts fill the workspace), prompts of d = 64 split along the keys, and the other way round."""
    gen = torch.Generator().manual_seed(21)
    w = workspace(api, 8, 8, 128)
    seqs = -(-12 * sms // 8) + 10
    lens = [100 + 37 * s % 160 for s in range(seqs)]
    for _ in range(2):
        check_call(api, gen, w, [1] * seqs, lens, 1, 8, 64, 128)
        check_call(api, gen, w, [128, 100], [4096, 700], 1, 8, 64, 64, times=2)
        check_call(api, gen, w, [140], [3000], 2, 2, 32, 128, times=2)
        check_call(api, gen, w, [1] * seqs, lens, 1, 8, 16, 64)
    assert int(w[:20 * 4 * sms].sum()) == 0              # the counters of both kernels are at its beginning, and 0 again


# ---------------------------------------------------------------- entries that are not numbers

def attend_with_nan(api, gen, new, lens, G, page, d, causal):
    """NaN among the keys and values of four heads; a row is NaN where it sees a NaN key, a feature of it where it sees a NaN value, and
    nothing else is (0: values of new tokens, 1: a key of a new token, 2: keys of cached tokens, one in eight, 3: values of the
    first and last tokens)."""
    Hkv, cu = 4, ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    clean = [k.clone(), v.clone()]
    T = cu[-1]
    rows, cells = torch.zeros(T, G * Hkv, dtype=torch.bool), torch.zeros(T, G * Hkv, d, dtype=torch.bool)
    for s, (n, m) in enumerate(zip(new, lens)):
        at = m - n
        marks = [(1, h, j, f) for h, j, f in [(0, at, 3), (0, at + n // 2, d - 1), (0, m - 1, 0), (3, min(5, m - 1), 17), (3, m - 1, 40)]]
        marks += [(0, 1, at + (n - 1) // 2, 9)] + [(0, 2, j, (7 * j) % d) for j in range(67, at, 8 * (1 + at // 100))]
        for which, h, j, f in marks:
            p, r = int(table[s, j // page]), j % page
            (k, v)[which].view(torch.uint8)[p, h, r, f] = 0xFF if (j + f) % 2 else 0x7F
            clean[which].view(torch.uint8)[p, h, r, f] = 0
            first = cu[s] + (max(0, j - at) if causal else 0)              # the first row that sees key j
            for g in range(h * G, (h + 1) * G):
                if which:
                    cells[first:cu[s + 1], g, f] = True
                else:
                    rows[first:cu[s + 1], g] = True
    rows, cells = rows.cuda(), (cells | rows[..., None]).cuda()
    Q = torch.randn(T, G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    O, lse = torch.full_like(Q, 7.0), torch.full((T, G * Hkv), 7.0, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), max(new), 0.1, workspace(api, G * Hkv, Hkv, d), causal=causal, lse=lse)
    torch.cuda.synchronize()
    R, L, A, B = ref.attention(Q, *clean, ke, ve, table, cu, lens, 0.1, causal)
    assert torch.equal(torch.isnan(O), cells), (int((torch.isnan(O) & ~cells).sum()), int((cells & ~torch.isnan(O)).sum()))
    assert torch.equal(torch.isnan(lse), rows)
    ref.check_attention(torch.where(cells, R, O.double()), torch.where(rows, L, lse.double()), (R, L, A, B), d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("G,new,lens", [(2, [4, 3, 1], [300, 77, 1000]), (7, [5, 2], [1500, 40]), (1, [64], [64]), (8, [8, 1], [8, 500]), (1, [300], [1900]),
                                        (2, [200, 90], [400, 90]), (3, [150, 3, 1], [700, 200, 64])])
def test_nan_reaches_what_sees_it(api, d, page, causal, G, new, lens):
    attend_with_nan(api, torch.Generator().manual_seed(sum(lens) + G), new, lens, G, page, d, causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,G,n", [(16, 2, 4), (64, 4, 4)])
def test_nan_where_items_are_dealt_to_single_warps(api, sms, d, page, G, n):
    seqs = -(-12 * sms // 4)
    lens = [n + 53 * s % 300 for s in range(seqs)]
    attend_with_nan(api, torch.Generator().manual_seed(22), [n] * seqs, lens, G, page, d, True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,new,lens", [(4, [1, 1], [300, 40]), (2, [4, 1], [500, 77]), (2, [150, 90], [1500, 90])])
def test_queries_that_are_not_finite(api, d, G, new, lens):
    """Rows with NaN or infinite features are NaN, but for those whose logits are all -inf: like rows that see nothing, they are 0 and lse
    -inf, as everywhere in the library.  The other rows are as without them."""
    gen, Hkv, page, cu = torch.Generator().manual_seed(30), 2, 32, ref.offsets(new)
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    Q = torch.randn(cu[-1], G * Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    R, L, A, B = ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True)
    nan, none = (torch.zeros(Q.shape[:2], dtype=torch.bool, device="cuda") for _ in range(2))
    for i, (row, head, value) in enumerate([(0, 1, math.nan), (cu[1], 0, math.inf), (cu[-1] - 1, G * Hkv - 1, -math.inf), (cu[1] // 2, G, math.nan)]):
        Q[row, head, 7 * i + 3] = value
        s = 0 if row < cu[1] else 1
        ids = [int(p) for p in table[s][:-(-lens[s] // page)]]
        keys = ref.values(k, ke, ids, lens[s], head // G)[:row - cu[s] + lens[s] - new[s] + 1]
        x = (Q[row, head].double() * keys).sum(1)
        (none if (x == -math.inf).all() else nan)[row, head] = True
    O, lse = torch.full_like(Q, 7.0), torch.full(Q.shape[:2], 7.0, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), max(new), 0.1, workspace(api, G * Hkv, Hkv, d), causal=True, lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(O[nan]).all() and torch.isnan(lse[nan]).all()
    assert (O[none] == 0).all() and (lse[none] == -math.inf).all()
    bad = nan | none
    ref.check_attention(torch.where(bad[..., None], R, O.double()), torch.where(bad, L, lse.double()), (R, L, A, B), d)


# ---------------------------------------------------------------- scales at the ends of the range

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 5, 200])
@pytest.mark.parametrize("keys,values,size", [((112, 124), (10, 22), 1.0), ((10, 14), (112, 124), 2.0 ** 111), ((112, 124), (225, 238), 1.0)])
def test_least_and_largest_scales(api, d, new, keys, values, size):
    """Values down to the least scale that an append writes (whose numbers bf16 still holds), keys too (under large queries)."""
    gen = torch.Generator().manual_seed(23)
    lens, cu, Hkv, G, page = [700, 20000], ref.offsets([new, new]), 2, 2, 32
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    ke.copy_(torch.randint(*keys, ke.shape, generator=gen).to(torch.uint8))
    ve.copy_(torch.randint(*values, ve.shape, generator=gen).to(torch.uint8))
    Q = (torch.randn(cu[-1], G * Hkv, d, generator=gen) * size).to(torch.bfloat16).cuda()
    O, lse = torch.empty_like(Q), torch.empty(cu[-1], G * Hkv, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints(cu), ints(lens), new, 0.1, workspace(api, G * Hkv, Hkv, d), causal=True, lse=lse)
    torch.cuda.synchronize()
    R, L, A, B = ref.attention(Q, k, v, ke, ve, table, cu, lens, 0.1, True)
    up = 2.0 ** (117 - (values[0] + values[1]) // 2)     # (a power of two: the bounds count relative to values of about 1)
    ref.check_attention(O.double() * up, lse, (R * up, L, A * up, B), d)


@pytest.mark.parametrize("new,longest", [(1, 1 << 26), (70, 1 << 24)])
def test_least_scale_over_many_keys(api, new, longest):
    """Values at the least scale, of a page that the table names again and again: weights add up to 2^35 and more, and the outputs are the page's."""
    d, page = 64, 16
    gen = torch.Generator().manual_seed(28)
    k, v, ke, ve, _ = ref.make_cache(gen, [page], 1, page, d, "cuda", spare=0, exps=(114, 116))
    ve.fill_(10)
    table = torch.zeros(1, longest // page, dtype=torch.int32, device="cuda")
    Q = torch.randn(new, 1, d, generator=gen).to(torch.bfloat16).cuda()
    O, lse = torch.empty_like(Q), torch.empty(new, 1, device="cuda")
    api.flat_attn_cache_fwd(Q, O, k, v, ke, ve, table, ints([0, new]), ints([longest]), new, 0.125, workspace(api, 1, 1, d), causal=False, lse=lse)
    torch.cuda.synchronize()
    R, L, A, B = ref.attention(Q, k, v, ke, ve, [[0]], [0, new], [page], 0.125, False)
    # (long sums: half a step, 2^-24, for each of the weights that a lane adds up and 2^-23 for each sixteen keys, at most 2^24 / 16 keys of
    # a part: one token, 2^26 keys in more than 64 parts of four warps, eight lanes a row each; 70 tokens, a thread a row and 64 keys at a time)
    keys = longest / (256 if new == 1 else 16)
    more = keys / (8 if new == 1 else 64) * 2.0 ** -24 + keys / 16 * 2.0 ** -23
    logits = d * 2.0 ** -24 * B
    err, up = (O.double() - R).abs(), 2.0 ** 117
    assert (err * up <= (2.0 ** -8 * R.abs() + (2.0 ** -10 + 2 * logits[..., None] + more) * A) * up).all(), float((err / A).max())
    assert ((lse.double() - (L + math.log(longest // page))).abs() <= logits + 2.0 ** -18 * (1 + 20) + more).all()


# ---------------------------------------------------------------- forms that only large batches take

@pytest.mark.parametrize("d,page,G,n", [(128, 64, 1, 1), (128, 16, 4, 1), (128, 16, 5, 3), (128, 128, 8, 4), (64, 64, 2, 1), (64, 128, 1, 2), (64, 32, 7, 4),
                                        (64, 128, 5, 2)])
def test_items_dealt_to_single_warps(api, sms, d, page, G, n):
    """At least twelve items an SM: shares that begin and end inside items, some of them longer than a share."""
    gen, Hkv = torch.Generator().manual_seed(24), 8
    seqs = -(-12 * sms // (Hkv * -(-n * G // 16))) + 3
    lens = [n + int(x) for x in torch.randint(0, 400, (seqs,), generator=gen)]
    lens[seqs // 2], lens[-1] = 5000, n
    check_call(api, gen, workspace(api, G * Hkv, Hkv, d), [n] * seqs, lens, G, Hkv, page, d, times=2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,most", [(40, 300), (100, 90)])
def test_prompts_of_many_sequences(api, d, seqs, most):
    """More sequences than a warp has lanes, prompts, single tokens and sequences without new tokens among them."""
    gen = torch.Generator().manual_seed(seqs)
    new = [int(x) for x in torch.randint(0, most, (seqs,), generator=gen)]
    new[3::7] = [1] * len(new[3::7])
    new[5::11] = [0] * len(new[5::11])
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 700, (seqs,), generator=gen))]
    lens[seqs // 2] += 6000
    check_call(api, gen, workspace(api, 6, 2, d), new, lens, 3, 2, 32, d, times=2)


# ---------------------------------------------------------------- appending

def check_append(api, gen, cu, lens, good, most, Hkv, page, d, T, code=0):
    """Appending with offsets `cu` of which only the sequences `good` are right, against the plain form, bit by bit."""
    k, v, ke, ve, table = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    K, V = (torch.randn(T, Hkv, d, generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    want = [t.clone() for t in (k, v, ke, ve)]
    for s in good:
        for x, c, e in ((K, want[0], want[2]), (V, want[1], want[3])):
            ref.append(x[cu[s]:cu[s + 1]].double(), c, e, table[s:s + 1].tolist(), [0, cu[s + 1] - cu[s]], [lens[s]])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.flat_attn_cache_append(K, V, k, v, ke, ve, table, ints(cu), ints(lens), most, status=status)
    torch.cuda.synchronize()
    assert int(status) == code
    for got, w in zip((k, v, ke, ve), want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (128, 128), (64, 32)])
def test_append_prompts_among_single_tokens(api, d, page):
    gen, S = torch.Generator().manual_seed(25), 140
    new = [1] * S
    new[17], new[90], new[139], new[5], new[60] = 1000, 333, 48, 0, 0
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 200, (S,), generator=gen))]
    check_append(api, gen, [c + 3 for c in ref.offsets(new)], lens, range(S), 1000, 2, page, d, sum(new) + 8)


def test_append_beside_sequences_that_do_not_fit(api):
    """Offsets that go back, more new tokens than announced or than the sequence is long: those sequences are left out, the others are not."""
    gen = torch.Generator().manual_seed(26)
    cu, lens = [0, 20, 19, 60, 90, 95, 300, 310, 330, 320], [40, 30, 50, 25, 20, 400, 15, 64, 9]
    #   new:       20, -1, 41, 30 > length, 5, 205 > most, 10, 20, -10
    check_append(api, gen, cu, lens, [0, 2, 4, 6, 7], 50, 2, 16, 64, 330, api.FLAT_CACHE_BAD_LENGTH)


def test_append_of_tokens_owned_twice(api):
    """Offsets that go back so far that the sequences own more tokens than there are: said, and nothing is written."""
    gen = torch.Generator().manual_seed(29)
    cu, lens = [0, 500] * 20, [500] * 39
    check_append(api, gen, cu, lens, [], 500, 1, 16, 64, 500, api.FLAT_CACHE_BAD_LENGTH)


def test_append_with_room_for_many_pages_of_many_heads(api):
    """As many pages and heads as a cache may have, few of them with new tokens: no number of possible places is refused."""
    gen = torch.Generator().manual_seed(27)
    Hkv, d, page, n, longest = 512, 64, 16, 21, 1 << 25
    k, v, ke, ve, _ = ref.make_cache(gen, [48], Hkv, page, d, "cuda", spare=0)
    table = torch.full((1, longest // page), 2, dtype=torch.int32, device="cuda")
    table[0, -2:] = ints([0, 1])
    x = torch.randn(1, Hkv, d, generator=gen).to(torch.bfloat16).cuda()
    want = [t.clone() for t in (k, v, ke, ve)]
    for i in range(2):                                   # (the last 21 of the 32 tokens of a sequence of two pages)
        ref.append(x.double().expand(n, Hkv, d), want[i], want[2 + i], [[0, 1]], [0, n], [32])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    many = x.expand(longest, Hkv, d)
    api.flat_attn_cache_append(many, many, k, v, ke, ve, table, ints([0, n]), ints([longest]), longest, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for got, w in zip((k, v, ke, ve), want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


# ---------------------------------------------------------------- one call after another

@pytest.mark.parametrize("d,page,Hkv,new,lens", [(128, 64, 4, [70, 1, 1, 30, 1] + [1] * 40, [2000, 9000, 40, 333, 5000] + [400 + 30 * i for i in range(40)]),
                                                 (64, 16, 2, [30, 1, 1, 1], [60, 90, 40, 300])])
def test_inputs_that_change_from_call_to_call(api, d, page, Hkv, new, lens):
    """Rotation, append and a mixed batch's attention again and again on the same buffers, other tokens and lengths each time: without a wait in
    between, and in a graph, the bits are those of calls that are waited for."""
    gen, G, N = torch.Generator().manual_seed(31), 4, 6
    cu, T = ref.offsets(new), sum(new)
    cache = ref.make_cache(gen, lens, Hkv, page, d, "cuda")
    saved = [t.clone() for t in cache[:4]]
    tokens = [[(torch.randn(T, h, d, generator=gen) * 2.0 ** (i % s)).to(torch.bfloat16).cuda() for h, s in ((G * Hkv, 1), (Hkv, N), (Hkv, 3))] for i in range(N)]
    lengths = [ints(lens), ints([m - (m > n + 5) for n, m in zip(new, lens)])]
    rope, _ = api.flat_attn_rope_table(d)
    at, dcu, dlens, work = ints([m - n + i for n, m in zip(new, lens) for i in range(n)]), ints(cu), ints(lens), workspace(api, G * Hkv, Hkv, d)
    Q, K, outs = torch.empty_like(tokens[0][0]), torch.empty_like(tokens[0][1]), [torch.empty_like(tokens[0][0]) for _ in range(N)]

    def steps(wait):
        for i, (q, k, v) in enumerate(tokens):
            dlens.copy_(lengths[i % 2])
            api.flat_attn_rope_fwd(q, k, rope, Q, K, positions=at)
            wait()
            api.flat_attn_cache_append(K, v, *cache, dcu, dlens, max(new))
            wait()
            api.flat_attn_cache_fwd(Q, outs[i], *cache, dcu, dlens, max(new), 0.1, work, causal=True)
            wait()

    def again():
        for a, b in zip(cache, saved):
            a.view(torch.uint8).copy_(b.view(torch.uint8))
        for o in outs:
            o.zero_()
    steps(torch.cuda.synchronize)
    want = [o.clone() for o in outs]
    again()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(lambda: None)
    for run in [lambda: steps(lambda: None), graph.replay] * 20:
        again()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
