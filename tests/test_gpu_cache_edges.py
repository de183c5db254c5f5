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
