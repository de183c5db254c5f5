"""What rotary positions, the 8-bit paged cache and its attention refuse, before the device is touched (no GPU needed)."""
import ctypes
import math
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def api():
    from paper_2107_06419_b200 import build
    build.build()
    from paper_2107_06419_b200 import api as _api
    return _api


def filled(struct, **kw):
    for k, v in kw.items():
        setattr(struct, k, (ctypes.c_longlong * 3)(*v) if isinstance(v, tuple) else v)
    return struct


def rope(api, **kw):
    a = dict(Q=0x10000, K=0x20000, Qr=0x30000, Kr=0x40000, B=2, N=10, Hq=4, Hk=2, d=64, q_stride=(2560, 640, 64), k_stride=(1280, 640, 64),
             qr_stride=(2560, 640, 64), kr_stride=(1280, 640, 64), positions=0x50000, positions_stride_b=10, table=0x60000, rotary_dim=64,
             interleaved=0, amplitude=1.0, dtype=0)
    a.update(kw)
    return filled(api.flat_attn_rope_params_t(), **a)


@pytest.mark.parametrize("kw,code", [
    (dict(Q=None), 1), (dict(Qr=None), 1), (dict(table=None), 1), (dict(Kr=None), 1), (dict(K=None), 1),
    (dict(B=0), 2), (dict(N=-1), 2), (dict(Hq=0), 2), (dict(Hk=0), 2), (dict(B=65536), 2), (dict(B=65535, N=2 ** 30), 2), (dict(Hq=65535), 2),
    (dict(amplitude=math.nan), 2), (dict(amplitude=math.inf), 2),
    (dict(q_stride=(2560, 640, 60)), 2), (dict(q_stride=(-2560, 640, 64)), 2), (dict(positions_stride_b=-1), 2),
    (dict(qr_stride=(2560, 640, 0)), 2), (dict(qr_stride=(2560, 0, 64)), 2), (dict(kr_stride=(0, 640, 64)), 2), (dict(qr_stride=(2560, 632, 64)), 2),
    (dict(qr_stride=(64, 640, 64)), 2), (dict(qr_stride=(2560, 640, 56)), 2),
    (dict(d=48), 3), (dict(d=256), 3), (dict(rotary_dim=0), 3), (dict(rotary_dim=66), 3), (dict(rotary_dim=33), 3), (dict(interleaved=2), 3), (dict(dtype=2), 3),
    (dict(Q=0x10008), 4), (dict(Kr=0x40004), 4), (dict(positions=0x50002), 4), (dict(table=0x60004), 4)])
def test_rope(api, kw, code):
    p = rope(api, **kw)
    for call in (api._lib.flat_attn_rope_fwd, api._lib.flat_attn_rope_bwd):
        assert call(ctypes.byref(p), None) == code
        assert call(None, None) == 1


def test_rope_table(api):
    for kw, code in ((dict(rotary_dim=0), 3), (dict(rotary_dim=130), 3), (dict(rotary_dim=7), 3), (dict(scaling=4), 3), (dict(scaling=-1), 3),
                     (dict(base=1.0), 2), (dict(base=math.nan), 2), (dict(base=1e31), 2), (dict(factor=0.5), 2), (dict(factor=math.inf), 2),
                     (dict(scaling=3), 2), (dict(scaling=3, original_len=64, low=2.0, high=2.0), 2), (dict(scaling=3, original_len=64, low=-1.0), 2),
                     (dict(scaling=3, original_len=64, high=math.inf), 2)):
        with pytest.raises(api.FlatAttnError) as e:
            api.flat_attn_rope_table(**{"rotary_dim": 64, "device": "cpu", **kw})
        assert e.value.code == code, kw
    assert api._lib.flat_attn_rope_table(64, 1e4, 0, 1.0, 0, 1.0, 32.0, None, None) == 1


@pytest.mark.parametrize("r", [2, 6, 64, 128])
def test_rope_frequencies(api, r):
    """Every frequency within its 2^-64 turns and the rounding of the float64 it is compared with."""
    for scaling, factor, original in ((0, 1.0, 0), (1, 8.0, 0), (2, 8.0, 0), (3, 8.0, 4096)):
        table, a = api.flat_attn_rope_table(r, 10000.0, scaling, factor, original, device="cpu")
        base = 10000.0 * factor ** (r / (r - 2)) if scaling == 2 and r > 2 else 10000.0
        assert a == pytest.approx(0.1 * math.log(factor) + 1 if scaling == 3 else 1.0, rel=1e-6)
        for i, word in enumerate(table.tolist()):
            f = base ** (-2 * i / r)
            if scaling == 1:
                f /= factor
            if scaling == 3:
                keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - 1) / 31))
                f = (1 - keep) * f / factor + keep * f
            assert (word % 2 ** 64) * 2.0 ** -64 == pytest.approx(f / (2 * math.pi), rel=1e-13)


def cache(api, **kw):
    a = dict(k_cache=0x100000, v_cache=0x200000, k_exp=0x300001, v_exp=0x400001, page_table=0x500000, cu_seqlens=0x600000, seq_lens=0x700000,
             num_pages=100, Hkv=2, page=64, d=128, num_seqs=3, max_pages=10, status=None)
    a.update(kw)
    return filled(api.flat_attn_cache_t(), **a)


BAD_CACHES = [(dict(k_cache=None), 1), (dict(v_exp=None), 1), (dict(page_table=None), 1), (dict(cu_seqlens=None), 1), (dict(seq_lens=None), 1),
              (dict(num_pages=0), 2), (dict(Hkv=0), 2), (dict(num_seqs=0), 2), (dict(max_pages=0), 2), (dict(max_pages=2 ** 25), 2), (dict(Hkv=65536), 2),
              (dict(page=8), 3), (dict(page=48), 3), (dict(page=256), 3), (dict(d=32), 3), (dict(d=256), 3),
              (dict(k_cache=0x100008), 4), (dict(page_table=0x500002), 4), (dict(seq_lens=0x700001), 4), (dict(status=0x800002), 4)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches(api, kw, code):
    c = cache(api, **kw)
    assert api._lib.flat_attn_cache_append(ctypes.byref(c), 0x900000, 0xa00000, 30, 256, 128, 256, 128, 10, None) == code
    p = attention(api)
    assert api._lib.flat_attn_cache_fwd(ctypes.byref(c), ctypes.byref(p), None) == code


def test_append(api):
    def call(K=0x900000, V=0xa00000, total=30, kt=256, kh=128, vt=256, vh=128, most=10, c=cache(api)):
        return api._lib.flat_attn_cache_append(c if c is None else ctypes.byref(c), K, V, total, kt, kh, vt, vh, most, None)
    assert call(K=None) == 1 and call(V=None) == 1 and call(c=None) == 1
    assert call(total=0) == 2 and call(most=0) == 2 and call(most=31) == 2 and call(total=2 ** 31) == 2 and call(kt=250) == 2 and call(vh=-8) == 2
    assert call(K=0x900008) == 4


def attention(api, **kw):
    a = dict(Q=0x900000, O=0xa00000, Hq=8, total=30, q_stride_t=1024, q_stride_h=128, o_stride_t=1024, o_stride_h=128, max_new=10, causal=1,
             scale=0.1, lse=None, workspace=0xb00000, workspace_bytes=1 << 40)
    a.update(kw)
    return filled(api.flat_attn_cache_fwd_params_t(), **a)


@pytest.mark.parametrize("kw,code", [
    (dict(Q=None), 1), (dict(O=None), 1), (dict(workspace=None), 1),
    (dict(Hq=0), 2), (dict(total=0), 2), (dict(max_new=0), 2), (dict(max_new=31), 2), (dict(scale=math.nan), 2), (dict(total=2 ** 29), 2),
    (dict(q_stride_t=1020), 2), (dict(o_stride_h=0), 2), (dict(o_stride_t=0), 2), (dict(o_stride_t=1016), 2), (dict(q_stride_h=-8), 2),
    (dict(Hq=7), 3), (dict(Hq=2 * 129), 3), (dict(causal=2), 3),
    (dict(Q=0x900004), 4), (dict(O=0xa00008), 4), (dict(workspace=0xb00010), 4), (dict(lse=0xc00002), 4),
    (dict(workspace_bytes=1000), 5)])
def test_attention(api, kw, code):
    if "total" in kw and kw["total"] > 1000:
        kw = dict(kw, max_new=10)
    c, p = cache(api), attention(api, **kw)
    assert api._lib.flat_attn_cache_fwd(ctypes.byref(c), ctypes.byref(p), None) == code
    assert api._lib.flat_attn_cache_fwd(ctypes.byref(c), None, None) == 1 and api._lib.flat_attn_cache_fwd(None, ctypes.byref(p), None) in (1, code)


def test_workspace_bytes(api):
    assert api.flat_attn_cache_workspace_bytes(8, 3, 128) == 0 and api.flat_attn_cache_workspace_bytes(0, 1, 64) == 0
    assert api.flat_attn_cache_workspace_bytes(8, 2, 96) == 0
    assert api.flat_attn_cache_workspace_bytes(8, 2, 128) > api.flat_attn_cache_workspace_bytes(8, 2, 64) > 0


def test_shapes_and_types(api):
    """What the long way says about tensors that do not fit (it looks at them before it asks where they are)."""
    import torch
    bf = torch.bfloat16
    q, table = torch.zeros(1, 2, 4, 64, dtype=bf), torch.zeros(32, dtype=torch.int64)
    ok = dict(Q=q, K=q, table=table, Qr=q, Kr=q)
    for bad, error in ((dict(Q=q.half()), TypeError), (dict(Q=q[0, 0]), ValueError), (dict(Kr=None), ValueError), (dict(Qr=q[:, :1]), ValueError),
                       (dict(K=q.float()), ValueError), (dict(K=q.transpose(2, 3)), ValueError), (dict(table=table.int()), ValueError),
                       (dict(positions=torch.zeros(3, dtype=torch.int32)), ValueError), (dict(positions=torch.zeros(4)), ValueError), ({}, ValueError)):
        with pytest.raises(error):
            api.flat_attn_rope_fwd(**{**ok, **bad})
    k = torch.zeros(5, 2, 16, 64, dtype=torch.float8_e4m3fn)
    e, t = torch.zeros(5, 2, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.int32)
    x, w = torch.zeros(3, 2, 64, dtype=bf), torch.zeros(8, dtype=torch.uint8)
    cu, lens = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    ok = dict(k_cache=k, v_cache=k, k_exp=e, v_exp=e, page_table=t, cu_seqlens=cu, seq_lens=lens)
    for bad in (dict(v_cache=k[:4]), dict(k_cache=k.view(torch.uint8)), dict(k_exp=e.int()), dict(page_table=t[:2]), dict(page_table=t.t()), dict(cu_seqlens=lens),
                dict(seq_lens=lens.long()), {}):
        with pytest.raises(ValueError):
            api.flat_attn_cache_append(x, x, **{**ok, **bad}, max_new=1)
        with pytest.raises(ValueError):
            api.flat_attn_cache_fwd(x, x, **{**ok, **bad}, max_seqlen_q=1, scale=1.0, workspace=w)


PROGRAM = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2107_06419_b200 import api
torch.cuda.current_device = lambda: %d
bf = torch.bfloat16
def t(*shape, dtype=bf):
    return torch.empty(2, *shape, device="cuda", dtype=dtype)
i = torch.int32
cache = [lambda: t(5, 2, 16, 64, dtype=torch.float8_e4m3fn)] * 2 + [lambda: t(5, 2, dtype=torch.uint8)] * 2 + [lambda: t(3, 4, dtype=i), lambda: t(4, dtype=i), lambda: t(3, dtype=i)]
calls = {
    "rope": (lambda q, w, r: api.flat_attn_rope_fwd(q, None, w, r, None), [lambda: t(1, 2, 4, 64), lambda: t(32, dtype=torch.int64), lambda: t(1, 2, 4, 64)]),
    "append": (lambda k, v, *c: api.flat_attn_cache_append(k, v, *c, 1), [lambda: t(3, 2, 64)] * 2 + cache),
    "attention": (lambda q, o, w, *c: api.flat_attn_cache_fwd(q, o, *c, 1, 1.0, w), [lambda: t(3, 4, 64)] * 2 + [lambda: t(9, dtype=torch.uint8)] + cache),
}
call, make = calls[%r]
with FakeTensorMode():
    try:
        torch.vmap(call)(*(m() for m in make))
    except (RuntimeError, ValueError) as e:
        print("raised", "data pointer" in str(e), "current device" in str(e))
"""


@pytest.mark.parametrize("name", ["rope", "append", "attention"])
@pytest.mark.parametrize("device", [0, 1])
def test_tensors_without_memory_and_of_another_device(name, device):
    """Torch's error for tensors that have no memory, and a refusal of those of a device that is not the current one."""
    r = subprocess.run([sys.executable, "-c", PROGRAM % (device, name)], cwd=ROOT, capture_output=True, text=True, env={**os.environ, "PYTHONPATH": ROOT})
    assert r.returncode == 0 and r.stdout.split() == ["raised", str(device == 0), str(device == 1)], r.stdout + r.stderr[-2000:]
