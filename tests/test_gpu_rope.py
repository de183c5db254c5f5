"""Rotary positions and their gradient, against a plain float64 form and against differences."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2107_06419_b200 import api as _api
    return _api


def frequencies(r, base=10000.0, scaling=0, factor=1.0, original=0, low=1.0, high=32.0):
    b = base * factor ** (r / (r - 2)) if scaling == 2 and r > 2 else base
    f = torch.tensor([b ** (-2 * i / r) for i in range(r // 2)], dtype=torch.float64)
    if scaling == 1:
        f = f / factor
    if scaling == 3:
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = (1 - keep) * f / factor + keep * f
    return f, 0.1 * math.log(factor) + 1 if scaling == 3 else 1.0


def rotated(x, f, a, positions, interleaved, back=False):
    """x [..., N, d] float64, positions [..., N]."""
    r = 2 * f.numel()
    t = positions.double()[..., None] * f.to(x.device)
    c, s = a * torch.cos(t), a * torch.sin(t) * (-1 if back else 1)
    y = x.clone()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    return y


def check(got, x, f, a, positions, interleaved, back=False):
    """Half a step of the result's type, and 2^-21 of a (|x1| + |x2|): cosine, sine (2 ulp), angle (2.6e-8), amplitude, two products, a sum."""
    want = rotated(x.double(), f, a, positions, interleaved, back)
    r = 2 * f.numel()
    size = x.double().abs()
    mate = size.clone()
    if interleaved:
        mate[..., 0:r:2], mate[..., 1:r:2] = size[..., 1:r:2], size[..., 0:r:2]
    else:
        mate[..., :r // 2], mate[..., r // 2:r] = size[..., r // 2:r], size[..., :r // 2]
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + 2.0 ** -21 * a * (size + mate)
    assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() / tol.clamp_min(1e-30)).max())
    assert torch.equal(got[..., r:], x[..., r:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(16, 16), (16, 6), (32, 2), (32, 32), (64, 32), (64, 22), (64, 64), (128, 128), (128, 64), (128, 96), (128, 126), (128, 16)])
@pytest.mark.parametrize("B,N,Hq,Hk", [(2, 37, 3, 1), (1, 1, 1, 1), (1, 700, 4, 4)])
@pytest.mark.parametrize("back", [False, True])
def test_dense(api, dtype, interleaved, d, r, B, N, Hq, Hk, back):
    gen = torch.Generator(device="cuda").manual_seed(d + r + N)
    table, a = api.flat_attn_rope_table(r, scaling=api.FLAT_ROPE_PARTS, factor=4.0, original_len=512)
    f, a2 = frequencies(r, scaling=3, factor=4.0, original=512)
    assert abs(a - a2) < 1e-6
    Q = torch.randn(B, Hq, N, d, device="cuda", generator=gen).to(dtype)
    K = torch.randn(B, Hk, N, d, device="cuda", generator=gen).to(dtype)
    pos = torch.randint(-5, 1 << 20, (B, N), device="cuda", generator=gen, dtype=torch.int32)
    call = api.flat_attn_rope_bwd if back else api.flat_attn_rope_fwd
    Qr, Kr = torch.full_like(Q, 9), torch.full_like(K, 9)
    call(Q, K, table, Qr, Kr, positions=pos, interleaved=interleaved, amplitude=a)
    torch.cuda.synchronize()
    check(Qr, Q, f, a, pos[:, None], interleaved, back)
    check(Kr, K, f, a, pos[:, None], interleaved, back)
    X, Y = Q.clone(), K.clone()                          # in place
    call(X, Y, table, X, Y, positions=pos, interleaved=interleaved, amplitude=a)
    torch.cuda.synchronize()
    assert torch.equal(X, Qr) and torch.equal(Y, Kr)


@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
@pytest.mark.parametrize("r", [2, 20, 64])
def test_scalings_and_far_positions(api, scaling, r):
    gen = torch.Generator(device="cuda").manual_seed(r)
    table, a = api.flat_attn_rope_table(r, 500000.0, scaling, 8.0, 8192, 1.0, 4.0)
    f, _ = frequencies(r, 500000.0, scaling, 8.0, 8192, 1.0, 4.0)
    Q = torch.randn(1, 2, 9, 64, device="cuda", generator=gen)
    pos = torch.tensor([0, 1, -1, 4095, 131071, 1048576, 1 << 30, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    Qr = torch.empty_like(Q)
    assert api.flat_attn_rope_fwd(Q, None, table, Qr, None, positions=pos, amplitude=a) is Qr
    torch.cuda.synchronize()
    # (beyond 2^20 the float64 form itself is off by |t| 2^-53: still below 1e-6)
    check(Qr, Q, f, a, pos, False)


def test_packed_slices_and_default_positions(api):
    gen = torch.Generator(device="cuda").manual_seed(2)
    T, Hq, Hk, d = 77, 6, 2, 64
    table, a = api.flat_attn_rope_table(64)
    f, _ = frequencies(64)
    fused = torch.randn(T, (Hq + 2 * Hk) * d, device="cuda", generator=gen).to(torch.bfloat16)
    kept = fused.clone()
    Q, K = fused[:, :Hq * d].view(T, Hq, d), fused[:, Hq * d:(Hq + Hk) * d].view(T, Hk, d)
    Qr = torch.empty(1, Hq, T, d, dtype=torch.bfloat16, device="cuda")[0].transpose(0, 1)
    api.flat_attn_rope_fwd(Q, K, table, Qr, K)           # keys in place, inside the fused tensor
    torch.cuda.synchronize()
    at = torch.arange(T, device="cuda")
    check(Qr.transpose(0, 1), kept[:, :Hq * d].view(T, Hq, d).transpose(0, 1), f, a, at, False)
    check(K.transpose(0, 1), kept[:, Hq * d:(Hq + Hk) * d].view(T, Hk, d).transpose(0, 1), f, a, at, False)
    assert torch.equal(fused[:, :Hq * d], kept[:, :Hq * d]) and torch.equal(fused[:, (Hq + Hk) * d:], kept[:, (Hq + Hk) * d:])


def test_broadcast_input(api):
    """One key head seen as many (stride 0): read so, written to each; as an output it is refused."""
    table, _ = api.flat_attn_rope_table(64)
    x = torch.randn(2, 1, 50, 64, device="cuda").expand(2, 4, 50, 64)
    y = torch.empty(2, 4, 50, 64, device="cuda")
    api.flat_attn_rope_fwd(x, None, table, y, None)
    torch.cuda.synchronize()
    check(y, x, frequencies(64)[0], 1.0, torch.arange(50, device="cuda"), False)
    with pytest.raises(api.FlatAttnError) as e:
        api.flat_attn_rope_fwd(y, None, table, x, None)
    assert e.value.code == 2


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(api, interleaved):
    """Along a direction u the loss <g, rope(x)> changes by <rope_bwd(g), u>: the map is linear, so one difference is exact up to rounding."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    table, a = api.flat_attn_rope_table(32, scaling=api.FLAT_ROPE_PARTS, factor=8.0, original_len=64)
    x, u, g = (torch.randn(2, 3, 65, 64, device="cuda", generator=gen) for _ in range(3))
    y0, y1, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    kw = {"interleaved": interleaved, "amplitude": a}
    api.flat_attn_rope_fwd(x, None, table, y0, None, **kw)
    api.flat_attn_rope_fwd(x + u, None, table, y1, None, **kw)
    api.flat_attn_rope_bwd(g, None, table, dx, None, **kw)
    torch.cuda.synchronize()
    left = (g.double() * (y1.double() - y0.double())).sum()
    right = (dx.double() * u.double()).sum()
    # every term off by a few 2^-24 of its factors: 25,000 terms of size 1 add like a random walk, far below their worst sum
    size = (g.double().abs() * (y1.double().abs() + y0.double().abs()) + dx.double().abs() * u.double().abs()).sum()
    assert abs(float(left - right)) <= 2.0 ** -21 * float(size)


def test_relative_positions(api):
    """What it is for: a logit depends on the distance of its tokens."""
    table, _ = api.flat_attn_rope_table(64)
    q, k = (torch.randn(1, 1, 1, 64, device="cuda").expand(1, 1, 6, 64).contiguous() for _ in range(2))
    at = torch.tensor([0, 7, 100, 5000, 100000, 1000000], dtype=torch.int32, device="cuda")
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    api.flat_attn_rope_fwd(q, None, table, qr, None, positions=at + 11)
    api.flat_attn_rope_fwd(k, None, table, kr, None, positions=at)
    torch.cuda.synchronize()
    dots = (qr.double() * kr.double()).sum(-1).flatten()
    bound = 2.0 ** -20 * float((q.double().norm() * k.double().norm()) / 6)     # (each of six rows: |q| |k|; two roundings of 2^-21)
    assert float((dots - dots[0]).abs().max()) <= 4 * bound


def test_more_than_2_31_elements(api):
    N, H, d = 70000, 256, 128
    x = torch.empty(1, H, N, d, dtype=torch.bfloat16, device="cuda").uniform_(-1, 1)
    table, a = api.flat_attn_rope_table(d)
    f, _ = frequencies(d)
    y = torch.empty_like(x)
    api.flat_attn_rope_fwd(x, None, table, y, None)
    torch.cuda.synchronize()
    at = torch.tensor([0, 5, 33333, N - 1], device="cuda")
    for h in (0, 100, H - 1):
        check(y[0, h, at], x[0, h, at], f, a, at, False)


def test_other_stream_and_graph(api):
    table, _ = api.flat_attn_rope_table(128)
    Q, K = torch.randn(2, 4, 300, 128, device="cuda").to(torch.bfloat16), torch.randn(2, 2, 300, 128, device="cuda").to(torch.bfloat16)
    out = [torch.empty_like(Q) for _ in range(3)], [torch.empty_like(K) for _ in range(3)]
    api.flat_attn_rope_fwd(Q, K, table, out[0][0], out[1][0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    api.flat_attn_rope_fwd(Q, K, table, out[0][1], out[1][1], stream=side)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        api.flat_attn_rope_fwd(Q, K, table, out[0][2], out[1][2])
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(side_[0], side_[i]) for side_ in out for i in (1, 2))
