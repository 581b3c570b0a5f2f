"""Rotary positions against 64-bit complex products.  A result is one rounding (u = eps / 2 of its value) of two fp32 products and
their sum, off by at most 2^-24 (|a| + |b|) each: bound u |y| + 2^-22 (|a| + |b|)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, cos, sin, pos, heads, d, interleaved, inverse):
    rows, half = x.shape[0], cos.shape[1]
    t = x.double().reshape(rows, heads, d)
    c, s = cos.double()[pos.long()][:, None], sin.double()[pos.long()][:, None] * (-1 if inverse else 1)
    y, mag = t.clone(), t.abs()
    ia = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    ib = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    a, b = t[..., ia], t[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
    return y.reshape(rows, -1), mag.reshape(rows, -1)


def check(y, ref, mag, dtype):
    u = torch.finfo(dtype).eps / 2
    assert ((y.double() - ref).abs() <= u * ref.abs() * 1.001 + 2.0 ** -22 * mag + 1e-38).all()


SHAPES = [(1, 1, 2, 2), (1, 4, 64, 64), (3, 1, 7, 2), (5, 3, 10, 6), (64, 8, 64, 64), (33, 5, 80, 48), (7, 2, 96, 96), (129, 3, 128, 32),
          (2, 40, 128, 128), (70, 1, 320, 318), (3, 2, 1030, 1030), (6000, 2, 24, 20)]


@pytest.mark.parametrize("rows,heads,d,rot", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (3, 1)])
def test_matches_the_definition(rows, heads, d, rot, dtype, interleaved, pad, offset):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    span = 300
    cos, sin = (torch.randn(span, rot // 2, generator=g, device="cuda") for _ in range(2))
    pos = torch.randint(0, span, (rows,), generator=g, device="cuda", dtype=torch.int32)
    w = heads * d
    wide = torch.randn(rows, w + pad, generator=g, device="cuda").to(dtype)
    x = wide[:, offset:offset + w]
    out = torch.full((rows, w + pad), 3.0, dtype=dtype, device="cuda")
    for inverse in (False, True):
        ref, mag = reference(x, cos, sin, pos, heads, d, interleaved, inverse)
        Bn.k_rotary(x, out[:, offset:offset + w], cos, sin, heads, d, positions=pos, interleaved=interleaved, inverse=inverse)
        check(out[:, offset:offset + w], ref, mag, dtype)
        rest = torch.ones(w + pad, dtype=torch.bool, device="cuda")
        rest[offset:offset + w] = False
        assert (out[:, rest] == 3).all()
        same = wide.clone()
        Bn.k_rotary(same[:, offset:offset + w], same[:, offset:offset + w], cos, sin, heads, d, positions=pos, interleaved=interleaved, inverse=inverse)
        assert torch.equal(same[:, offset:offset + w], out[:, offset:offset + w])  # in place, the same bits
        assert torch.equal(same[:, rest], wide[:, rest])


def test_rows_are_their_own_positions_and_the_inverse_is_the_gradient():
    from paper_2609_13645_b200 import binding as Bn
    rows, heads, d = 257, 6, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(rows, heads * d, generator=g, device="cuda") for _ in range(2))
    cos, sin = torch.empty(rows, d // 2, device="cuda"), torch.empty(rows, d // 2, device="cuda")
    Bn.k_rotary_tables(cos, sin, 10000.0)
    y, dx, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    Bn.k_rotary(x, y, cos, sin, heads, d)
    ref, mag = reference(x, cos, sin, torch.arange(rows, device="cuda"), heads, d, False, False)
    check(y, ref, mag, torch.float32)
    Bn.k_rotary(dy, dx, cos, sin, heads, d, inverse=True)
    # <y(x), dy> = <x, dx>: the map is linear; each element's error is under 2^-21 of its pair
    a, b = float((y.double() * dy.double()).sum()), float((x.double() * dx.double()).sum())
    assert abs(a - b) < 2.0 ** -19 * float(x.double().norm() * dy.double().norm())
    Bn.k_rotary(y, back, cos, sin, heads, d, inverse=True)
    assert float((back - x).abs().max()) < 1e-5  # a rotation: the inverse brings x back


@pytest.mark.parametrize("span,rot,theta,mscale,scaled", [(1, 2, 10000.0, 1.0, False), (300, 64, 10000.0, 1.0, False), (131072, 48, 500000.0, 0.75, True),
                                                          (1 << 20, 16, 10000.0, 1.0, True), (1000, 30, 100.0, 1.5, False)])
def test_tables(span, rot, theta, mscale, scaled):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rot)
    factors = 1.0 + 7.0 * torch.rand(rot // 2, generator=g, device="cuda") if scaled else None
    cos, sin = torch.full((span, rot // 2), 5.0, device="cuda"), torch.full((span, rot // 2), 5.0, device="cuda")
    Bn.k_rotary_tables(cos, sin, theta, factors=factors, mscale=mscale)
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    step = float(np.float32(theta)) ** (-2.0 * i / rot) / (factors.double() if scaled else 1.0)
    angle = torch.arange(span, dtype=torch.float64, device="cuda")[:, None] * step
    # the reduced angle is rounded to fp32 once (2^-24 of at most pi) and the functions are within 2^-22; the 64-bit angle of
    # either side is off by 2^-50 of up to 2^20 turns
    for got, want in ((cos, angle.cos()), (sin, angle.sin())):
        assert float((got.double() - mscale * want).abs().max()) < mscale * (3.2 * 2.0 ** -24 + 2.0 ** -22) + 1e-8


def test_positions_outside_the_tables_are_reported_and_their_rows_left():
    from paper_2609_13645_b200 import binding as Bn
    heads, d = 2, 16
    cos, sin = torch.ones(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    x, y = torch.randn(3, heads * d, device="cuda"), torch.full((3, heads * d), 3.0, device="cuda")
    for bad in (-1, 4, 2 ** 31 - 1, -2 ** 31):
        Bn.k_rotary(x, y.fill_(3.0), cos, sin, heads, d, positions=torch.tensor([0, bad, 3], dtype=torch.int32, device="cuda"))
        with pytest.raises(Bn.ForgeStepError) as e:
            Bn.k_status()
        assert e.value.status == Bn.FT_EINVAL
        assert torch.equal(y[[0, 2]], x[[0, 2]]) and (y[1] == 3).all()
    Bn.k_status()


def test_replays_read_the_positions():
    from paper_2609_13645_b200 import binding as Bn
    heads, d, rows = 4, 32, 50
    cos, sin = torch.empty(90, 16, device="cuda"), torch.empty(90, 16, device="cuda")
    Bn.k_rotary_tables(cos, sin)
    x = torch.randn(rows, heads * d, device="cuda").bfloat16()
    y = torch.empty_like(x)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    Bn.k_rotary(x, y, cos, sin, heads, d, positions=pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Bn.k_rotary(x, y, cos, sin, heads, d, positions=pos)
    pos += 40
    graph.replay()
    ref, mag = reference(x, cos, sin, pos, heads, d, False, False)
    check(y, ref, mag, torch.bfloat16)


@pytest.mark.parametrize("interleaved", [False, True])
def test_columns_beside_each_other(interleaved):
    """From some columns of a row into others; columns that share any are refused."""
    from paper_2609_13645_b200 import binding as Bn
    rows, heads, d = 70, 3, 32
    w = heads * d
    both = torch.randn(rows, 2 * w + 8, device="cuda").bfloat16()
    old = both.clone()
    cos, sin = torch.randn(rows, d // 2, device="cuda"), torch.randn(rows, d // 2, device="cuda")
    Bn.k_rotary(both[:, :w], both[:, w + 8:], cos, sin, heads, d, interleaved=interleaved)
    ref, mag = reference(old[:, :w], cos, sin, torch.arange(rows, device="cuda"), heads, d, interleaved, False)
    check(both[:, w + 8:], ref, mag, torch.bfloat16)
    assert torch.equal(both[:, :w + 8], old[:, :w + 8])
    for y in (both[:, w - 8:2 * w - 8], both[:, 8:w + 8]):
        with pytest.raises(Bn.ForgeStepError) as e:
            Bn.k_rotary(both[:, :w], y, cos, sin, heads, d, interleaved=interleaved)
        assert e.value.status == Bn.FT_EINVAL


def test_rows_past_32_bits():
    from paper_2609_13645_b200 import binding as Bn
    heads, d, ld = 2, 64, (1 << 30) + 64
    buf = torch.empty(2 * ld + heads * d, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, heads * d), (ld, 1))
    x.copy_(torch.randn(3, heads * d, device="cuda"))
    cos, sin = torch.randn(3, 32, device="cuda"), torch.randn(3, 32, device="cuda")
    ref, mag = reference(x, cos, sin, torch.arange(3, device="cuda"), heads, d, False, False)
    y = torch.empty(3, heads * d, dtype=torch.bfloat16, device="cuda")
    Bn.k_rotary(x, y, cos, sin, heads, d)
    Bn.k_rotary(x, x, cos, sin, heads, d)
    check(y, ref, mag, torch.bfloat16)
    assert torch.equal(x, y)
