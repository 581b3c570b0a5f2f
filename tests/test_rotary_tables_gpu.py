"""The rotation tables against angles in 64 bits.  Sine and cosine, below 1, are off by a last place of theirs (2^-24 at most) and by half of one where
what is left of the angle is added, times mscale; the product with mscale is rounded to half a last place of the product, which is not mscale times as
much: 2^-25 for products below 1 (0.74 has the places of 0.99) and 2^-24 for those from 1 to 2.  The 64-bit angles themselves, of either side, are
off by 2^-51 of the angle."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def definition(span, rot, theta, factors, mscale):
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    step = float(np.float32(theta)) ** (-2.0 * i / rot) / (factors.double() if factors is not None else 1.0)
    angle = torch.arange(span, dtype=torch.float64, device="cuda")[:, None] * step
    return angle, mscale * angle.cos(), mscale * angle.sin()


@pytest.mark.parametrize("span,rot,theta,mscale,scaled", [(1, 2, 10000.0, 1.0, False), (300, 64, 10000.0, 1.0, False), (131072, 48, 500000.0, 0.75, True),
                                                          (1 << 20, 16, 10000.0, 1.0, True), (1000, 30, 100.0, 1.5, False), (4096, 128, 1e6, 1.0, False)])
def test_entries_are_within_two_last_places(span, rot, theta, mscale, scaled):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rot)
    factors = 1.0 + 7.0 * torch.rand(rot // 2, generator=g, device="cuda") if scaled else None
    cos, sin = torch.full((span, rot // 2), 5.0, device="cuda"), torch.full((span, rot // 2), 5.0, device="cuda")
    Bn.k_rotary_tables(cos, sin, theta, factors=factors, mscale=mscale)
    angle, want_cos, want_sin = definition(span, rot, theta, factors, mscale)
    half_a_place = 2.0 ** -25 if mscale <= 1 else 2.0 ** -24
    for got, want in ((cos, want_cos), (sin, want_sin)):
        assert ((got.double() - want).abs() <= mscale * (1.5 * 2.0 ** -24 + 2.0 ** -51 * angle) + half_a_place).all()
    # sines of small angles to two last places of themselves
    small = (angle > 0) & (angle < 0.5)
    assert ((sin.double() - want_sin)[small].abs() <= 2.0 * 2.0 ** -23 * want_sin[small].abs() + mscale * 2.0 ** -51 * angle[small]).all()


def test_the_norm_of_the_error_is_that_of_roundings():
    """131072 positions of 24 frequencies: roundings to 24 bits are off by 2^-24 / sqrt(3) times 0.72 of the value in the 2-norm, 2.5e-8 (0.72 2^-24 / 3^0.5); of two and the
    functions' own, at most 2^-24 of a value, which averages like a rounding of twice the step: sqrt(1 + 1 + 4) 2.5e-8."""
    from paper_2609_13645_b200 import binding as Bn
    span, rot = 131072, 48
    cos, sin = torch.empty(span, rot // 2, device="cuda"), torch.empty(span, rot // 2, device="cuda")
    Bn.k_rotary_tables(cos, sin, 10000.0)
    _, want_cos, want_sin = definition(span, rot, 10000.0, None, 1.0)
    for got, want in ((cos, want_cos), (sin, want_sin)):
        error = float((got.double() - want).norm() / want.norm())
        assert error < 6.0 ** 0.5 * 2.5e-8


@pytest.mark.parametrize("bad", [0.0, -0.0, float("nan")])
def test_a_factor_without_an_angle_gives_no_entries(bad):
    from paper_2609_13645_b200 import binding as Bn
    span, half = 500, 40
    factors = torch.linspace(1.0, 3.0, half, device="cuda")
    factors[7] = bad
    cos, sin = torch.empty(span, half, device="cuda"), torch.empty(span, half, device="cuda")
    Bn.k_rotary_tables(cos, sin, 10000.0, factors=factors)
    rest = torch.arange(half, device="cuda") != 7
    for t in (cos, sin):
        assert t[:, 7].isnan().all() and t[:, rest].isfinite().all()
    still = torch.full((half,), float("inf"), device="cuda")  # angles of 0
    Bn.k_rotary_tables(cos, sin, 10000.0, factors=still)
    assert (cos == 1).all() and (sin == 0).all()
