"""LayerNorm forward and backward against a plain 64-bit implementation.

Tolerances: bf16 outputs carry one rounding (half a step, 2^-8 of the value at most; over many values, whose distance to
the next step is uniform, 2^-8 / sqrt(3) times 0.72, the mean over a binade: 1.7e-3 in the 2-norm; the 2-norm is allowed
2.5e-3, or 2^-8 for tensors of under 100 elements, where the mean means nothing); fp32 outputs the error of fp32 sums over a row or a column, about
sqrt(n) 2^-24 of their terms' norm, allowed 1e-5 relative in the 2-norm (the reference uses the fp32 statistics the kernel got).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _rel(a, b):
    return float((a.double() - b).norm() / b.norm().clamp_min(1e-300))


def _rand(g, rows, h, dtype, pad=0, offset=0, spread=1.0, shift=0.0):
    """[rows, h]; with pad, rows of a wider buffer; with offset, starting that many elements into it."""
    t = (torch.randn(rows, h + pad + offset, generator=g, device="cuda") * spread + shift).to(dtype)
    return t[:, offset:offset + h]


def _reference(x, gain, bias, eps):
    x = x.double()
    mean = x.mean(-1)
    rstd = 1.0 / ((x - mean[:, None]).square().mean(-1) + eps).sqrt()
    y = (x - mean[:, None]) * rstd[:, None] * gain.double()
    return (y if bias is None else y + bias.double()), mean, rstd


def _reference_bwd(dy, x, mean, rstd, gain, resid):
    x, dy, mean, rstd = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    xh, g = (x - mean) * rstd, dy * gain.double()
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return (dx if resid is None else dx + resid.double()), (dy * xh).sum(0), dy.sum(0)


# one row, one column, odd widths, each vector width, each group width, several groups a block, widths past 2048 and 8192
SHAPES = [(1, 1), (3, 2), (1, 7), (5, 8), (37, 31), (130, 64), (1000, 96), (77, 257), (19, 768), (300, 771), (9, 1024), (13, 1030),
          (600, 2048), (7, 2052), (33, 4096), (5, 4104), (3, 8192), (2, 8200), (3, 16384), (4000, 40)]


@pytest.mark.parametrize("rows,h", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", [True, False])
def test_forward_and_backward_match_the_definition(rows, h, dtype, bias):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + h)
    x = _rand(g, rows, h, dtype, spread=1.5, shift=0.25)
    gain = (1 + 0.2 * torch.randn(h, generator=g, device="cuda")).to(dtype)
    b = (0.2 * torch.randn(h, generator=g, device="cuda")).to(dtype) if bias else None
    y, mean, rstd = torch.full_like(x, 7.0), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, b, y, mean, rstd, 1e-5)
    y_ref, mean_ref, rstd_ref = _reference(x, gain, b, 1e-5)
    tol = 1e-5 if dtype == F32 else 2.5e-3 if rows * h >= 100 else 2.0 ** -8
    assert float((mean.double() - mean_ref).abs().max()) < 1e-5 * float(x.float().abs().max())
    assert _rel(rstd, rstd_ref) < 1e-5
    if h > 1:  # of one column nothing but the bias is left
        assert _rel(y, y_ref) < tol
    else:
        assert torch.equal(y, torch.zeros_like(y) if b is None else b.expand(rows, 1))

    dy, r = _rand(g, rows, h, dtype), (_rand(g, rows, h, dtype) if bias else None)
    dx, dgain = torch.full_like(x, 7.0), torch.full((h,), 7.0, device="cuda")
    dbias = torch.full((h,), 7.0, device="cuda") if bias else None
    scratch = torch.full((Bn.layernorm_scratch_bytes(rows, h) // 4,), float("nan"), device="cuda").view(torch.uint8)
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, dx, dgain, dbias, scratch)
    dx_ref, dg_ref, db_ref = _reference_bwd(dy, x, mean, rstd, gain, r)
    if h > 2 or r is not None:  # two columns leave no direction for the gradient: dx is rounding noise of rstd |dy|
        assert _rel(dx, dx_ref) < tol
    assert float((dx.double() - dx_ref).abs().max()) < (2.0 ** -8 if dtype == BF16 else 1e-4) * float(rstd.max() * dy.float().abs().max() * 2 + 8)
    terms = (dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])).norm()
    assert float((dgain.double() - dg_ref).norm()) <= 1e-5 * float(dg_ref.norm()) + 1e-6 * float(terms)
    if bias:
        assert float((dbias.double() - db_ref).norm()) <= 1e-5 * float(db_ref.norm()) + 1e-6 * float(dy.double().norm())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,offset", [(3, 0), (8, 0), (4, 4), (5, 1), (2, 2)])
def test_strided_and_unaligned_rows_give_the_same_bits_as_packed_ones(dtype, pad, offset):
    """Strides and offsets only change the width of the accesses: per column the sums run over the same rows in the same order
    where the vector width is the same, and to rounding where it is not; the elements around the rows stay."""
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 203, 520
    g = torch.Generator(device="cuda").manual_seed(pad * 10 + offset)
    x, dy, r = (_rand(g, rows, h, dtype, pad, offset) for _ in range(3))
    gain = torch.randn(h, generator=g, device="cuda").to(dtype)
    bias = torch.randn(h, generator=g, device="cuda").to(dtype)
    out = torch.full((rows, h + pad + offset), 3.0, dtype=dtype, device="cuda")
    y = out[:, offset:offset + h]
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, bias, y, mean, rstd)
    y_ref, _, _ = _reference(x, gain, bias, 1e-5)
    tol = 2.5e-3 if dtype == BF16 else 1e-5
    assert _rel(y, y_ref) < tol
    rest = torch.ones(h + pad + offset, dtype=torch.bool, device="cuda")
    rest[offset:offset + h] = False
    assert (out[:, rest] == 3).all()
    dgain, dbias = torch.empty(h, device="cuda"), torch.empty(h, device="cuda")
    scratch = torch.empty(Bn.layernorm_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda")
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, y, dgain, dbias, scratch)
    dx_ref, dg_ref, db_ref = _reference_bwd(dy, x, mean, rstd, gain, r)
    assert _rel(y, dx_ref) < tol and _rel(dgain, dg_ref) < 1e-5 and _rel(dbias, db_ref) < 1e-5
    assert (out[:, rest] == 3).all()


def test_rows_with_a_large_mean_keep_their_variance():
    """Mean 4096 times the standard deviation: sum(x^2) / h - mean^2 would have lost every digit of the variance."""
    from paper_2609_13645_b200 import binding as Bn
    for rows, h in ((16, 768), (4, 5000)):
        g = torch.Generator(device="cuda").manual_seed(h)
        x = _rand(g, rows, h, F32, shift=4096.0)
        gain, y = torch.ones(h, device="cuda"), torch.empty(rows, h, device="cuda")
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        Bn.k_layernorm_fwd(x, gain, None, y, mean, rstd)
        y_ref, _, rstd_ref = _reference(x, gain, None, 1e-5)
        # the fp32 mean is off by up to 2^-24 * 4096 * 2 of a standard deviation
        assert _rel(rstd, rstd_ref) < 1e-5 and _rel(y, y_ref) < 1e-3


def test_constant_rows_and_outputs_in_place():
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 12, 512
    x = torch.full((rows, h), 3.0, dtype=BF16, device="cuda")
    gain, bias = torch.ones(h, dtype=BF16, device="cuda"), torch.full((h,), 0.5, dtype=BF16, device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, bias, x, mean, rstd)
    assert (x == 0.5).all() and (mean == 3).all()
    g = torch.Generator(device="cuda").manual_seed(2)
    for dtype in (BF16, F32):
        for hh in (512, 9000):
            x, dy, r = (_rand(g, rows, hh, dtype) for _ in range(3))
            gain = torch.ones(hh, dtype=dtype, device="cuda")
            y = torch.empty_like(x)
            Bn.k_layernorm_fwd(x, gain, None, y, mean, rstd)
            out = []
            for target in (torch.empty_like(x), dy.clone(), r.clone()):
                dgain, dbias = torch.empty(hh, device="cuda"), torch.empty(hh, device="cuda")
                scratch = torch.empty(Bn.layernorm_scratch_bytes(rows, hh), dtype=torch.uint8, device="cuda")
                a = target if len(out) == 1 else dy
                b = target if len(out) == 2 else r
                Bn.k_layernorm_bwd(a, x, mean, rstd, gain, b, target, dgain, dbias, scratch)
                out.append((target, dgain, dbias))
            for other in out[1:]:
                assert all(torch.equal(p, q) for p, q in zip(out[0], other))


def test_bit_identical_from_run_to_run_and_when_replayed():
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 4099, 1536
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy, r = (_rand(g, rows, h, BF16) for _ in range(3))
    gain, bias = torch.randn(h, device="cuda", generator=g).to(BF16), torch.randn(h, device="cuda", generator=g).to(BF16)
    bufs = lambda: (torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),  # noqa: E731
                    torch.empty_like(x), torch.empty(h, device="cuda"), torch.empty(h, device="cuda"))
    scratch = torch.empty(Bn.layernorm_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda")

    def step(t):
        Bn.k_layernorm_fwd(x, gain, bias, t[0], t[1], t[2])
        Bn.k_layernorm_bwd(dy, x, t[1], t[2], gain, r, t[3], t[4], t[5], scratch)

    first, second, third = bufs(), bufs(), bufs()
    step(first)
    step(second)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(third)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_gradients_agree_with_differences():
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 20, 96
    g = torch.Generator(device="cuda").manual_seed(8)
    x, dy = _rand(g, rows, h, F32), _rand(g, rows, h, F32)
    gain, bias = torch.randn(h, device="cuda", generator=g), torch.randn(h, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, bias, y, mean, rstd)
    dx, dgain, dbias = torch.empty_like(x), torch.empty(h, device="cuda"), torch.empty(h, device="cuda")
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, None, dx, dgain, dbias, torch.empty(Bn.layernorm_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda"))
    f = lambda a, b, c: (_reference(a, b, c, 1e-5)[0] * dy.double()).sum()  # noqa: E731
    eps = 1e-5
    for t, grad, at in ((x, dx, 0), (gain, dgain, 1), (bias, dbias, 2)):
        v = torch.randn(t.shape, dtype=torch.float64, device="cuda", generator=g)
        args = [x.double(), gain.double(), bias.double()]
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + eps * v, args[at] - eps * v
        diff = float((f(*up) - f(*down)) / (2 * eps))
        assert abs(diff - float((grad.double() * v).sum())) < 1e-4 * float(grad.double().norm()) * float(v.norm()) ** 0.5


def _at(t, ld, offset):
    """A copy of t whose rows are ld apart and begin `offset` elements into an allocation that ends with the last of them."""
    rows, h = t.shape
    buf = torch.empty(offset + (rows - 1) * ld + h, dtype=t.dtype, device=t.device)
    view = torch.as_strided(buf, (rows, h), (ld, 1), offset)
    view.copy_(t)
    return view


# every tensor starts elsewhere against the 16-byte boundaries, and moves on differently from row to row
@pytest.mark.parametrize("rows,h", [(1, 3), (3, 1), (5, 7), (2, 9), (40, 241), (40, 243), (1500, 33), (2600, 300), (700, 2047), (9, 4095), (4, 8179), (3, 8191),
                                    (3, 16371), (3, 16384)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_tensor_at_an_alignment_of_its_own(rows, h, dtype):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    x, dy, r = (_at(_rand(g, rows, h, dtype), h + e, o) for e, o in ((3, 1), (0, 6), (10, 3)))
    y, dx = (_at(torch.full((rows, h), 7.0, dtype=dtype, device="cuda"), h + e, o) for e, o in ((1, 5), (5, 2)))
    gain = torch.randn(h + 1, generator=g, device="cuda").to(dtype)[1:]
    bias = torch.randn(h + 3, generator=g, device="cuda").to(dtype)[3:]
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, bias, y, mean, rstd)
    y_ref, mean_ref, rstd_ref = _reference(x, gain, bias, 1e-5)
    tol = 1e-5 if dtype == F32 else 2.5e-3 if rows * h >= 100 else 2.0 ** -8
    assert float((mean.double() - mean_ref).abs().max()) < 1e-5 * float(x.float().abs().max()) and _rel(rstd, rstd_ref) < 1e-5
    assert _rel(y, y_ref) < tol
    dgain, dbias = torch.empty(h, device="cuda"), torch.empty(h, device="cuda")
    scratch = torch.full((Bn.layernorm_scratch_bytes(rows, h) // 4,), float("nan"), device="cuda").view(torch.uint8)
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, dx, dgain, dbias, scratch)
    dx_ref, dg_ref, db_ref = _reference_bwd(dy, x, mean, rstd, gain, r)
    # the terms of dx, rstd g, rstd mean(g) and rstd xhat mean(g xhat), are rounded where they are as large as rstd |g|, and may
    # cancel (of one column nothing is left, with rstd = 1 / sqrt(eps) = 316): 4 roundings of 2^-24 of that beside the relative error
    slack = 4 * 2.0 ** -24 * float((rstd.double()[:, None] * dy.double() * gain.double()).norm())
    assert float((dx.double() - dx_ref).norm()) < tol * float(dx_ref.norm()) + slack
    terms = (dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])).norm()
    assert float((dgain.double() - dg_ref).norm()) <= 1e-5 * float(dg_ref.norm()) + 1e-6 * float(terms)
    assert float((dbias.double() - db_ref).norm()) <= 1e-5 * float(db_ref.norm()) + 1e-6 * float(dy.double().norm())
    # in place, over the rows the kernel reads
    z = _at(x, h + 3, 1)
    Bn.k_layernorm_fwd(z, gain, bias, z, mean, rstd)
    assert torch.equal(z, y) or _rel(z, y_ref) < tol
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, r, dgain, dbias, scratch)
    assert float((r.double() - dx_ref).norm()) < tol * float(dx_ref.norm()) + slack
    w, d = _at(x, h + 3, 1), _at(x, h + 3, 1)
    Bn.k_layernorm_bwd(dy, w, mean, rstd, gain, None, d, dgain, dbias, scratch)
    Bn.k_layernorm_bwd(dy, w, mean, rstd, gain, None, w, dgain, dbias, scratch)
    assert torch.equal(w, d)
