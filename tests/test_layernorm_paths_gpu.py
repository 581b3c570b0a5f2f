"""LayerNorm where a block holds one row at a time and leaves its own partial sums, and where a group of warps takes many rows, so
that every slot of its ring of rows is filled again and again.  Definition and tolerances as in test_layernorm_gpu.py."""
import pytest
import torch

from tests.test_layernorm_gpu import BF16, F32, _at, _rand, _reference, _reference_bwd, _rel

pytestmark = pytest.mark.gpu


def _check(x, dy, r, gain, bias, y, dx, runs=1):
    from paper_2609_13645_b200 import binding as Bn
    rows, h = x.shape
    tol = 2.5e-3 if x.dtype == BF16 else 1e-5
    first = None
    for _ in range(runs):
        y.fill_(7)
        dx.fill_(7)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        Bn.k_layernorm_fwd(x, gain, bias, y, mean, rstd)
        dgain = torch.full((h,), 7.0, device="cuda")
        dbias = torch.full((h,), 7.0, device="cuda") if bias is not None else None
        scratch = torch.full((Bn.layernorm_scratch_bytes(rows, h) // 4,), float("nan"), device="cuda").view(torch.uint8)
        Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, dx, dgain, dbias, scratch)
        got = [t.clone() for t in (y, mean, rstd, dx, dgain) + ((dbias,) if bias is not None else ())]
        if first is None:
            first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    y_ref, mean_ref, rstd_ref = _reference(x, gain, bias, 1e-5)
    assert float((mean.double() - mean_ref).abs().max()) < 1e-5 * float(x.float().abs().max()) and _rel(rstd, rstd_ref) < 1e-5
    assert _rel(y, y_ref) < tol
    # row by row: one wrong row of thousands would not show in the norm over all (of at least 33 elements a row, a row's
    # 2-norm is within half a step of each, 2^-8 in bf16; fp32 as above)
    by_row = lambda a, b: float(((a.double() - b).norm(dim=1) / b.norm(dim=1)).max())  # noqa: E731
    row_tol = 2.0 ** -8 if x.dtype == BF16 else 1e-5
    assert by_row(y, y_ref) < row_tol
    dx_ref, dg_ref, db_ref = _reference_bwd(dy, x, mean, rstd, gain, r)
    assert _rel(dx, dx_ref) < tol and by_row(dx, dx_ref) < row_tol
    terms = (dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])).norm(dim=0)
    # column by column: fp32 sums of `rows` terms, 1e-6 of their 2-norm as for the whole vector, here with 8 times the room for
    # the worst of h columns
    assert ((dgain.double() - dg_ref).abs() <= 1e-5 * dg_ref.abs() + 8e-6 * terms).all()
    if bias is not None:
        assert ((dbias.double() - db_ref).abs() <= 1e-5 * db_ref.abs() + 8e-6 * dy.double().norm(dim=0)).all()


# one row a block and more rows than one launch of a cluster takes; rows beyond the number of SMs; each chunk width (4104, 4100
# and 4099 columns are multiples of 8, 4 and 1); fp32 rows past 8192 columns, which have no ring
@pytest.mark.parametrize("rows,h", [(17, 4104), (200, 8192), (160, 4100), (400, 4099), (160, 8200), (300, 16384), (149, 12288), (700, 2052)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("full", [True, False])
def test_one_row_a_block_past_the_cluster(rows, h, dtype, full):
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    x = _rand(g, rows, h, dtype, spread=1.5, shift=0.25)
    dy, r = _rand(g, rows, h, dtype), (_rand(g, rows, h, dtype) if full else None)
    gain = (1 + 0.2 * torch.randn(h, generator=g, device="cuda")).to(dtype)
    bias = (0.2 * torch.randn(h, generator=g, device="cuda")).to(dtype) if full else None
    _check(x, dy, r, gain, bias, torch.empty_like(x), torch.empty_like(x))


# rows a group takes: about 28, 5, 10, 19, 10 and 8 backward and a third to all of that forward; groups of 4, 1, 2, 16 and 17 warps
@pytest.mark.parametrize("rows,h", [(8192, 2047), (20000, 33), (6000, 771), (3000, 8191), (1300, 16371), (1200, 16383)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_a_group_at_alignments_of_their_own(rows, h, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    x, dy, r = (_at(_rand(g, rows, h, dtype), h + e, o) for e, o in ((3, 1), (0, 6), (10, 3)))
    y, dx = (_at(torch.empty(rows, h, dtype=dtype, device="cuda"), h + e, o) for e, o in ((1, 5), (5, 2)))
    gain = (1 + 0.2 * torch.randn(h + 1, generator=g, device="cuda")).to(dtype)[1:]
    bias = (0.2 * torch.randn(h + 3, generator=g, device="cuda")).to(dtype)[3:]
    _check(x, dy, r, gain, bias, y, dx, runs=2)


@pytest.mark.parametrize("rows,h", [(8192, 2047), (1500, 8191)])
def test_many_odd_rows_in_place(rows, h):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(h)
    x, dy, r = (_rand(g, rows, h, BF16) for _ in range(3))
    gain = torch.randn(h, generator=g, device="cuda").to(BF16)
    mean, rstd, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    Bn.k_layernorm_fwd(x, gain, None, y, mean, rstd)
    z = x.clone()
    Bn.k_layernorm_fwd(z, gain, None, z, mean, rstd)
    assert torch.equal(z, y)
    want, dgain = torch.empty_like(x), torch.empty(h, device="cuda")
    scratch = torch.empty(Bn.layernorm_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda")
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, want, dgain, None, scratch)
    for at in range(3):
        t = [dy.clone(), x.clone(), r.clone()]
        Bn.k_layernorm_bwd(t[0], t[1], mean, rstd, gain, t[2], t[at], dgain, None, scratch)
        assert torch.equal(t[at], want), at
