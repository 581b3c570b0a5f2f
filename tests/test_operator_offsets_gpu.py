"""The decoder-block operators where element offsets pass 32 bits: rows far apart in one allocation, more elements than 2^32 in one
call, and packed q, k, v of more than 2^31 elements.  Tolerances as in the operators' own tests."""
import numpy as np
import pytest
import torch

from tests.test_attention_window_gpu import _inputs, _reference_bwd, _reference_fwd, _rel
from tests.test_dropout_gpu import M64, _mix
from tests.test_layernorm_gpu import BF16, F32, _reference, _reference_bwd as _ln_reference_bwd, _rel as _ln_rel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,h,ld,odd", [(3, 2048, 1 << 31, 0), (300, 4104, (1 << 24) + 8, 0), (300, 1023, (1 << 24) + 3, 5)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layernorm_and_dropout_of_rows_far_apart(rows, h, ld, odd, dtype):
    from paper_2609_13645_b200 import binding as Bn
    if dtype == F32:
        ld //= 2
        ld += ld % 2 * (odd > 0)
    buf = torch.empty((rows - 1) * ld + 6 * (h + 64), dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(h)
    at = [torch.as_strided(buf, (rows, h), (ld, 1), i * (h + 64 - h % 8) + odd * (i % 3)) for i in range(6)]
    x, dy, r, y, dx, z = at
    for t in (x, dy, r):
        t.copy_(torch.randn(rows, h, generator=g, device="cuda"))
    for t in (y, dx, z):
        t.fill_(7)
    gain, bias = (torch.randn(h, generator=g, device="cuda").to(dtype) for _ in range(2))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    Bn.k_layernorm_fwd(x, gain, bias, y, mean, rstd)
    tol = 2.5e-3 if dtype == BF16 else 1e-5
    assert _ln_rel(y, _reference(x, gain, bias, 1e-5)[0]) < tol
    dgain, dbias = torch.empty(h, device="cuda"), torch.empty(h, device="cuda")
    scratch = torch.empty(Bn.layernorm_scratch_bytes(rows, h), dtype=torch.uint8, device="cuda")
    Bn.k_layernorm_bwd(dy, x, mean, rstd, gain, r, dx, dgain, dbias, scratch)
    dx_ref, dg_ref, db_ref = _ln_reference_bwd(dy, x, mean, rstd, gain, r)
    assert _ln_rel(dx, dx_ref) < tol and _ln_rel(dgain, dg_ref) < 1e-5 and _ln_rel(dbias, db_ref) < 1e-5
    Bn.k_dropout_add(x, r, z, 0.25, 3, 1)
    packed = torch.empty(rows, h, dtype=dtype, device="cuda")
    Bn.k_dropout_add(x.clone(), r.clone(), packed, 0.25, 3, 1)
    assert torch.equal(z, packed)


def _keep(first, n, p, seed, site):
    """Whether the elements [first, first + n) of a tensor are kept, at step 0."""
    with np.errstate(over="ignore"):
        key = _mix(_mix(np.array([(seed ^ ((site + 1) * 0xD1B54A32D192ED03)) & M64], dtype=np.uint64)))
        i = np.arange(first, first + n, dtype=np.uint64)
        word = _mix(key ^ (i // np.uint64(4) * np.uint64(0x8CB92BA72F3D8DD7)))
        bits = (word >> (np.uint64(16) * (i % np.uint64(4)))) & np.uint64(0xFFFF)
    return torch.from_numpy(bits >= np.uint64(int(p * 65536 + 0.5))).cuda()


@pytest.mark.parametrize("rows,h", [(70000, 65536), (66000, 65537)])
def test_dropout_of_more_elements_than_32_bits_count(rows, h):
    from paper_2609_13645_b200 import binding as Bn
    x = torch.ones(rows, h, dtype=BF16, device="cuda")
    out = x if h % 8 == 0 else torch.empty(rows, h + 7, dtype=BF16, device="cuda")[:, 3:3 + h]
    Bn.k_dropout_add(x, None, out, 0.5, 77, 2)
    for row in (0, 1, 32767, 32768, 65535, 65536, rows - 1):
        assert torch.equal(out[row] != 0, _keep(row * h, h, 0.5, 77, 2)), row


# a query head for each of 43 kv heads, whose dS^T is kept in rounds, and 128 query heads on one kv head, which recompute it
@pytest.mark.parametrize("nh,nkv", [(43, 43), (128, 1)])
def test_attention_over_more_elements_than_32_bits_count(nh, nkv):
    from paper_2609_13645_b200 import binding as Bn
    S, d, window, n = 131200, 128, 100, 500
    qkv, do = _inputs(1, S, nh, nkv, d, seed=nh)
    assert qkv.numel() > 2 ** 31
    o, lse = torch.empty(S, nh * d, dtype=BF16, device="cuda"), torch.empty(1, nh, S, device="cuda")
    Bn.k_attention_window_fwd(qkv, o, lse, 1, S, nh, nkv, d, window, 0)
    dqkv = torch.empty_like(qkv)
    scratch = torch.empty(Bn.attention_window_scratch_bytes(1, S, nh, nkv, d, window, 0), dtype=torch.uint8, device="cuda")
    Bn.k_attention_window_bwd(qkv, o, do, lse, dqkv, scratch, 1, S, nh, nkv, d, window, 0)
    # without sinks, what a run of rows sees and is seen by lies within a window of it: runs of 500 rows as sequences of their own,
    # compared where neither end cuts anything off
    for i0 in (0, 65000, S - n):
        rows = slice(i0, i0 + n)
        part = qkv[rows].contiguous()
        o_ref, lse_ref = _reference_fwd(part, 1, n, nh, nkv, d, window, 0)
        ref = _reference_bwd(part, o[rows], do[rows], 1, n, nh, nkv, d, window, 0)
        a, b = 0 if i0 == 0 else window, n if i0 + n == S else n - window
        assert _rel(o[rows][a:], o_ref[a:]) < 3e-3, i0
        assert float((lse[0, :, rows].double() - lse_ref[0])[:, a:].abs().max()) < 2e-5, i0
        got, hq = dqkv[rows], nh * d
        assert _rel(got[a:, :hq], ref[a:, :hq]) < 3e-3, i0
        assert _rel(got[a:b, hq:], ref[a:b, hq:]) < 3e-3, i0
