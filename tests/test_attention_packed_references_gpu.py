"""Softmax references that move between the blocks of a row, in every way in which the two-tile forward kernel of the packed attention pairs its
tiles: heads that share K and V or have their own, and neighbouring blocks of queries of a head, of which one may join behind the other.

Keys of any size from 2^-6 to 2^6 make scores of up to 64 * 30: an fp32 score is a sum of d terms, off by up to d 2^-24 of 2000, by which a row's
log-sum-exp may be off and, relative to themselves, its weights; o has its own 3e-3 of roundings beside."""
import numpy as np
import pytest
import torch

from .packed_util import inputs, reference_fwd, rel
from .test_attention_packed_gpu import run_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nh,nkv,d,T", [(16, 8, 128, 7200), (24, 12, 64, 4800), (24, 24, 64, 4800), (12, 4, 64, 9500), (24, 24, 128, 4750), (27, 9, 128, 4300),
                                        (33, 11, 64, 3500), (33, 33, 64, 3470), (18, 6, 128, 6401)])
@pytest.mark.parametrize("long", [True, False])
def test_references_that_move(nh, nkv, d, T, long):
    """Long documents: references move many times a row.  Short ones: tiles that begin and end apart from each other."""
    assert (T + 127) // 128 * nh >= 6 * 148  # calls that the two-tile kernel serves
    g = np.random.RandomState(T + nh)
    lens = [1200, 0, 1, T - 2000, 400] if long else [int(m) for m in g.randint(1, 500, T // 250 - 8)] + [129]
    n = sum(lens)
    assert 0 < n <= T
    qkv, _ = inputs(lens, T - n, nh, nkv, d, 12)
    r = torch.Generator(device="cuda").manual_seed(3)
    qkv[:n, nh * d:(nh + nkv) * d] *= torch.exp2(torch.randint(-6, 7, (n, 1), generator=r, device="cuda").float()).bfloat16()
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    off = d * 2.0 ** -24 * 2000
    r = nh // nkv
    for a in range(nkv):  # the reference by kv heads: its scores are many
        cols = [h * d + c for h in list(range(a * r, (a + 1) * r)) + [nh + a, nh + nkv + a] for c in range(d)]
        want, want_lse = reference_fwd(qkv[:, cols], lens, r, 1, d)
        assert rel(o[:n, a * r * d:(a + 1) * r * d], want) < off + 3e-3, a
        assert float((lse[a * r:(a + 1) * r, :n].double() - want_lse).abs().max()) < off, a
    assert (o[n:] == 7).all() and (lse[:, n:] == 7).all()
    o2, lse2, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
