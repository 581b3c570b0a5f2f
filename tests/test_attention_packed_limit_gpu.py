"""The limit on a document's rows that the backward pass of the packed attention is planned for, against the bounds it is given."""
import pytest
import torch

from .packed_util import inputs, offsets, reference_bwd, rel, tables

pytestmark = pytest.mark.gpu

GUARD = 4096


def setup(lens, tail, nh, nkv, d, longest, rope):
    """A forward pass with bounds of any document, and the backward call for documents of up to `longest`."""
    from paper_2609_13645_b200 import binding as Bn
    T = sum(lens) + tail
    qkv, do = inputs(lens, tail, nh, nkv, d, 4, garbage=1.0)
    bounds = torch.empty(3, T, dtype=torch.int32, device="cuda")
    o, lse = torch.zeros(T, nh * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(nh, T, device="cuda")
    cu = offsets(lens)
    Bn.k_packed_bounds(cu, bounds, T)
    Bn.k_attention_packed_fwd(qkv, o, lse, bounds, T, nh, nkv, d)
    Bn.k_status()
    size = Bn.attention_packed_scratch_bytes(T, nh, nkv, d, longest)
    scratch = torch.full((size + GUARD,), 77, dtype=torch.uint8, device="cuda")
    dqkv = torch.full_like(qkv, 9.0)
    cos, sin = tables(longest, d) if rope else (None, None)

    def call():
        Bn.k_attention_packed_bwd(qkv, o, do, lse, dqkv, bounds, scratch[:size], T, nh, nkv, d, longest, cos=cos, sin=sin)
    return call, dqkv, scratch[size:], (qkv, o, do, cu, bounds, cos, sin, T)


@pytest.mark.parametrize("nh,nkv,d", [(6, 1, 64), (12, 12, 64), (16, 8, 128)])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("lens,tail,longest", [([200, 301, 100], 30, 300), ([2], 0, 1), ([100, 0, 128, 1025, 64], 3, 129), ([1, 900] * 4, 200, 899),
                                               ([300] * 25, 57, 250)])
def test_longer_documents_are_reported(nh, nkv, d, rope, lens, tail, longest):
    from paper_2609_13645_b200 import binding as Bn
    call, dqkv, guard, (qkv, *_) = setup(lens, tail, nh, nkv, d, longest, rope)
    old = qkv.clone()
    call()
    with pytest.raises(Bn.ForgeStepError) as e:
        Bn.k_status()
    assert e.value.status == Bn.FT_EINVAL
    Bn.k_status()
    assert (dqkv[sum(lens):] == 9).all() and (guard == 77).all() and torch.equal(qkv, old)


@pytest.mark.parametrize("nh,nkv,d", [(6, 1, 64), (16, 8, 128)])
def test_documents_of_the_limit(nh, nkv, d):
    """As many rows as the limit, and a captured call whose replays meet longer ones and then shorter ones again."""
    from paper_2609_13645_b200 import binding as Bn
    lens, longest = [300, 0, 77, 300, 128], 300
    call, dqkv, _, (qkv, o, do, cu, bounds, cos, sin, T) = setup(lens, 0, nh, nkv, d, longest, True)
    call()
    Bn.k_status()
    want = reference_bwd(qkv, o, do, lens, nh, nkv, d, cos, sin)
    assert rel(dqkv, want) < 3e-3  # dS and the result are rounded to bf16: sqrt(2) 1.7e-3
    first = dqkv.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for one in ([301, 1, 75, 300, 128], lens):
        cu.copy_(offsets(one))
        Bn.k_packed_bounds(cu, bounds, T)
        graph.replay()
        if one == lens:
            Bn.k_status()
        else:
            with pytest.raises(Bn.ForgeStepError):
                Bn.k_status()
    assert torch.equal(dqkv, first)
