"""Attention inside the documents of a packed batch, forward and backward, against a plain 64-bit implementation of its definition.

Tolerances, relative in the 2-norm of a tensor unless said otherwise.  One rounding to bf16 is off by at most half a step,
u = 2^-8 of the value; over many values, whose distance to the next step is uniform, by 2^-8 / sqrt(3) times 0.72 (the mean
over a binade) = 1.7e-3 in the 2-norm, and independent roundings add in squares.
  o        P is rounded (its error averages like the sum it enters) and o is:         sqrt(2) 1.7e-3 = 2.4e-3, taken as 3e-3
  lse      fp32 scores (d terms of |s| <= 30, d 2^-24 relative) and exp2 / log2 (2^-22): absolute <= 2e-5
  d_v      P rounded, d_v rounded; d_q, d_k: dS rounded, result rounded: the same 2.4e-3, taken as 3e-3.  delta is formed
           from the o that the reference is given too.
Tensors of under 1000 elements are too few for the mean and are held to 2 u = 2^-7.  d_q and d_k of documents of one row are
differences that cancel to 0 but for dO v - dO o, whose o is rounded (half a step of o): they are compared in absolute terms.
"""
import numpy as np
import pytest
import torch

from .packed_util import inputs, offsets, reference_bwd, reference_fwd, rel, tables

pytestmark = pytest.mark.gpu

DOCS = [
    ([1], 0), ([0, 1, 0], 2), ([2], 0), ([5, 0, 3], 7), ([63, 1], 1), ([64, 64], 0), ([127, 1, 129], 0), ([128, 128], 1), ([130], 126),
    ([1] * 200, 5), ([3, 61, 64, 65, 0, 0, 127, 128, 129, 200], 33), ([700], 68), ([17, 900, 4, 333], 130), ([40] * 37, 0),
]


def tol(n):
    return 3e-3 if n >= 1000 else 2.0 ** -7


def run_fwd(qkv, lens, T, nh, nkv, d):
    from paper_2609_13645_b200 import binding as Bn
    o = torch.full((T, nh * d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((nh, T), 7.0, device="cuda")
    bounds = torch.empty(3, T, dtype=torch.int32, device="cuda")
    Bn.k_packed_bounds(offsets(lens), bounds, T, max(max(lens), 1))
    Bn.k_attention_packed_fwd(qkv, o, lse, bounds, T, nh, nkv, d)
    Bn.k_status()
    return o, lse, bounds


def run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, longest, cos=None, sin=None):
    from paper_2609_13645_b200 import binding as Bn
    dqkv = torch.full_like(qkv, 9.0)
    scratch = torch.full((Bn.attention_packed_scratch_bytes(T, nh, nkv, d, longest),), 255, dtype=torch.uint8, device="cuda")  # NaN
    Bn.k_attention_packed_bwd(qkv, o, do, lse, dqkv, bounds, scratch, T, nh, nkv, d, longest, cos=cos, sin=sin)
    Bn.k_status()
    return dqkv


@pytest.mark.parametrize("lens,tail", DOCS + [([], 3)])
def test_bounds(lens, tail):
    from paper_2609_13645_b200 import binding as Bn
    T, n = sum(lens) + tail, sum(lens)
    bounds = torch.full((3, T), -1, dtype=torch.int32, device="cuda")
    Bn.k_packed_bounds(offsets(lens), bounds, T)
    Bn.k_status()
    want, at = np.zeros((3, T), dtype=np.int32), 0
    for m in lens:
        want[0, at:at + m], want[1, at:at + m], want[2, at:at + m] = at, at + m, np.arange(m)
        at += m
    want[0, n:], want[1, n:] = T, n
    assert np.array_equal(bounds.cpu().numpy(), want)


@pytest.mark.parametrize("lens,tail", DOCS)
@pytest.mark.parametrize("nh,nkv,d", [(2, 1, 64), (4, 4, 64), (4, 2, 128)])
def test_forward(lens, tail, nh, nkv, d):
    T, n = sum(lens) + tail, sum(lens)
    qkv, _ = inputs(lens, tail, nh, nkv, d, n + tail)
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    want, want_lse = reference_fwd(qkv, lens, nh, nkv, d)
    assert (o[n:] == 7).all() and (lse[:, n:] == 7).all()
    assert rel(o[:n], want) < tol(want.numel())
    assert float((lse[:, :n].double() - want_lse).abs().max()) < 2e-5
    single = torch.tensor([m == 1 for m in lens for _ in range(m)], device="cuda")  # a row that sees itself alone returns its value
    v = qkv[:n].view(n, nh + 2 * nkv, d)[:, nh + nkv:].repeat_interleave(nh // nkv, 1).reshape(n, -1)
    assert torch.equal(o[:n][single], v[single])


@pytest.mark.parametrize("lens,tail", DOCS)
@pytest.mark.parametrize("nh,nkv,d,rope", [(2, 1, 64, True), (4, 4, 64, False), (4, 2, 128, True), (3, 1, 128, False)])
def test_backward(lens, tail, nh, nkv, d, rope):
    T, n, longest = sum(lens) + tail, sum(lens), max(lens)
    qkv, do = inputs(lens, tail, nh, nkv, d, n + 2 * tail + nh)
    o, lse, bounds = run_fwd(qkv, lens, T, nh, nkv, d)
    o[n:], lse[:, n:] = float("nan"), float("nan")
    cos, sin = tables(longest, d) if rope else (None, None)
    got = run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, longest, cos, sin)
    want = reference_bwd(qkv, o, do, lens, nh, nkv, d, cos, sin)
    assert (got[n:] == 9).all()
    got = got[:n]
    q, k = nh * d, nkv * d
    alone = max(lens) == 1
    for name, a, b in (("dq", 0, q), ("dk", q, q + k), ("dv", q + k, q + 2 * k)):
        if alone and name != "dv":
            # dS = dO (v - o) = 0 exactly: o is the value itself; what is left are the fp32 sums' orders, d terms of up to 4 * 4
            assert float(got[:, a:b].abs().max()) < 1e-3
            continue
        assert rel(got[:, a:b], want[:, a:b]) < tol(want[:, a:b].numel()), name


@pytest.mark.parametrize("nh,nkv,d", [(8, 1, 64), (4, 2, 128)])
def test_gradient_against_differences(nh, nkv, d):
    """d(sum(o do)) along a random direction, by differences of the 64-bit definition, against the kernels' gradient."""
    lens = [50, 1, 200, 131]
    n = sum(lens)
    qkv, do = inputs(lens, 0, nh, nkv, d, 5)
    o, lse, bounds = run_fwd(qkv, lens, n, nh, nkv, d)
    got = run_bwd(qkv, o, do, lse, bounds, n, nh, nkv, d, max(lens)).double()
    g = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(3):
        v = torch.randn(qkv.shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-4
        f = lambda t: float((reference_fwd(t, lens, nh, nkv, d)[0] * do.double()).sum())  # noqa: E731
        slope = (f(qkv.double() + h * v) - f(qkv.double() - h * v)) / (2 * h)
        # the error of got is at most 3e-3 of its norm, and v is independent of it: 4 standard deviations
        assert abs(float((got * v).sum()) - slope) < 4 * 3e-3 * float(got.norm())


@pytest.mark.parametrize("d", [64, 128])
def test_one_document_is_causal_attention(d):
    from paper_2609_13645_b200 import binding as Bn
    nh, nkv, T = 4, 2, 777
    qkv, do = inputs([T], 0, nh, nkv, d, 3)
    o, lse, bounds = run_fwd(qkv, [T], T, nh, nkv, d)
    o2, lse2 = torch.empty_like(o), torch.empty(1, nh, T, device="cuda")
    Bn.k_attention_window_fwd(qkv, o2, lse2, 1, T, nh, nkv, d, T)
    # both are within 2.4e-3 of the definition, by roundings of their own
    assert rel(o, o2) < 5e-3 and float((lse - lse2[0]).abs().max()) < 4e-5
    got = run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, T)
    dq2 = torch.empty_like(qkv)
    scratch = torch.empty(Bn.attention_window_scratch_bytes(1, T, nh, nkv, d, T, 0), dtype=torch.uint8, device="cuda")
    Bn.k_attention_window_bwd(qkv, o2, do, lse2, dq2, scratch, 1, T, nh, nkv, d, T)
    assert rel(got, dq2) < 5e-3


@pytest.mark.parametrize("nh,nkv,d", [(6, 1, 64), (12, 12, 64), (16, 8, 128)])
def test_many_blocks(nh, nkv, d):
    """Thousands of rows: parts of key blocks, both block sizes of d = 64, several blocks a document; bit-identical twice."""
    g = np.random.RandomState(nh)
    lens = [int(m) for m in g.randint(0, 900, 12)] + [1500]
    tail, n = 77, sum(lens)
    qkv, do = inputs(lens, tail, nh, nkv, d, 11, garbage=float("inf"))
    o, lse, bounds = run_fwd(qkv, lens, n + tail, nh, nkv, d)
    want, want_lse = reference_fwd(qkv, lens, nh, nkv, d)
    assert rel(o[:n], want) < 3e-3 and float((lse[:, :n].double() - want_lse).abs().max()) < 2e-5
    cos, sin = tables(2000, d)
    got = run_bwd(qkv, o, do, lse, bounds, n + tail, nh, nkv, d, 2000, cos, sin)  # longest may be more than the longest is
    want = reference_bwd(qkv, o, do, lens, nh, nkv, d, cos, sin)
    for a, b in ((0, nh * d), (nh * d, (nh + nkv) * d), ((nh + nkv) * d, (nh + 2 * nkv) * d)):
        assert rel(got[:n, a:b], want[:, a:b]) < 3e-3
    assert (got[n:] == 9).all()
    o2, lse2, _ = run_fwd(qkv, lens, n + tail, nh, nkv, d)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert torch.equal(got, run_bwd(qkv, o, do, lse, bounds, n + tail, nh, nkv, d, 2000, cos, sin))


def test_dq_without_stored_scores():
    """Room for a document so long that dS^T of one kv head passes 4 GiB: dQ recomputes the scores."""
    from paper_2609_13645_b200 import binding as Bn
    nh, nkv, d, lens, tail = 64, 1, 64, [3000, 1, 2500, 60, 2600], 39  # 64 heads x 65 * 65 / 2 tiles of 32 KB
    T, n = sum(lens) + tail, sum(lens)
    assert Bn.attention_packed_scratch_bytes(T, nh, nkv, d, T) < 1 << 30
    qkv, do = inputs(lens, tail, nh, nkv, d, 21)
    o, lse, bounds = run_fwd(qkv, lens, T, nh, nkv, d)
    o[n:] = float("nan")
    cos, sin = tables(T, d)
    got = run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, T, cos, sin)
    want = reference_bwd(qkv, o, do, lens, nh, nkv, d, cos, sin)
    for a, b in ((0, nh * d), (nh * d, (nh + nkv) * d), ((nh + nkv) * d, (nh + 2 * nkv) * d)):
        assert rel(got[:n, a:b], want[:, a:b]) < 3e-3
    assert (got[n:] == 9).all()


def test_large_scores_and_equal_scores():
    """Rows whose softmax is one key, and rows that weigh all keys alike."""
    nh, nkv, d, lens = 2, 2, 64, [300, 40, 211]
    n = sum(lens)
    qkv, _ = inputs(lens, 0, nh, nkv, d, 2, qscale=300.0)
    o, lse, _ = run_fwd(qkv, lens, n, nh, nkv, d)
    want, want_lse = reference_fwd(qkv, lens, nh, nkv, d)
    # scores of up to 300 * 30: an fp32 score is off by up to 64 terms' roundings, 2^-24 * 64 of 9000 = 0.03, which changes the
    # weights of near ties by 3 %; those are few
    assert rel(o, want) < 3e-2 and float((lse.double() - want_lse).abs().max()) < 0.04
    qkv[:, :nh * d] = 0
    o, lse, _ = run_fwd(qkv, lens, n, nh, nkv, d)
    want, want_lse = reference_fwd(qkv, lens, nh, nkv, d)
    assert rel(o, want) < 3e-3 and float((lse.double() - want_lse).abs().max()) < 2e-5


def test_new_offsets_in_a_captured_call():
    """A captured batch is replayed with other documents in the same buffers, and with fewer rows."""
    from paper_2609_13645_b200 import binding as Bn
    nh, nkv, d, T = 4, 2, 64, 600
    first, second = [100, 250, 250], [30, 400, 0]
    qkv, do = inputs([T], 0, nh, nkv, d, 8)
    cu = offsets(first)
    bounds = torch.empty(3, T, dtype=torch.int32, device="cuda")
    o, lse, dqkv = torch.zeros(T, nh * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(nh, T, device="cuda"), torch.zeros_like(qkv)
    scratch = torch.empty(Bn.attention_packed_scratch_bytes(T, nh, nkv, d, 400), dtype=torch.uint8, device="cuda")

    def step():
        Bn.k_packed_bounds(cu, bounds, T, 400)
        Bn.k_attention_packed_fwd(qkv, o, lse, bounds, T, nh, nkv, d)
        Bn.k_attention_packed_bwd(qkv, o, do, lse, dqkv, bounds, scratch, T, nh, nkv, d, 400)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in (second, first):
        n = sum(lens)
        cu.copy_(offsets(lens))
        o.fill_(7.0), dqkv.fill_(9.0)
        graph.replay()
        Bn.k_status()
        want, _ = reference_fwd(qkv[:n], lens, nh, nkv, d)
        assert rel(o[:n], want) < 3e-3 and (o[n:] == 7).all()
        assert rel(dqkv[:n], reference_bwd(qkv[:n], o, do, lens, nh, nkv, d)) < 3e-3 and (dqkv[n:] == 9).all()


@pytest.mark.parametrize("cu", [[0, 5, 3, 10], [0, 4, 11], [1, 4, 10], [0, 9, 10], [-3, 4, 10]])
def test_offsets_that_are_refused_on_the_device(cu):
    """Descending, past the buffer, not from 0, a document over the limit of 6, negative: reported, everything stays in bounds, and the
    next status is clean."""
    from paper_2609_13645_b200 import binding as Bn
    T = 10
    bounds = torch.empty(3, T, dtype=torch.int32, device="cuda")
    Bn.k_packed_bounds(torch.tensor(cu, dtype=torch.int32, device="cuda"), bounds, T, 6)
    with pytest.raises(Bn.ForgeStepError) as e:
        Bn.k_status()
    assert e.value.status == Bn.FT_EINVAL
    Bn.k_status()
    b = bounds.cpu()
    assert (b[:2] >= 0).all() and (b[:2] <= T).all() and (b[2] >= 0).all() and (b[2] < T).all()


@pytest.mark.parametrize("nh,nkv,d,T", [(30, 15, 64, 6500), (24, 24, 64, 7900), (33, 11, 64, 5900), (34, 17, 64, 6500), (28, 28, 64, 7900), (39, 13, 64, 5900), (30, 15, 128, 6500), (24, 24, 128, 7900), (25, 5, 128, 7700)])
def test_two_tiles_a_block(nh, nkv, d, T):
    """Calls of many tiles an SM, whose blocks work on two tiles: heads that share K and V or have their own, odd numbers of
    them, an odd number of query blocks, documents from one row to most of the batch, rows behind them; bit-identical twice."""
    g = np.random.RandomState(T + nh)
    lens = [1, 0, 127, 129, 1, 2500] + [int(m) for m in g.randint(0, 400, 11)]
    tail = T - sum(lens)
    assert tail > 0 and (T + 127) // 128 * nh >= 1480
    n = sum(lens)
    qkv, _ = inputs(lens, tail, nh, nkv, d, 31)
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    for a in range(0, nh, nh // nkv):  # the reference by kv heads: its scores are many
        r = nh // nkv
        cols = [h * d + c for h in list(range(a, a + r)) + [nh + a // r, nh + nkv + a // r] for c in range(d)]
        want, want_lse = reference_fwd(qkv[:, cols], lens, r, 1, d)
        assert rel(o[:n, a * d:(a + r) * d], want) < 3e-3 and float((lse[a:a + r, :n].double() - want_lse).abs().max()) < 2e-5
    assert (o[n:] == 7).all() and (lse[:, n:] == 7).all()
    o2, lse2, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_large_scores_in_two_tiles_a_block():
    """References that move by hundreds, up and down, between a row's blocks."""
    nh, nkv, d, lens, T = 30, 15, 64, [3000, 700, 2600], 6500
    n = sum(lens)
    qkv, _ = inputs(lens, T - n, nh, nkv, d, 12)
    g = torch.Generator(device="cuda").manual_seed(3)
    qkv[:n, nh * d:(nh + nkv) * d] *= torch.exp2(torch.randint(-6, 7, (n, 1), generator=g, device="cuda").float()).bfloat16()  # keys of any size
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    cols = [h * d + c for h in (0, 1, nh, nh + nkv) for c in range(d)]
    want, want_lse = reference_fwd(qkv[:, cols], lens, 2, 1, d)
    # scores of up to 64 * 30: an fp32 score is off by up to 2^-24 * 64 of 2000 = 0.008, which moves near ties' weights by 1 %
    assert rel(o[:n, :2 * d], want) < 1e-2 and float((lse[:2, :n].double() - want_lse).abs().max()) < 0.01


def test_elements_past_32_bits():
    """A batch whose qkv has more than 2^31 elements: the last documents, which rows behind them follow."""
    from paper_2609_13645_b200 import binding as Bn
    nh, nkv, d, tail = 16, 8, 128, 77
    last = [300, 1, 700]
    lens = [1000] * 540 + last
    T, n = sum(lens) + tail, sum(lens)
    m = sum(last)
    assert (n - m) * (nh + 2 * nkv) * d > 2 ** 31
    qkv = torch.zeros(T, (nh + 2 * nkv) * d, dtype=torch.bfloat16, device="cuda")
    do = torch.zeros(T, nh * d, dtype=torch.bfloat16, device="cuda")
    qkv[n - m:], do[n - m:] = inputs(last, tail, nh, nkv, d, 5)
    o, lse, bounds = run_fwd(qkv, lens, T, nh, nkv, d)
    want, want_lse = reference_fwd(qkv[n - m:n], last, nh, nkv, d)
    assert rel(o[n - m:n], want) < 3e-3 and float((lse[:, n - m:n].double() - want_lse).abs().max()) < 2e-5
    assert not o[:n - m].any() and (o[n:] == 7).all() and (lse[:, n:] == 7).all()
    cos, sin = tables(1000, d)
    dqkv = run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, 1000, cos, sin)
    want = reference_bwd(qkv[n - m:n], o[n - m:n], do[n - m:n], last, nh, nkv, d, cos, sin)
    got = dqkv[n - m:n].view(m, -1, d)
    for a, b in ((0, nh), (nh, nh + nkv), (nh + nkv, nh + 2 * nkv)):
        assert rel(got[:, a:b], want.view(m, -1, d)[:, a:b]) < 3e-3
    assert not dqkv[:n - m].any() and (dqkv[n:] == 9).all()


def test_two_calls_on_two_streams():
    """Batches that are worked on at the same time, each with its own scratch, give the bits of batches one after the other."""
    from paper_2609_13645_b200 import binding as Bn
    shapes = [([700, 3, 900], 5, 4, 2, 128), ([128] * 9, 0, 6, 1, 64)]
    runs, streams = [], [torch.cuda.Stream() for _ in shapes]
    for k, (lens, tail, nh, nkv, d) in enumerate(shapes):
        T = sum(lens) + tail
        qkv, do = inputs(lens, tail, nh, nkv, d, k)
        o, lse, bounds = run_fwd(qkv, lens, T, nh, nkv, d)
        runs.append((qkv, do, o, lse, bounds, run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, max(lens)), T, nh, nkv, d, max(lens)))
    torch.cuda.synchronize()
    again = []
    for qkv, do, o, lse, bounds, dqkv, *shape in runs:
        scratch = torch.empty(Bn.attention_packed_scratch_bytes(*shape), dtype=torch.uint8, device="cuda")
        again.append((torch.full_like(o, 7.0), torch.full_like(lse, 7.0), torch.full_like(dqkv, 9.0), scratch))
    torch.cuda.synchronize()
    for _ in range(5):
        for (qkv, do, o, lse, bounds, dqkv, *shape), (o2, lse2, dqkv2, scratch), stream in zip(runs, again, streams):
            with torch.cuda.stream(stream):
                Bn.k_attention_packed_fwd(qkv, o2, lse2, bounds, *shape[:4])
                Bn.k_attention_packed_bwd(qkv, o2, do, lse2, dqkv2, bounds, scratch, *shape)
    torch.cuda.synchronize()
    Bn.k_status()
    for (qkv, do, o, lse, bounds, dqkv, *shape), (o2, lse2, dqkv2, scratch) in zip(runs, again):
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(dqkv, dqkv2)


@pytest.mark.parametrize("nh,nkv,d,rope", [(16, 8, 128, True), (12, 12, 64, False), (5, 5, 64, True), (16, 2, 128, False)])
@pytest.mark.parametrize("lens,tail", [([400, 1, 0, 77, 400, 400, 128, 128, 3, 390, 400, 400, 250, 400, 123], 600), ([128] * 30, 260), ([4100], 0), ([1], 4099)])
def test_tiles_in_order_of_length(nh, nkv, d, rope, lens, tail):
    """Calls of one to a few tiles an SM, which start with the longest: documents of many lengths and of one, tiles that nobody owns."""
    T, n = sum(lens) + tail, sum(lens)
    assert (T + 127) // 128 == 33
    qkv, do = inputs(lens, tail, nh, nkv, d, 77)
    o, lse, bounds = run_fwd(qkv, lens, T, nh, nkv, d)
    cos, sin = tables(max(lens), d) if rope else (None, None)
    dqkv = run_bwd(qkv, o, do, lse, bounds, T, nh, nkv, d, max(lens), cos, sin)
    assert (o[n:] == 7).all() and (lse[:, n:] == 7).all() and (dqkv[n:] == 9).all()
    r = nh // nkv
    for a in range(nkv):  # the reference by kv heads: its scores are many
        cols = [h * d + c for h in list(range(a * r, (a + 1) * r)) + [nh + a, nh + nkv + a] for c in range(d)]
        part, own = qkv[:, cols], slice(a * r * d, (a + 1) * r * d)
        want, want_lse = reference_fwd(part, lens, r, 1, d)
        assert rel(o[:n, own], want) < tol(want.numel()) and float((lse[a * r:(a + 1) * r, :n].double() - want_lse).abs().max()) < 2e-5
        if n == 1:
            continue  # differences that cancel to 0
        want = reference_bwd(part, o[:, own].contiguous(), do[:, own].contiguous(), lens, r, 1, d, cos, sin)
        got = dqkv[:n, cols].view(n, r + 2, d)
        for k in (slice(0, r), slice(r, r + 1), slice(r + 1, r + 2)):
            assert rel(got[:, k], want.view(n, r + 2, d)[:, k]) < 3e-3


def test_large_scores_in_two_tiles_of_64():
    """References that move by hundreds, up and down, between a row's blocks."""
    nh, nkv, d, lens, T = 34, 17, 64, [3000, 700, 2600], 6500
    n = sum(lens)
    qkv, _ = inputs(lens, T - n, nh, nkv, d, 12)
    g = torch.Generator(device="cuda").manual_seed(3)
    qkv[:n, nh * d:(nh + nkv) * d] *= torch.exp2(torch.randint(-6, 7, (n, 1), generator=g, device="cuda").float()).bfloat16()  # keys of any size
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    cols = [h * d + c for h in (0, 1, nh, nh + nkv) for c in range(d)]
    want, want_lse = reference_fwd(qkv[:, cols], lens, 2, 1, d)
    # as in test_large_scores_in_two_tiles_a_block
    assert rel(o[:n, :2 * d], want) < 1e-2 and float((lse[:2, :n].double() - want_lse).abs().max()) < 0.01


@pytest.mark.parametrize("T,nh,nkv,d", [(10000, 5, 5, 64), (20001, 6, 3, 64), (24100, 5, 1, 64), (30100, 4, 2, 128), (16300, 7, 1, 128)])
def test_orders_of_many_tiles(T, nh, nkv, d):
    """Hundreds of tiles of a head, by themselves, two heads at a time and two neighbours at a time, in the order of their lengths."""
    g = np.random.RandomState(T)
    lens = [0, 1, 1500, 128, 128]
    while sum(lens) < T - 700:
        lens.append(int(g.randint(0, 600)))
    n = sum(lens)
    qkv, _ = inputs(lens, T - n, nh, nkv, d, 3)
    o, lse, _ = run_fwd(qkv, lens, T, nh, nkv, d)
    r = nh // nkv
    for a in range(nkv):  # the reference by kv heads: its scores are many
        cols = [h * d + c for h in list(range(a * r, (a + 1) * r)) + [nh + a, nh + nkv + a] for c in range(d)]
        want, want_lse = reference_fwd(qkv[:, cols], lens, r, 1, d)
        err = (o[:n, a * r * d:(a + 1) * r * d].double() - want).view(n, r, d).norm(dim=2)
        assert float(err.max()) < 2.0 ** -6 * float(want.view(n, r, d).norm(dim=2).max())  # no row is another's: two roundings of 2^-8 each
        assert rel(o[:n, a * r * d:(a + 1) * r * d], want) < 3e-3 and float((lse[a * r:(a + 1) * r, :n].double() - want_lse).abs().max()) < 2e-5
    assert (o[n:] == 7).all() and (lse[:, n:] == 7).all()
