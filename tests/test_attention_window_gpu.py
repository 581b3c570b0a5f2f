"""Windowed attention with sink keys, forward and backward, against a plain 64-bit implementation of its definition.

Tolerances, relative in the 2-norm of a tensor unless said otherwise.  One rounding to bf16 is off by at most half a step,
u = 2^-8 of the value; over many values, whose distance to the next step is uniform, by 2^-8 / sqrt(3) times 0.72 (the mean
over a binade) = 1.7e-3 in the 2-norm, and independent roundings add in squares.
  o        P is rounded (its error averages like the sum it enters) and o is:         sqrt(2) 1.7e-3 = 2.4e-3, taken as 3e-3
  lse      fp32 scores (d terms of |s| <= 30, d 2^-24 relative) and exp2 / log2 (2^-22): absolute <= 2e-5
  d_v      P rounded, d_v rounded; d_q, d_k: dS rounded, result rounded: the same 2.4e-3, taken as 3e-3.  delta is formed
           from the o that the reference is given too.
Tensors of under 1000 elements are too few for the mean and are held to 2 u = 2^-7.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _inputs(B, S, nh, nkv, d, seed, qscale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(B * S, (nh + 2 * nkv) * d, device="cuda", generator=g)
    qkv[:, :nh * d] *= qscale
    do = torch.randn(B * S, nh * d, device="cuda", generator=g)
    return qkv.bfloat16(), do.bfloat16()


def _mask(S, window, sinks):
    i, j = torch.arange(S, device="cuda")[:, None], torch.arange(S, device="cuda")[None, :]
    return (j <= i) & ((i - j < window) | (j < sinks))


def _heads(qkv, B, S, nh, nkv, d):
    """fp64 q [B, nh, S, d], k and v expanded to the query heads."""
    t = qkv.double().view(B, S, nh + 2 * nkv, d).transpose(1, 2)
    r = nh // nkv
    return t[:, :nh], t[:, nh:nh + nkv].repeat_interleave(r, 1), t[:, nh + nkv:].repeat_interleave(r, 1)


def _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks):
    q, k, v = _heads(qkv, B, S, nh, nkv, d)
    s = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(~_mask(S, window, sinks), -math.inf)
    return (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(B * S, nh * d), torch.logsumexp(s, -1)


def _reference_bwd(qkv, o, do, B, S, nh, nkv, d, window, sinks, cos=None, sin=None):
    q, k, v = _heads(qkv, B, S, nh, nkv, d)
    rows = lambda t: t.double().view(B, S, nh, d).transpose(1, 2)  # noqa: E731
    s = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(~_mask(S, window, sinks), -math.inf)
    p = torch.softmax(s, -1)
    ds = p * (rows(do) @ v.transpose(-1, -2) - (rows(do) * rows(o)).sum(-1, keepdim=True)) / math.sqrt(d)
    group = lambda t: t.view(B, nkv, nh // nkv, S, d).sum(2)  # noqa: E731
    dq, dk, dv = ds @ k, group(ds.transpose(-1, -2) @ q), group(p.transpose(-1, -2) @ rows(do))
    if cos is not None:
        def back(t):
            a, b = t.chunk(2, -1)
            return torch.cat([a * cos.double() + b * sin.double(), b * cos.double() - a * sin.double()], -1)
        dq, dk = back(dq), back(dk)
    return torch.cat([dq, dk, dv], 1).transpose(1, 2).reshape(B * S, -1)


def _rel(a, b):
    return float((a.double() - b).norm() / b.norm().clamp_min(1e-300))


def _tol(t):
    return 3e-3 if t.numel() >= 1000 else 2.0 ** -7


def _fwd(qkv, B, S, nh, nkv, d, window, sinks):
    from paper_2609_13645_b200 import binding as Bn
    o = torch.full((B * S, nh * d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, nh, S), 7.0, device="cuda")
    Bn.k_attention_window_fwd(qkv, o, lse, B, S, nh, nkv, d, window, sinks)
    return o, lse


def _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks, cos=None, sin=None, poison=float("nan")):
    from paper_2609_13645_b200 import binding as Bn
    n = Bn.attention_window_scratch_bytes(B, S, nh, nkv, d, window, sinks)
    # contents on entry must not matter: NaN everywhere
    scratch = torch.full(((n + 3) // 4,), poison, device="cuda").view(torch.uint8)
    dqkv = torch.full_like(qkv, 7.0)
    Bn.k_attention_window_bwd(qkv, o, do, lse, dqkv, scratch, B, S, nh, nkv, d, window, sinks, cos=cos, sin=sin)
    return dqkv


def _rope(S, d):
    ang = torch.arange(S, dtype=torch.float64, device="cuda")[:, None] * 1e4 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    return ang.cos().float(), ang.sin().float()


# one token, less than a tile, window of one key, windows that end inside tiles and at their edges, sinks inside the window,
# sinks over several blocks, window and sinks past the sequence, one kv head for all query heads, tiles past the end
SHAPES = [
    (1, 1, 2, 1, 64, 1, 0), (2, 7, 4, 2, 128, 3, 1), (1, 64, 2, 2, 64, 1, 0), (1, 65, 2, 2, 128, 64, 2), (2, 128, 4, 4, 64, 32, 4),
    (1, 129, 2, 1, 128, 1, 1), (1, 300, 4, 2, 64, 128, 0), (1, 321, 4, 1, 128, 100, 70), (2, 512, 4, 2, 128, 64, 4),
    (1, 640, 2, 2, 64, 65, 200), (1, 777, 7, 1, 128, 130, 129), (3, 413, 6, 1, 64, 33, 7), (1, 1024, 4, 4, 64, 1024, 0),
    (1, 500, 2, 1, 128, 900, 900), (1, 1300, 2, 2, 64, 256, 640), (2, 1000, 8, 2, 128, 191, 5),
]


@pytest.mark.parametrize("B,S,nh,nkv,d,window,sinks", SHAPES)
def test_forward_matches_the_definition(B, S, nh, nkv, d, window, sinks):
    qkv, _ = _inputs(B, S, nh, nkv, d, seed=S)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    o_ref, lse_ref = _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks)
    assert _rel(o, o_ref) < _tol(o)
    assert float((lse.double() - lse_ref).abs().max()) < 2e-5


@pytest.mark.parametrize("B,S,nh,nkv,d,window,sinks", SHAPES)
@pytest.mark.parametrize("rope", [False, True])
def test_backward_matches_the_definition(B, S, nh, nkv, d, window, sinks, rope):
    qkv, do = _inputs(B, S, nh, nkv, d, seed=S + 1)
    o_ref, lse_ref = _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks)
    o, lse = o_ref.bfloat16(), lse_ref.float()
    cos, sin = _rope(S, d) if rope else (None, None)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks, cos, sin)
    ref = _reference_bwd(qkv, o, do, B, S, nh, nkv, d, window, sinks, cos, sin)
    hq, hkv = nh * d, nkv * d
    assert _rel(got[:, hq + hkv:], ref[:, hq + hkv:]) < _tol(ref[:, hq + hkv:])
    if S > 1:  # a single key's softmax is constant: d_q and d_k are 0 up to the rounding of delta
        if window > 1 or sinks > 0:
            assert _rel(got[:, :hq], ref[:, :hq]) < _tol(ref[:, :hq])
            assert _rel(got[:, hq:hq + hkv], ref[:, hq:hq + hkv]) < _tol(ref[:, hq:hq + hkv])
    assert torch.isfinite(got.float()).all()


def test_a_row_that_sees_one_key_returns_its_value():
    """window 1: the only weight is 1 whatever the score, so the rounding of P must cancel."""
    B, S, nh, nkv, d = 2, 200, 4, 2, 64
    qkv, do = _inputs(B, S, nh, nkv, d, seed=8, qscale=3.0)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, 1, 0)
    v = qkv.view(B * S, nh + 2 * nkv, d)[:, nh + nkv:].repeat_interleave(nh // nkv, 1).reshape(B * S, nh * d)
    assert torch.equal(o, v)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, 1, 0)
    ref = do.double().view(B * S, nkv, nh // nkv, d).sum(2).reshape(B * S, nkv * d)
    assert _rel(got[:, (nh + nkv) * d:], ref) < 3e-3


@pytest.mark.parametrize("qscale", [6.0, 40.0])
def test_large_scores_and_references_that_jump_between_blocks(qscale):
    """Rows whose maximum moves by hundreds between blocks, and whose oldest block shows them nothing at all."""
    B, S, nh, nkv, d, window, sinks = 1, 700, 2, 1, 64, 150, 3
    qkv, do = _inputs(B, S, nh, nkv, d, seed=3, qscale=qscale)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    o_ref, lse_ref = _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks)
    assert _rel(o, o_ref) < 3e-3
    assert float((lse.double() - lse_ref).abs().max()) < 2e-6 * float(lse_ref.abs().max()) + 2e-5
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
    assert torch.isfinite(got.float()).all()


def test_masked_scores_may_overflow():
    """Keys outside the mask with products beyond fp32's exponent range after the softmax reference is taken away."""
    B, S, nh, nkv, d, window, sinks = 1, 400, 2, 2, 64, 64, 0
    qkv, do = _inputs(B, S, nh, nkv, d, seed=5)
    k = qkv.view(S, 3, nh, d)[:, 1]
    k[:100] *= 3e4  # seen by the first rows only
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    o_ref, lse_ref = _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks)
    late = slice(200, S)
    assert _rel(o[late], o_ref[late]) < 3e-3 and torch.isfinite(o.float()).all()
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
    assert torch.isfinite(got.float()).all()


def test_a_window_over_the_whole_sequence_is_causal_attention():
    """The same definition; the two kernels differ in whether P enters the normalising sum rounded (2.4e-3 from the definition
    each, as above, and the same way for most elements)."""
    from paper_2609_13645_b200 import binding as Bn
    B, S, nh, nkv, d = 2, 700, 4, 2, 128
    qkv, do = _inputs(B, S, nh, nkv, d, seed=11)
    want_o, want_lse = torch.empty(B * S, nh * d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, nh, S, device="cuda")
    Bn.k_attention_fwd(qkv, want_o, want_lse, B, S, nh, nkv, d)
    for window, sinks in ((S, 0), (2 ** 31 - 1, 5), (10 * S, 2 ** 31 - 1)):
        o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
        assert _rel(o, want_o.double()) < 3e-3
        assert float((lse - want_lse).abs().max()) < 1e-5
        got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
        delta, want = torch.empty(B, nh, S, device="cuda"), torch.empty_like(qkv)
        Bn.k_attention_bwd(qkv, o, do, lse, delta, want, B, S, nh, nkv, d)
        assert _rel(got, want.double()) < 3e-3


def test_gradients_agree_with_differences_of_the_forward_pass():
    """(f(x + e) - f(x - e)) / 2 against the gradient, along random directions, with f in 64 bits."""
    B, S, nh, nkv, d, window, sinks = 1, 200, 4, 2, 64, 40, 3
    qkv, do = _inputs(B, S, nh, nkv, d, seed=21)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks).double()
    g = torch.Generator(device="cuda").manual_seed(1)
    f = lambda t: (_reference_fwd(t, B, S, nh, nkv, d, window, sinks)[0] * do.double()).sum()  # noqa: E731
    for _ in range(4):
        v = torch.randn(qkv.shape, device="cuda", dtype=torch.float64, generator=g)
        eps = 1e-5
        diff = float((f(qkv.double() + eps * v) - f(qkv.double() - eps * v)) / (2 * eps))
        dot = float((got * v).sum())
        # the error of the dot product is the gradient's relative error (< 3e-3) times |v . g| ~ |g|: v is a unit direction
        # scaled by sqrt(n), so 5 standard deviations are 5 * 3e-3 * |g|
        assert abs(dot - diff) < 5 * 3e-3 * float(got.norm())


@pytest.mark.parametrize("B,S,nh,nkv,d,window,sinks", [(4, 2048, 16, 8, 128, 512, 4), (8, 1024, 12, 12, 64, 256, 0), (1, 8192, 8, 1, 128, 384, 130)])
def test_bit_identical_from_run_to_run(B, S, nh, nkv, d, window, sinks):
    qkv, do = _inputs(B, S, nh, nkv, d, seed=9)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    first = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
    for poison in (float("nan"), 1e30):
        o2, lse2 = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
        assert torch.equal(_bwd(qkv, o2, do, lse2, B, S, nh, nkv, d, window, sinks, poison=poison), first)
    # and right, on sampled rows: a query's row of d_q against the definition
    q, k, v = _heads(qkv[:S], 1, S, nh, nkv, d)
    for i in (0, 127, 128, S // 2 + 3, S - 1):
        seen = _mask(S, window, sinks)[i]
        s = (q[0, :, i:i + 1] @ k[0].transpose(-1, -2) / math.sqrt(d)).masked_fill(~seen, -math.inf)
        p = torch.softmax(s, -1)
        doi, oi = do[i].double().view(nh, 1, d), o[i].double().view(nh, 1, d)
        dq = (p * (doi @ v[0].transpose(-1, -2) - (doi * oi).sum(-1, keepdim=True)) / math.sqrt(d)) @ k[0]
        if i > 0:
            assert _rel(first[i, :nh * d], dq.reshape(-1)) < 1e-2


def test_no_element_outside_the_outputs_is_written():
    """Outputs inside larger buffers: what lies before and behind them stays."""
    from paper_2609_13645_b200 import binding as Bn
    B, S, nh, nkv, d, window, sinks = 2, 201, 4, 2, 64, 50, 2
    qkv, do = _inputs(B, S, nh, nkv, d, seed=4)
    pad = 4096
    big_o = torch.full((B * S * nh * d + 2 * pad,), 3.0, dtype=torch.bfloat16, device="cuda")
    big_l = torch.full((B * S * nh + 2 * pad,), 3.0, device="cuda")
    big_g = torch.full((qkv.numel() + 2 * pad,), 3.0, dtype=torch.bfloat16, device="cuda")
    n = Bn.attention_window_scratch_bytes(B, S, nh, nkv, d, window, sinks)
    big_s = torch.full((n + 2 * pad,), 3, dtype=torch.uint8, device="cuda")
    o, lse, dqkv = big_o[pad:-pad], big_l[pad:-pad], big_g[pad:-pad]
    Bn.k_attention_window_fwd(qkv, o, lse, B, S, nh, nkv, d, window, sinks)
    Bn.k_attention_window_bwd(qkv, o, do, lse, dqkv, big_s[pad:-pad], B, S, nh, nkv, d, window, sinks)
    for t in (big_o, big_l, big_g, big_s):
        assert (t[:pad] == 3).all() and (t[-pad:] == 3).all()
    assert torch.equal(dqkv.view(qkv.shape), _bwd(qkv, o.view(B * S, -1), do, lse, B, S, nh, nkv, d, window, sinks))


def test_captured_and_replayed_on_another_stream():
    from paper_2609_13645_b200 import binding as Bn
    B, S, nh, nkv, d, window, sinks = 1, 600, 4, 1, 64, 100, 4
    qkv, do = _inputs(B, S, nh, nkv, d, seed=6)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    want = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
    o2, lse2, got = torch.empty_like(o), torch.empty_like(lse), torch.empty_like(qkv)
    scratch = torch.empty(Bn.attention_window_scratch_bytes(B, S, nh, nkv, d, window, sinks), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Bn.k_attention_window_fwd(qkv, o2, lse2, B, S, nh, nkv, d, window, sinks)
        Bn.k_attention_window_bwd(qkv, o2, do, lse2, got, scratch, B, S, nh, nkv, d, window, sinks)
    for _ in range(2):
        got.zero_()
        o2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o2, o) and torch.equal(got, want)
    from ctypes import c_void_p
    L = Bn.lib()
    L.ft_k_status.argtypes = [c_void_p]
    assert L.ft_k_status(c_void_p(torch.cuda.current_stream().cuda_stream)) == Bn.FT_OK


def _check_backward_by_heads(B, S, nh, nkv, d, window, sinks, seed, heads_at_once, rope=True):
    """The backward pass against the definition, a few query heads at a time (the 64-bit score matrices of all do not fit)."""
    qkv, do = _inputs(B, S, nh, nkv, d, seed=seed)
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    cos, sin = _rope(S, d) if rope else (None, None)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks, cos, sin)
    t = qkv.view(B, S, nh + 2 * nkv, d)
    n_rep, w = nh // nkv, min(heads_at_once, nh // nkv)
    ref = torch.zeros(B, S, nh + 2 * nkv, d, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h0 in range(0, nh, w):
            kv = h0 // n_rep
            sub = torch.cat([t[b, :, h0:h0 + w], t[b, :, nh + kv:nh + kv + 1], t[b, :, nh + nkv + kv:nh + nkv + kv + 1]], 1)
            cut = lambda x: x.view(B, S, nh, d)[b, :, h0:h0 + w].reshape(S, w * d)  # noqa: E731
            r = _reference_bwd(sub.reshape(S, -1), cut(o), cut(do), 1, S, w, 1, d, window, sinks, cos, sin).view(S, w + 2, d)
            ref[b, :, h0:h0 + w] = r[:, :w]
            ref[b, :, nh + kv] += r[:, w]  # rotating back is linear: the sum of the heads' parts
            ref[b, :, nh + nkv + kv] += r[:, w + 1]
    got = got.view(B, S, nh + 2 * nkv, d)
    for part in (slice(0, nh), slice(nh, nh + nkv), slice(nh + nkv, nh + 2 * nkv)):
        if window == 1 and sinks == 0 and part.start < nh + nkv:
            continue  # d_q and d_k are 0 up to the rounding of delta
        assert _rel(got[:, :, part], ref[:, :, part]) < 3e-3


# heads of 64 in launches of many blocks, where the streamed blocks are half as long: odd lengths, sinks over several blocks,
# blocks split between CTAs, one block, a window of one key, the whole sequence
@pytest.mark.parametrize("B,S,nh,nkv,window,sinks", [
    (2, 1531, 20, 4, 300, 0), (1, 1500, 32, 1, 190, 133), (4, 449, 64, 64, 1, 0), (2, 700, 40, 8, 700, 0), (40, 70, 24, 24, 20, 2),
    (2, 1300, 36, 36, 129, 65), (1, 2049, 64, 2, 64, 300)])
def test_backward_of_many_heads_of_64(B, S, nh, nkv, window, sinks):
    _check_backward_by_heads(B, S, nh, nkv, 64, window, sinks, seed=S, heads_at_once=64)


# dS^T of one kv head's queries is over a third of what is kept at a time (two rounds, of two heads and one), and over all of
# it (the queries' gradients recompute the scores), with and without sink blocks outside the window
@pytest.mark.parametrize("S,nh,nkv,d,window,sinks", [
    (4200, 36, 3, 64, 4150, 3), (4200, 36, 3, 128, 4150, 0), (8400, 64, 1, 64, 2000, 130), (8400, 64, 1, 128, 2000, 1)])
def test_backward_of_scores_beyond_the_scratch(S, nh, nkv, d, window, sinks):
    _check_backward_by_heads(1, S, nh, nkv, d, window, sinks, seed=7, heads_at_once=4)


def test_two_calls_at_once_with_scratch_of_their_own():
    shapes = [(1, 1531, 6, 1, 64, 333, 7), (2, 700, 4, 2, 128, 190, 3)]
    ins = [_inputs(*s[:5], seed=i) for i, s in enumerate(shapes)]
    alone = []
    for (qkv, do), s in zip(ins, shapes):
        o, lse = _fwd(qkv, *s)
        alone.append((o, _bwd(qkv, o, do, lse, *s)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in shapes]
    for _ in range(5):
        got = []
        for st, (qkv, do), s in zip(streams, ins, shapes):
            with torch.cuda.stream(st):
                o, lse = _fwd(qkv, *s)
                got.append((o, _bwd(qkv, o, do, lse, *s)))
        torch.cuda.synchronize()
        for (o, g), (o1, g1) in zip(got, alone):
            assert torch.equal(o, o1) and torch.equal(g, g1)
