"""Windowed attention element by element: every output against the 64-bit definition within a bound of its own, made of the
roundings on the way to it, so that a single wrong element shows.

u = 2^-8 is half a step of bf16.  With |.| element by element and s = q k / sqrt(d), the bounds count
  scores       products of 16 terms a step, of each of which at most 2^-22 of the running magnitude is lost, d / 16 <= 8 steps:
               2^-19 sum |q||k| / sqrt(d); exp2 2^-22, its argument and the log-sum-exp in fp32: 2^-22 |lse| + 2^-20.
               Their sum E is the relative error of a weight before it is rounded.
  o            weights rounded once (u), in the numerator and, on edges of the mask, in the sum too; o rounded:
               |o - ref| <= (expm1(E) + u) P|v| + (max E + 2 u) |ref|
  d_v          (expm1(E) + u) P^T|do| + u |ref|
  dS           P (dP - delta): dP and delta in fp32, D = 2^-19 |do||v| + 2^-20 |do||o|; rounded:
               e = P ((expm1(E) + u) |dP - delta| + (1 + expm1(E) + u) D)
  d_q, d_k     e|k| and e^T|q|, the rotation of the bounds with |cos| and |sin|, one rounding
and for every sum of n products n / 16 + 8 steps of 2^-22 of the terms' magnitude.  (1 + u) covers products of two of these.
"""
import math

import pytest
import torch

from tests.test_attention_window_gpu import _bwd, _fwd, _heads, _inputs, _mask, _reference_fwd, _rope

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def _sum_error(n):
    return (n / 16 + 8) * 2.0 ** -22


def _weights(qkv, B, S, nh, nkv, d, window, sinks):
    """Of every head: P, the relative error of its elements, the log-sum-exp, and q, k, v."""
    q, k, v = _heads(qkv, B, S, nh, nkv, d)
    seen = _mask(S, window, sinks)
    s = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.softmax(s, -1)
    e = 2.0 ** -19 * (q.abs() @ k.abs().transpose(-1, -2)) / math.sqrt(d) + 2.0 ** -22 * lse.abs()[..., None] + 2.0 ** -20
    return p, e.masked_fill(~seen, 0.0), lse, q, k, v


def _out(t):  # [B, nh, S, d] -> [B * S, nh * d]
    B, n, S, d = t.shape
    return t.transpose(1, 2).reshape(B * S, n * d)


def _assert_within(name, got, ref, bound):
    over = (got.double() - ref).abs() - bound * (1 + U) - 1e-37
    worst = int(over.argmax())
    assert float(over.max()) <= 0, (name, worst, float(got.flatten()[worst]), float(ref.flatten()[worst]), float(bound.flatten()[worst]))
    # the bound means something: for most elements that are not near zero it is a small part of the value
    assert float((bound > ref.abs()).double().mean()) < 0.5, name


def _check_forward(qkv, B, S, nh, nkv, d, window, sinks):
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    p, e, lse_ref, _, _, v = _weights(qkv, B, S, nh, nkv, d, window, sinks)
    ref, top = p @ v, e.amax(-1, keepdim=True)
    bound = (p * (e.expm1() + U + _sum_error(S))) @ v.abs() + (top.expm1() + 2 * U + _sum_error(S)) * ref.abs()
    _assert_within("o", o, _out(ref), _out(bound))
    assert ((lse.double() - lse_ref).abs() <= top[..., 0] + 2.0 ** -20 * (1 + lse_ref.abs())).all()


def _check_backward(qkv, do, B, S, nh, nkv, d, window, sinks, rope):
    o_ref, lse_ref = _reference_fwd(qkv, B, S, nh, nkv, d, window, sinks)
    o, lse = o_ref.bfloat16(), lse_ref.float()
    cos, sin = _rope(S, d) if rope else (None, None)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks, cos, sin)
    p, e, _, q, k, v = _weights(qkv, B, S, nh, nkv, d, window, sinks)
    rows = lambda t: t.double().view(B, S, nh, d).transpose(1, 2)  # noqa: E731
    group = lambda t: t.view(B, nkv, nh // nkv, S, d).sum(2)  # noqa: E731
    do_, o_, T = rows(do), rows(o), (-1, -2)
    diff = do_ @ v.transpose(*T) - (do_ * o_).sum(-1, keepdim=True)
    err = 2.0 ** -19 * (do_.abs() @ v.abs().transpose(*T)) + 2.0 ** -20 * (do_.abs() * o_.abs()).sum(-1, keepdim=True)
    rel, scale, n_k = e.expm1() + U, 1.0 / math.sqrt(d), S * (nh // nkv)
    ds = p * diff
    e_ds = p * (rel * diff.abs() + (1 + rel) * err)
    dq, dk, dv = scale * (ds @ k), scale * group(ds.transpose(*T) @ q), group(p.transpose(*T) @ do_)
    b_dq = scale * ((e_ds + _sum_error(S) * ds.abs()) @ k.abs())
    b_dk = scale * group((e_ds + _sum_error(n_k) * ds.abs()).transpose(*T) @ q.abs())
    b_dv = group((p * (rel + _sum_error(n_k))).transpose(*T) @ do_.abs())
    if rope:
        c, s = cos.double(), sin.double()

        def back(t, c, s):
            a, b = t.chunk(2, -1)
            return torch.cat([a * c + b * s, b * c - a * s], -1)

        def back_bound(t, m):  # of a bound: every term counts, and its two products and one sum in fp32
            t = t + 2.0 ** -22 * m
            a, b = t.chunk(2, -1)
            return torch.cat([a * c.abs() + b * s.abs(), b * c.abs() + a * s.abs()], -1)
        b_dq, b_dk = back_bound(b_dq, dq.abs()), back_bound(b_dk, dk.abs())
        dq, dk = back(dq, c, s), back(dk, c, s)
    hq, hkv = nh * d, nkv * d
    parts = [("d_v", got[:, hq + hkv:], dv, b_dv)]
    if S > 1 and (window > 1 or sinks > 0):  # of one key nothing is left of d_q and d_k but roundings: no value to compare with
        parts += [("d_q", got[:, :hq], dq, b_dq), ("d_k", got[:, hq:hq + hkv], dk, b_dk)]
    for name, a, ref, bound in parts:
        _assert_within(name, a, _out(ref), _out(bound + U * ref.abs()))


# lengths within and beyond a tile, windows and sinks that end inside blocks, one kv head for all, both block sizes of heads of 64,
# key blocks divided between thread blocks, a window over everything
SHAPES = [(1, 1, 2, 1, 64, 1, 0), (1, 129, 2, 1, 128, 1, 1), (1, 300, 4, 2, 64, 128, 0), (1, 321, 4, 1, 128, 100, 70), (2, 512, 4, 2, 128, 64, 4),
          (1, 777, 7, 1, 128, 130, 129), (3, 413, 6, 1, 64, 33, 7), (1, 500, 2, 1, 128, 900, 900), (1, 1300, 2, 2, 64, 256, 640),
          (2, 1531, 20, 4, 64, 300, 0), (1, 1500, 32, 1, 64, 190, 133), (1, 2049, 16, 8, 128, 512, 4)]


@pytest.mark.parametrize("B,S,nh,nkv,d,window,sinks", SHAPES)
def test_forward(B, S, nh, nkv, d, window, sinks):
    qkv, _ = _inputs(B, S, nh, nkv, d, seed=S + 5)
    _check_forward(qkv, B, S, nh, nkv, d, window, sinks)


@pytest.mark.parametrize("B,S,nh,nkv,d,window,sinks", SHAPES)
@pytest.mark.parametrize("rope", [False, True])
def test_backward(B, S, nh, nkv, d, window, sinks, rope):
    qkv, do = _inputs(B, S, nh, nkv, d, seed=S + 6)
    _check_backward(qkv, do, B, S, nh, nkv, d, window, sinks, rope)


@pytest.mark.parametrize("qscale", [6.0, 40.0])
@pytest.mark.parametrize("d", [64, 128])
def test_large_scores(qscale, d):
    B, S, nh, nkv, window, sinks = 1, 700, 2, 1, 150, 3
    qkv, do = _inputs(B, S, nh, nkv, d, seed=3, qscale=qscale)
    _check_forward(qkv, B, S, nh, nkv, d, window, sinks)
    _check_backward(qkv, do, B, S, nh, nkv, d, window, sinks, False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("loud", [3e2, 3e4])
def test_masked_scores_that_overflow_when_taken_for_visible_ones(d, loud):
    """Keys that the first rows alone see have scores up to 1e5 times those of the others: as weights of the later rows, which
    do not see them, they pass fp32.  The later rows' gradients are those of the definition all the same."""
    B, S, nh, nkv, window, sinks = 1, 400, 2, 2, 64, 0
    qkv, do = _inputs(B, S, nh, nkv, d, seed=5)
    k = qkv.view(S, 3, nh, d)[:, 1]
    k[:100] *= loud
    late = qkv.view(S, 3, nh, d)[100:].reshape(S - 100, -1).contiguous()  # the rows from 163 on see none of the first 100 keys
    o, lse = _fwd(qkv, B, S, nh, nkv, d, window, sinks)
    got = _bwd(qkv, o, do, lse, B, S, nh, nkv, d, window, sinks)
    assert torch.isfinite(got.float()).all()
    # the same rows as a sequence of their own, whose first 63 see fewer keys: everything from 163 on is as in the whole one
    o1, lse1 = _fwd(late, B, S - 100, nh, nkv, d, window, sinks)
    _check_forward(late, B, S - 100, nh, nkv, d, window, sinks)
    _check_backward(late, do[100:].contiguous(), B, S - 100, nh, nkv, d, window, sinks, False)
    got1 = _bwd(late, o1, do[100:].contiguous(), lse1, B, S - 100, nh, nkv, d, window, sinks)
    n = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())  # noqa: E731
    # queries from 163 on and keys from 163 on; two results whose every element has the errors above, in other blocks: twice
    # the 3e-3 of a tensor's 2-norm
    hq = nh * d
    assert n(o[163:], o1[63:]) < 6e-3 and n(got[163:, :hq], got1[63:, :hq]) < 6e-3 and n(got[163:, hq:], got1[63:, hq:]) < 6e-3


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_masked_keys_may_hold_anything_in_the_forward_pass(d, bad):
    """Keys (not values) that a query does not see change no bit of its row, in the warps and blocks where others see them too."""
    S, nh, nkv, window, sinks = 400, 2, 2, 64, 3
    qkv, _ = _inputs(1, S, nh, nkv, d, seed=12)
    o, lse = _fwd(qkv, 1, S, nh, nkv, d, window, sinks)
    k = qkv.view(S, 3, nh, d)[:, 1]
    k[40:50] = bad
    k[200:203, :, ::3] = bad
    o1, lse1 = _fwd(qkv, 1, S, nh, nkv, d, window, sinks)
    clear = torch.ones(S, dtype=torch.bool, device="cuda")
    clear[40:49 + window] = clear[200:202 + window] = False  # the queries that see one of them
    assert torch.equal(o1[clear], o[clear]) and torch.equal(lse1[..., clear], lse[..., clear])
