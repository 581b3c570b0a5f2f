"""Packed batches for the tests: inputs with garbage behind the last document, and a plain 64-bit attention inside documents."""
import math

import torch


def offsets(lens):
    return torch.tensor([0] + list(torch.tensor(lens, dtype=torch.int64).cumsum(0)) if lens else [0], dtype=torch.int32, device="cuda")


def inputs(lens, tail, nh, nkv, d, seed, garbage=float("nan"), qscale=1.0):
    """qkv and do of sum(lens) + tail rows; the tail holds `garbage`."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, T = sum(lens), sum(lens) + tail
    qkv = torch.randn(T, (nh + 2 * nkv) * d, device="cuda", generator=g)
    qkv[:, :nh * d] *= qscale
    do = torch.randn(T, nh * d, device="cuda", generator=g)
    qkv[n:], do[n:] = garbage, garbage
    return qkv.bfloat16(), do.bfloat16()


def heads(qkv, nh, nkv, d):
    """fp64 q [nh, T, d], k and v expanded to the query heads."""
    t = qkv.double().view(-1, nh + 2 * nkv, d).transpose(0, 1)
    r = nh // nkv
    return t[:nh], t[nh:nh + nkv].repeat_interleave(r, 0), t[nh + nkv:].repeat_interleave(r, 0)


def reference_fwd(qkv, lens, nh, nkv, d):
    """o [rows, nh d] and lse [nh, rows] of the rows inside documents."""
    q, k, v = heads(qkv, nh, nkv, d)
    n = sum(lens)
    o, lse = torch.zeros(nh, n, d, dtype=torch.float64, device="cuda"), torch.zeros(nh, n, dtype=torch.float64, device="cuda")
    at = 0
    for m in lens:
        s = q[:, at:at + m] @ k[:, at:at + m].transpose(1, 2) / math.sqrt(d)
        s = s.masked_fill(torch.ones(m, m, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        if m:
            o[:, at:at + m], lse[:, at:at + m] = torch.softmax(s, -1) @ v[:, at:at + m], torch.logsumexp(s, -1)
        at += m
    return o.transpose(0, 1).reshape(n, nh * d), lse


def reference_bwd(qkv, o, do, lens, nh, nkv, d, cos=None, sin=None):
    """dqkv of the rows inside documents, from the formulas; delta from the o that the kernels are given."""
    q, k, v = heads(qkv, nh, nkv, d)
    n, r = sum(lens), nh // nkv
    per = lambda t: t[:n].double().view(n, nh, d).transpose(0, 1)  # noqa: E731
    od, dod = per(o), per(do)
    dq, dk, dv = (torch.zeros(nh, n, d, dtype=torch.float64, device="cuda") for _ in range(3))
    at = 0
    for m in lens:
        a, b = at, at + m
        s = q[:, a:b] @ k[:, a:b].transpose(1, 2) / math.sqrt(d)
        s = s.masked_fill(torch.ones(m, m, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        p = torch.softmax(s, -1) if m else s
        ds = p * (dod[:, a:b] @ v[:, a:b].transpose(1, 2) - (dod[:, a:b] * od[:, a:b]).sum(-1, keepdim=True)) / math.sqrt(d)
        dq[:, a:b], dk[:, a:b], dv[:, a:b] = ds @ k[:, a:b], ds.transpose(1, 2) @ q[:, a:b], p.transpose(1, 2) @ dod[:, a:b]
        if cos is not None:
            c, s_ = cos[:m].double(), sin[:m].double()
            for t in (dq, dk):
                x, y = t[:, a:b, :d // 2].clone(), t[:, a:b, d // 2:].clone()
                t[:, a:b, :d // 2], t[:, a:b, d // 2:] = x * c + y * s_, y * c - x * s_
        at = b
    fold = lambda t: t.view(nkv, r, n, d).sum(1)  # noqa: E731
    return torch.cat([dq, fold(dk), fold(dv)]).transpose(0, 1).reshape(n, -1)


def tables(span, d):
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(span, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-2.0 * i / d)
    return angle.cos().float(), angle.sin().float()


def rel(a, b):
    n = float(b.double().norm())
    return float((a.double() - b.double()).norm()) / n if n else float(a.double().norm())
