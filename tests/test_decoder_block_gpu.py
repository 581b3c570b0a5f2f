"""The decoder-block operators together, as a training step of a pre-norm block would call them, with the framework's GEMM:

    n = layernorm(x);  qkv = n Wqkv^T;  a = windowed attention;  z = a Wo^T;  y = x + dropout(z)
    dz = dropout(dy);  da = dz Wo;  dWo = dz^T a;  dqkv = attention backward;  dn = dqkv Wqkv;  dWqkv = dqkv^T n
    dx, dgain, dbias = layernorm backward of dn, plus dy along the residual

against the same block in 64 bits (its own gradients from the formulas of torch's automatic differentiation).

Tolerances (relative, 2-norm): one rounding of a tensor to bf16 is 1.7e-3 (2^-8 half a step at most, / sqrt(3), mean over a
binade) and independent ones add in squares.  On the way to y's branch: n, qkv, P, a, z, y; the longest way back, to dgain and
dx: those of the forward pass as they enter the backward one (5), then dz, da, dS, dqkv, dn and the result (6).  A softmax
passes an error of its scores on multiplied by the scores' size (|s| of a few), the one step that enlarges: counted as 4
roundings more (16 in squares).  sqrt(6 + 16) 1.7e-3 = 8e-3 forwards, sqrt(11 + 2 16) 1.7e-3 = 1.1e-2 backwards: 1e-2 and 1.5e-2.
"""
import math

import pytest
import torch

from tests.test_dropout_gpu import keep_mask

pytestmark = pytest.mark.gpu

P, SEED, SITE, EPS = 0.1, 1234567, 2, 1e-5


class Block:
    """Buffers and the calls of one block; `run` enqueues the forward and the backward pass and allocates nothing."""

    def __init__(self, B, S, nh, nkv, d, h, window, sinks, seed=0):
        from paper_2609_13645_b200 import binding as Bn
        self.Bn, self.shape, self.h = Bn, (B, S, nh, nkv, d, window, sinks), h
        T, hq, nq = B * S, nh * d, (nh + 2 * nkv) * d
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, k=1.0, m=0.0: (torch.randn(*s, device="cuda", generator=g) * k + m).bfloat16()  # noqa: E731
        new = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.x, self.dy = rnd(T, h), rnd(T, h)
        self.gain, self.bias = rnd(h, k=0.2, m=1.0), rnd(h, k=0.1)
        self.wqkv, self.wo = rnd(nq, h, k=h ** -0.5), rnd(h, hq, k=hq ** -0.5)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.n, self.qkv, self.a, self.z, self.y = new(T, h), new(T, nq), new(T, hq), new(T, h), new(T, h)
        self.mean, self.rstd, self.lse = new(T, dt=f32), new(T, dt=f32), new(B, nh, S, dt=f32)
        self.dz, self.da, self.dqkv, self.dn, self.dx = new(T, h), new(T, hq), new(T, nq), new(T, h), new(T, h)
        self.dwo, self.dwqkv = new(h, hq, dt=f32), new(nq, h, dt=f32)
        self.dgain, self.dbias = new(h, dt=f32), new(h, dt=f32)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        # the two backward calls follow one another on one stream, so they may share their scratch
        self.scratch = new(max(Bn.attention_window_scratch_bytes(*self.shape), Bn.layernorm_scratch_bytes(T, h)), dt=torch.uint8)

    def run(self):
        Bn, (B, S, nh, nkv, d, window, sinks), h = self.Bn, self.shape, self.h
        T, hq, nq = B * S, nh * d, (nh + 2 * nkv) * d
        Bn.k_layernorm_fwd(self.x, self.gain, self.bias, self.n, self.mean, self.rstd, EPS)
        Bn.k_gemm(self.n, 0, self.wqkv, 0, self.qkv, 0, T, nq, h, self.err)
        Bn.k_attention_window_fwd(self.qkv, self.a, self.lse, B, S, nh, nkv, d, window, sinks)
        Bn.k_gemm(self.a, 0, self.wo, 0, self.z, 0, T, h, hq, self.err)
        Bn.k_dropout_add(self.z, self.x, self.y, P, SEED, SITE, step=self.step)
        Bn.k_dropout_add(self.dy, None, self.dz, P, SEED, SITE, step=self.step)
        Bn.k_gemm(self.dz, 0, self.wo, 1, self.da, 0, T, hq, h, self.err)
        Bn.k_gemm(self.dz, 1, self.a, 1, self.dwo, 2, h, hq, T, self.err)
        Bn.k_attention_window_bwd(self.qkv, self.a, self.da, self.lse, self.dqkv, self.scratch, B, S, nh, nkv, d, window, sinks)
        Bn.k_gemm(self.dqkv, 0, self.wqkv, 1, self.dn, 0, T, h, nq, self.err)
        Bn.k_gemm(self.dqkv, 1, self.n, 1, self.dwqkv, 2, nq, h, T, self.err)
        Bn.k_layernorm_bwd(self.dn, self.x, self.mean, self.rstd, self.gain, self.dy, self.dx, self.dgain, self.dbias, self.scratch)

    def outputs(self):
        return {k: getattr(self, k).clone() for k in ("y", "dx", "dgain", "dbias", "dwqkv", "dwo")}

    def reference(self, step):
        B, S, nh, nkv, d, window, sinks = self.shape
        T = B * S
        leaf = {k: getattr(self, k).double().requires_grad_() for k in ("x", "gain", "bias", "wqkv", "wo")}
        n = torch.nn.functional.layer_norm(leaf["x"], (self.h,), leaf["gain"], leaf["bias"], EPS)
        t = (n @ leaf["wqkv"].T).view(B, S, nh + 2 * nkv, d).transpose(1, 2)
        q, k, v = t[:, :nh], t[:, nh:nh + nkv].repeat_interleave(nh // nkv, 1), t[:, nh + nkv:].repeat_interleave(nh // nkv, 1)
        i, j = torch.arange(S, device="cuda")[:, None], torch.arange(S, device="cuda")[None, :]
        s = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(~((j <= i) & ((i - j < window) | (j < sinks))), -math.inf)
        z = (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(T, nh * d) @ leaf["wo"].T
        keep, thr = keep_mask(T, self.h, P, SEED, SITE, step)
        y = leaf["x"] + z * keep / (1.0 - thr / 65536.0)
        (y * self.dy.double()).sum().backward()
        return {"y": y.detach(), "dx": leaf["x"].grad, "dgain": leaf["gain"].grad, "dbias": leaf["bias"].grad,
                "dwqkv": leaf["wqkv"].grad, "dwo": leaf["wo"].grad}


def _assert_close(got, ref):
    for name, t in got.items():
        r = ref[name]
        e = float((t.double() - r).norm() / r.norm())
        assert e < (1e-2 if name == "y" else 1.5e-2), (name, e)


@pytest.mark.parametrize("B,S,nh,nkv,d,h,window,sinks", [
    (2, 256, 4, 2, 64, 256, 48, 4), (1, 411, 4, 1, 128, 328, 100, 0), (3, 128, 8, 8, 64, 512, 128, 0)])
def test_a_block_forwards_and_backwards(B, S, nh, nkv, d, h, window, sinks):
    blk = Block(B, S, nh, nkv, d, h, window, sinks)
    blk.run()
    _assert_close(blk.outputs(), blk.reference(0))
    assert int(blk.err.item()) == 0


def test_a_captured_block_draws_a_new_mask_at_every_step():
    """One graph of the whole block; the step counter on the device moves between replays.  Each replay equals the eager block
    of that step bit for bit, and the definition with that step's mask."""
    blk = Block(2, 192, 4, 2, 64, 256, 50, 3, seed=5)
    eager = []
    for s in (0, 1, 7):
        blk.step.fill_(s)
        blk.run()
        eager.append(blk.outputs())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.run()
    for s, want in zip((0, 1, 7), eager):
        blk.step.fill_(s)
        for t in (blk.y, blk.dx, blk.dgain, blk.dbias, blk.dwqkv, blk.dwo):
            t.zero_()
        graph.replay()
        got = blk.outputs()
        for name in got:
            assert torch.equal(got[name], want[name]), (s, name)
        _assert_close(got, blk.reference(s))
    assert not torch.equal(eager[0]["y"], eager[1]["y"])
    assert int(blk.err.item()) == 0
