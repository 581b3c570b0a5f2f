"""The operators for packed documents together, as a train step uses them: a causal attention block over a packed batch (LayerNorm,
projection, rotation at the documents' positions, attention, output projection with residual) forward and backward, and the
AdamW step of its parameters; against 64-bit autograd of the same, eager and captured."""
import math

import pytest
import torch

from .packed_util import offsets, rel

pytestmark = pytest.mark.gpu

H, NH, NKV, D, SPAN = 256, 4, 2, 64, 512
EPS, LR, B1, B2, ADAM_EPS, DECAY = 1e-5, 1e-2, 0.9, 0.95, 1e-8, 0.1
W = (NH + 2 * NKV) * D


class Block:
    """Parameters, buffers and the calls of one step; T rows, documents given by offsets on the device."""

    def __init__(self, T, seed, bits):
        from paper_2609_13645_b200 import binding as Bn
        self.Bn, self.T = Bn, T
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.masters = [1 + 0.1 * rand(H), 0.1 * rand(H), rand(W, H) / math.sqrt(H), rand(H, NH * D) / math.sqrt(NH * D)]
        bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.weights = [m.bfloat16() for m in self.masters]
        self.grads = [torch.zeros_like(m) for m in self.masters]
        self.x, self.dy = rand(T, H).bfloat16(), rand(T, H).bfloat16()
        self.h, self.qkv, self.o, self.y = bf(T, H), bf(T, W), bf(T, NH * D), bf(T, H)
        self.do, self.dqkv, self.dh, self.dx = bf(T, NH * D), bf(T, W), bf(T, H), bf(T, H)
        self.mean, self.rstd, self.lse = (torch.zeros(n, device="cuda") for n in (T, T, NH * T))
        self.bounds = torch.empty(3, T, dtype=torch.int32, device="cuda")
        self.cos, self.sin = torch.empty(SPAN, D // 2, device="cuda"), torch.empty(SPAN, D // 2, device="cuda")
        Bn.k_rotary_tables(self.cos, self.sin, 10000.0)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.scratch, self.ln_scratch = byte(Bn.attention_packed_scratch_bytes(T, NH, NKV, D, SPAN)), byte(Bn.layernorm_scratch_bytes(T, H))
        self.step, n = torch.zeros(1, dtype=torch.int64, device="cuda"), [m.numel() for m in self.masters]
        kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
        self.m, self.v = ([torch.zeros(k, device="cuda").to(kind) for k in n] for _ in range(2))
        runs = [torch.zeros(-(-k // 256), device="cuda") for k in n] if bits == 8 else None
        flat = lambda ts: [t.view(-1) for t in ts]  # noqa: E731
        self.plan = Bn.AdamWPlan(flat(self.masters), flat(self.grads), self.m, self.v, weight_decay=[0.0, 0.0, DECAY, DECAY], m_scales=runs,
                                 v_scales=[t.clone() for t in runs] if runs else None, copies=flat(self.weights))

    def run(self, cu):
        B, T = self.Bn, self.T
        gain, beta, wqkv, wo = self.weights
        B.k_packed_bounds(cu, self.bounds, T, SPAN)
        B.k_layernorm_fwd(self.x, gain, beta, self.h, self.mean, self.rstd, EPS)
        B.k_gemm(self.h, 0, wqkv, 0, self.qkv, 0, T, W, H, self.err)
        turned = self.qkv[:, :(NH + NKV) * D]
        B.k_rotary(turned, turned, self.cos, self.sin, NH + NKV, D, positions=self.bounds[2])
        B.k_attention_packed_fwd(self.qkv, self.o, self.lse, self.bounds, T, NH, NKV, D)
        B.k_gemm(self.o, 0, wo, 0, self.y, 1, T, H, NH * D, self.err, resid=self.x)
        # backward of sum(y dy)
        B.k_gemm(self.dy, 1, self.o, 1, self.grads[3], 2, H, NH * D, T, self.err)
        B.k_gemm(self.dy, 0, wo, 1, self.do, 0, T, NH * D, H, self.err)
        B.k_attention_packed_bwd(self.qkv, self.o, self.do, self.lse, self.dqkv, self.bounds, self.scratch, T, NH, NKV, D, SPAN, cos=self.cos, sin=self.sin)
        B.k_gemm(self.dqkv, 1, self.h, 1, self.grads[2], 2, W, H, T, self.err)
        B.k_gemm(self.dqkv, 0, wqkv, 1, self.dh, 0, T, H, W, self.err)
        B.k_layernorm_bwd(self.dh, self.x, self.mean, self.rstd, gain, self.dy, self.dx, self.grads[0], self.grads[1], self.ln_scratch)
        self.step += 1
        B.k_adamw(self.plan, LR, B1, B2, ADAM_EPS, self.step, seed=1)


def reference(block, lens, x):
    """y, dx and the parameters' gradients by autograd in 64 bits, from the weights the block holds now."""
    p = [w.double().requires_grad_() for w in block.weights]
    n = sum(lens)
    x = x[:n].double().requires_grad_()
    h = torch.nn.functional.layer_norm(x, (H,), p[0], p[1], EPS)
    t = (h @ p[2].T).view(n, NH + 2 * NKV, D).transpose(0, 1)
    pos = torch.cat([torch.arange(m, device="cuda") for m in lens])
    c, s = block.cos.double()[pos], block.sin.double()[pos]
    a, b = t[:NH + NKV, :, :D // 2], t[:NH + NKV, :, D // 2:]
    qk = torch.cat([a * c - b * s, b * c + a * s], -1)
    doc = torch.cat([torch.full((m,), i, device="cuda") for i, m in enumerate(lens)])
    seen = (doc[:, None] == doc[None, :]) & (torch.arange(n, device="cuda")[:, None] >= torch.arange(n, device="cuda")[None, :])
    r = NH // NKV
    k, v = qk[NH:].repeat_interleave(r, 0), t[NH + NKV:].repeat_interleave(r, 0)
    w = torch.softmax((qk[:NH] @ k.transpose(1, 2) / math.sqrt(D)).masked_fill(~seen, -math.inf), -1)
    y = x + (w @ v).transpose(0, 1).reshape(n, -1) @ p[3].T
    (y * block.dy[:n].double()).sum().backward()
    return y.detach(), x.grad, [q.grad for q in p]


def check(block, lens, before, ref):
    n = sum(lens)
    y, dx, grads = ref
    # a chain of bf16 tensors (h, qkv, rotated qkv, o, y and their gradients): every one adds its rounding of 1.7e-3 to what it
    # carries; eight of them in squares are 5e-3, taken as 8e-3; sums over rows of products carry the same
    assert rel(block.y[:n], y) < 8e-3 and rel(block.dx[:n], dx) < 8e-3
    for got, want in zip(block.grads, grads):
        assert rel(got, want) < 8e-3
    for k, (old, new) in enumerate(zip(before, block.masters)):  # AdamW from the gradients the kernels left, first step: m_hat = g
        g = block.grads[k].double()
        want = old.double() - LR * (g / (g.abs() + ADAM_EPS) + (DECAY if k > 1 else 0.0) * old.double())
        assert float((new.double() - want).abs().max()) < 1e-6
        assert torch.equal(block.weights[k], new.bfloat16())
    assert int(block.err.item()) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_one_step(bits):
    lens, T = [100, 0, 1, 250, 129, 32], 512
    block = Block(T, 3, bits)
    before = [m.clone() for m in block.masters]
    ref = reference(block, lens, block.x)
    block.run(offsets(lens))
    block.Bn.k_status()
    check(block, lens, before, ref)


def test_captured_steps_follow_the_batch_and_repeat_the_eager_bits():
    from paper_2609_13645_b200 import binding as Bn
    T = 512
    batches = [[512], [100, 0, 1, 250, 129, 32], [8] * 64, [300, 100, 112]]
    eager, block = Block(T, 5, 8), Block(T, 5, 8)
    cu = torch.zeros(65, dtype=torch.int32, device="cuda")

    def load(lens):  # documents behind the last one are empty
        o = offsets(lens)
        cu.fill_(int(o[-1]))
        cu[:o.numel()] = o
    load(batches[0])
    eager.run(cu)
    block.run(cu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.run(cu)
    for lens in batches[1:]:
        load(lens)
        eager.run(cu)
        graph.replay()
        Bn.k_status()
        for a, b in zip(eager.masters + eager.weights + eager.grads + [eager.y, eager.dx], block.masters + block.weights + block.grads + [block.y, block.dx]):
            assert torch.equal(a, b)
    assert int(block.step) == int(eager.step) == len(batches)
