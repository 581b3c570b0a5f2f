"""AdamW with moments in 8 bits where the definition's codes and scales are hard to reach in fp32: runs with several elements that may be
the greatest, moments whose terms cancel.

Codes and scales are those of the definition in 64 bits, bit for bit.  The parameter: an fp32 first moment is off by up to 8 roundings
(2^-24 each) of the magnitudes of its terms T = beta1 |m| + (1 - beta1) |g|; the update by 17 of its own: 3 in m times its correction, 8 in the
denominator, 4 in its inverse (2^-22), 2 in products and sums; and the result by one: with room,
bound 2^-24 |p| + lr (2^-19 |update| + 2^-19 T / den / (1 - beta1^t) + 2^-23 decay |p|)."""
import numpy as np
import pytest
import torch

from .test_adamw_gpu import randoms, runs, steps_of, unpack

pytestmark = pytest.mark.gpu

LR = float(np.float32(1e-2))
FLT_MAX = float(np.finfo(np.float32).max)


def fresh(n):
    return torch.zeros(n, device="cuda").to(torch.float8_e4m3fn), torch.zeros(-(-n // 256), device="cuda")


def tensors(m, ms, v, vs, g, p=None):
    """Lists of one tensor: codes, scales, gradients and parameters."""
    n = g.numel()
    p = torch.linspace(-1.0, 1.0, n, device="cuda") if p is None else p
    return dict(p=[p], g=[g], m=[m], v=[v], ms=[ms], vs=[vs])


def step(t, beta1, beta2, eps, count, seed, clip=1.0, decay=0.0):
    from paper_2609_13645_b200 import binding as Bn
    old = {k: [x.clone() for x in v] for k, v in t.items()}
    plan = Bn.AdamWPlan(t["p"], t["g"], t["m"], t["v"], weight_decay=decay, m_scales=t["ms"], v_scales=t["vs"])
    Bn.k_adamw(plan, LR, beta1, beta2, eps, torch.tensor([count], device="cuda"), grad_scale=torch.tensor([clip], device="cuda"), seed=seed)
    return old, t


def check(old, new, beta1, beta2, eps, count, seed, clip=1.0, decay=0.0):
    """Against the definition, its operations in its order."""
    base = 0
    clip = float(np.float32(clip))
    for k, p in enumerate(old["p"]):
        n = p.numel()
        g = old["g"][k].double() * clip
        m0, r0 = unpack(old["m"][k], old["ms"][k]), unpack(old["v"][k], old["vs"][k])
        m, v = beta1 * m0 + (1 - beta1) * g, beta2 * (r0 * r0) + (1 - beta2) * g * g
        den = (v / (1 - beta2 ** count)).sqrt() + float(np.float32(eps))
        update = (m / (1 - beta1 ** count)) / den
        want = p.double() - LR * (update + decay * p.double())
        terms = (beta1 * m0.abs() + (1 - beta1) * g.abs()) / (1 - beta1 ** count) / den
        bound = 2.0 ** -24 * want.abs() + LR * (2.0 ** -19 * (update.abs() + terms) + 2.0 ** -23 * decay * p.double().abs()) + 1e-45
        ok = ((new["p"][k].double() - want).abs() <= bound) | (want.isnan() & new["p"][k].isnan()) | (want.float() == new["p"][k])
        assert ok.all(), (k, want[~ok][:4], new["p"][k][~ok][:4])
        u = randoms(seed, count, base, n)
        base += -(-n // 256) * 256
        for name, x, low, col in (("m", m, 0.0, 0), ("v", v.sqrt(), 2.0 ** -9, 1)):
            top = runs(x.abs()).amax(1)
            beyond, none = top > FLT_MAX, top < 2.0 ** -100
            unit = top * (1.0 / 448.0)
            want_scale = torch.where(beyond, np.inf, torch.where(none, 0.0, unit)).float()
            assert torch.equal(new[name + "s"][k], want_scale), (k, name)
            per = lambda t: t.repeat_interleave(256)[:n]  # noqa: E731
            count_, size = steps_of(x, per(unit))
            q = ((count_ + u[:, col]).floor() * size).clamp(max=448.0)
            q = torch.where(x != 0, q.clamp(min=low), q)
            q = torch.where(per(none), 0.0, torch.where(per(beyond), 1.0, q))
            got = new[name][k].double()
            bad = got.abs() != q
            assert not bad.any(), (k, name, int(bad.sum()), x[bad][:4], got[bad][:4], q[bad][:4], per(unit)[bad][:4])
            assert ((got == 0) | per(beyond) | (torch.sign(got) == torch.sign(x))).all()


BETAS = [(0.9, 0.95), (0.95, 0.999), (0.5, 0.9)]


@pytest.mark.parametrize("beta1,beta2", BETAS)
@pytest.mark.parametrize("apart", [1, 2, 8, 64])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_elements_that_may_each_be_the_greatest(beta1, beta2, apart, grad):
    """Greatest elements a few last places apart: in the eight that a thread holds, in different threads, all of a run; equal ones."""
    n = 256 * 600
    g = torch.Generator(device="cuda").manual_seed(apart)
    one = torch.randn(n // 256, 1, generator=g, device="cuda")
    near = (one.view(torch.int32) + torch.randint(0, apart + 1, (n // 256, 256), generator=g, device="cuda", dtype=torch.int32)).view(torch.float32)
    x = near * torch.rand(n // 256, 256, generator=g, device="cuda") * 0.5  # the others are at most half as great
    run = torch.arange(n // 256, device="cuda")[:, None]
    where = torch.arange(256, device="cuda")[None]
    first = torch.randint(0, 256, (n // 256, 1), generator=g, device="cuda")
    kind = run % 3  # a thread's eight, two threads, the whole run
    tops = torch.where(kind == 0, where // 8 == first // 8, torch.where(kind == 1, where % 128 == first % 128, where >= 0))
    x = torch.where(tops, near, x).reshape(-1).to(grad)
    t = tensors(*fresh(n), *fresh(n), x)
    for count in (1, 2, 3):
        old, new = step(t, beta1, beta2, 1e-8, count, 3)
        check(old, new, beta1, beta2, 1e-8, count, 3)
    x.zero_()  # the codes alone: many equal ones
    for count in (4, 5):
        old, new = step(t, beta1, beta2, 1e-8, count, 3)
        check(old, new, beta1, beta2, 1e-8, count, 3)


def cancelling(n, beta1, places, seed, alone, m_scale=0.37 / 448):
    """Codes of m and gradients a few last places (`places`, at most) from those that cancel them.  alone: every run has one such element
    and nothing else."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.randint(0, 127, (n,), generator=g, device="cuda") + 128 * torch.randint(0, 2, (n,), generator=g, device="cuda")
    v = torch.randint(0, 127, (n,), generator=g, device="cuda")
    if alone:
        keep = torch.arange(n, device="cuda") % 256 == (torch.arange(n, device="cuda") // 256 * 37) % 256
        m, v = torch.where(keep, m, 0), torch.where(keep, v, 0)
    ms = torch.rand(-(-n // 256), generator=g, device="cuda") * m_scale + m_scale / 4
    m = m.to(torch.uint8).view(torch.float8_e4m3fn)
    grad = (-(beta1 / (1 - beta1)) * unpack(m, ms)).float()
    off = torch.randint(-places, places + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.where(grad != 0, (grad.view(torch.int32) + off).view(torch.float32), grad)
    return m, ms, v.to(torch.uint8).view(torch.float8_e4m3fn), ms.clone(), grad


@pytest.mark.parametrize("beta1,beta2", BETAS)
@pytest.mark.parametrize("places", [0, 3, 40, 600, 100000])
@pytest.mark.parametrize("alone", [False, True])
def test_moments_whose_terms_cancel(beta1, beta2, places, alone):
    """First moments next to 0 by cancellation, the greatest of their runs among them: no NaN codes, and the definition's."""
    n = 256 * 400
    t = tensors(*cancelling(n, beta1, places, places + 1, alone))
    old, new = step(t, beta1, beta2, 1e-8, 7, 11)
    assert ((new["m"][0].view(torch.uint8) & 127) < 127).all()
    check(old, new, beta1, beta2, 1e-8, 7, 11)
    for count in (8, 9):  # and what they leave behind, under other gradients
        t["g"][0].mul_(-1e-3)
        old, new = step(t, beta1, beta2, 1e-8, count, 11)
        check(old, new, beta1, beta2, 1e-8, count, 11)


def test_single_elements_whose_terms_cancel():
    """Tensors of one element: the greatest of its run is the one that cancels."""
    m, ms, v, vs, g = cancelling(256 * 300, 0.9, 600, 5, True)
    keep = (torch.arange(256 * 300, device="cuda") % 256 == (torch.arange(256 * 300, device="cuda") // 256 * 37) % 256).nonzero().view(-1)
    part = lambda x: [x[i:i + 1].clone() for i in keep.tolist()]  # noqa: E731
    t = dict(p=[torch.ones(1, device="cuda") for _ in keep], g=part(g), m=part(m.view(torch.uint8)), v=part(v.view(torch.uint8)),
             ms=[x.clone() for x in ms.split(1)], vs=[x.clone() for x in vs.split(1)])
    t["m"], t["v"] = ([x.view(torch.float8_e4m3fn) for x in t[name]] for name in "mv")
    for count in (3, 4):
        old, new = step(t, 0.9, 0.95, 1e-8, count, 2)
        assert all(torch.isfinite(x).all() for x in new["p"])
        check(old, new, 0.9, 0.95, 1e-8, count, 2)
