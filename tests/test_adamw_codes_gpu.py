"""AdamW with moments in 8 bits where the definition's codes and scales are hard to reach in fp32: runs with several elements that may be
the greatest, moments whose terms cancel, elements beyond what fp32's squares hold.

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
LOW, HIGH = 2.0 ** -78, 2.0 ** 47  # roots of v: within 2^-79 to 2^48, whose borders are fp32's


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
        low, high = (v > 0) & (v.sqrt() < LOW), (v.sqrt() > HIGH) | (g.abs() > HIGH)  # out of range: as if v were 0; unspecified
        ok |= high | (low & ((new["p"][k].double() - p.double() + LR * (m / (1 - beta1 ** count) / eps + decay * p.double())).abs() <= bound))
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
            bad = (got.abs() != q) & ~((name == "v") & (x < LOW) & (got == 0))
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


SIZES = [2.0 ** e for e in (-140, -110, -101, -99, -80, -77, -70, -63, -58, -50, -40, -20, 0, 20, 34, 44, 47, 50, 60, 64, 90, 120)]


@pytest.mark.parametrize("eps", [2.0 ** -64, 1e-8])
@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.95), (0.9, 0.999), (0.0, 0.5)])
@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("n", [256 * 40, 1, 777])
def test_gradients_of_any_size(eps, beta1, beta2, mixed, n):
    """Gradients whose squares pass fp32 on either side, from fresh moments and from those that the steps before left: codes and scales are
    the definition's.  mixed: of all sizes in one run, and some 0."""
    g = torch.Generator(device="cuda").manual_seed(n)
    for k, size in enumerate(SIZES):
        t = tensors(*fresh(n), *fresh(n), torch.zeros(n, device="cuda"))
        for count in (1, 2, 3):
            x = torch.randn(n, generator=g, device="cuda")
            if mixed:
                x = x * 2.0 ** -(40.0 * torch.rand(n, generator=g, device="cuda")) * (torch.rand(n, generator=g, device="cuda") < 0.8)
            t["g"][0].copy_(x.double() * size)
            old, new = step(t, beta1, beta2, eps, count, k)
            check(old, new, beta1, beta2, eps, count, k)


@pytest.mark.parametrize("clip", [0.0, 2.0 ** -64, 2.0 ** -16, -1.0, 65536.0])
@pytest.mark.parametrize("size", [1.0, 1e-30, 1e-20])
def test_scales_of_gradients_of_any_size(clip, size):
    n = 2000
    g = torch.Generator(device="cuda").manual_seed(7)
    t = tensors(*fresh(n), *fresh(n), torch.zeros(n, device="cuda"))
    for count in (1, 2, 3):
        t["g"][0].copy_(torch.randn(n, generator=g, device="cuda") * size)
        t["g"][0][::7] = 0
        old, new = step(t, 0.9, 0.95, 1e-8, count, 1, clip=clip, decay=0.1)
        check(old, new, 0.9, 0.95, 1e-8, count, 1, clip=clip, decay=0.1)


def test_moments_that_die_out():
    """No gradient for thousands of steps: v and m go to 0 run by run, through the range where fp32 does not hold the squares."""
    n = 256 * 8
    g = torch.Generator(device="cuda").manual_seed(1)
    code = torch.randint(0, 127, (n,), generator=g, device="cuda").to(torch.uint8).view(torch.float8_e4m3fn)
    for e in range(-103, -50, 2):
        scale = torch.full((n // 256,), 2.0 ** e / 448, device="cuda") * torch.linspace(0.5, 1.5, n // 256, device="cuda")
        t = tensors(code.clone(), scale.clone(), code.clone(), scale.clone(), torch.zeros(n, device="cuda"))
        for count in (2000, 2001):
            old, new = step(t, 0.9, 0.95, 1e-8, count, 5)
            check(old, new, 0.9, 0.95, 1e-8, count, 5)


def test_an_epsilon_of_nothing_is_refused():
    """With moments in 8 bits; beside it roots that fp32 does not hold would matter."""
    from paper_2609_13645_b200 import binding as Bn
    t = tensors(*fresh(10), *fresh(10), torch.ones(10, device="cuda"))
    plan = Bn.AdamWPlan(t["p"], t["g"], t["m"], t["v"], m_scales=t["ms"], v_scales=t["vs"])
    for eps in (0.0, 2.0 ** -65):
        with pytest.raises(Bn.ForgeStepError) as e:
            Bn.k_adamw(plan, LR, 0.9, 0.95, eps, torch.tensor([1], device="cuda"))
        assert e.value.status == Bn.FT_EINVAL
    wide = Bn.AdamWPlan(t["p"], t["g"], [torch.zeros(10, device="cuda")], [torch.zeros(10, device="cuda")])
    Bn.k_adamw(wide, LR, 0.9, 0.95, 0.0, torch.tensor([1], device="cuda"))  # as in the model's update
