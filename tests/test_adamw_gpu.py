"""AdamW over many tensors against its definition in 64 bits, moments in 32 and in 8 bits.

fp32: m, v and p are a few operations each, every one off by 2^-24, the root and the quotient of the update by 2^-22 each:
m and v within 2^-22 of the sum of their terms' magnitudes, p within 2^-24 |p| + lr (2^-20 |update| + 2^-22 decay |p|).  bf16
parameters add one rounding (2^-8 |p|).
8 bits: codes and scales are those of the definition in 64 bits; the tests' operations are ordered as the definition's are."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = [1, 7, 255, 256, 257, 0, 2048, 5000, 3, 40000]
B1, B2, EPS, LR = (0.9, 0.95, 1e-8, float(np.float32(1e-2)))


def mix(z):
    z = z + np.uint64(0x9E3779B97F4A7C15)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def randoms(seed, step, base, n):
    """[n, 2] numbers in [0, 1) of the elements from `base` (a multiple of 256) on."""
    with np.errstate(over="ignore"):
        key = mix(mix(np.array([seed], dtype=np.uint64)) ^ np.array([step * 0xA24BAED4963EE407 & (1 << 64) - 1], dtype=np.uint64))
        word = mix(key ^ (np.arange(base // 2, base // 2 + (n + 1) // 2, dtype=np.uint64) * np.uint64(0x8CB92BA72F3D8DD7)))
    part = [(word >> np.uint64(16 * k)) & np.uint64(0xFFFF) for k in range(4)]
    u = np.stack([np.stack([part[0], part[2]], 1).reshape(-1), np.stack([part[1], part[3]], 1).reshape(-1)], 1)[:n]
    return torch.from_numpy(u.astype(np.float64) / 65536.0).cuda()


def runs(t):
    return torch.nn.functional.pad(t, (0, -t.numel() % 256)).view(-1, 256)


def unpack(codes, scale):
    return (runs(codes.double()) * scale.double()[:, None]).view(-1)[:codes.numel()]


def steps_of(x, scale):
    """|x| / scale in steps of the 8-bit floats, and the step."""
    y = torch.where(scale > 0, x.abs() / scale, 0.0)
    step = torch.exp2(torch.log2(y.clamp(min=2.0 ** -6)).floor() - 3)
    return y / step, step


def make(sizes, param, grad, bits, copy, seed, offset=0, spread=True):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def at(n, dtype, value=None):  # `offset` elements behind the start of an allocation
        buf = torch.zeros(offset + n, device="cuda", dtype=torch.float32)
        buf[offset:] = torch.randn(n, generator=g, device="cuda") if value is None else value
        return buf.to(dtype)[offset:]
    out = dict(p=[], g=[], m=[], v=[], ms=[], vs=[], copy=[] if copy else None)
    for k, n in enumerate(sizes):
        size = 10.0 ** (-k % 5 - 2) if spread else 1e-2
        out["p"].append(at(n, param))
        out["g"].append(at(n, grad, torch.randn(n, generator=g, device="cuda") * size))
        m, r = torch.randn(n, generator=g, device="cuda") * size, torch.randn(n, generator=g, device="cuda").abs() * size
        if n > 20:
            r[3], m[3] = 0.0, 0.0  # an element that has had no gradient
            out["g"][-1][3] = 0
        if bits == 32:
            out["m"].append(at(n, torch.float32, m)), out["v"].append(at(n, torch.float32, r * r))
        else:
            for name, x in (("m", m), ("v", r)):
                scale = runs(x).abs().amax(1) / 448.0
                out[name].append(at(n, torch.float8_e4m3fn, (runs(x) / scale.clamp(min=1e-30)[:, None]).view(-1)[:n].clamp(-448, 448)))
                out[name + "s"].append(scale.clone())
        if copy:
            out["copy"].append(at(n, torch.bfloat16))
    return out


def plan_of(t, decay, bits):
    from paper_2609_13645_b200 import binding as Bn
    return Bn.AdamWPlan(t["p"], t["g"], t["m"], t["v"], weight_decay=decay, m_scales=t["ms"] if bits == 8 else None,
                        v_scales=t["vs"] if bits == 8 else None, copies=t["copy"])


def clone(t):
    return {k: [x.clone() for x in v] if v is not None else None for k, v in t.items()}


def check(old, new, bits, decay, step, clip, seed, lr=LR, base=0):
    for k, n in enumerate(old["p"]):
        n = n.numel()
        p, g = old["p"][k].double(), old["g"][k].double() * clip
        m0, v0 = (old["m"][k].double(), old["v"][k].double()) if bits == 32 else \
            (unpack(old["m"][k], old["ms"][k]), unpack(old["v"][k], old["vs"][k]) ** 2)
        m, v = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g  # the definition's order of operations
        update = (m / (1 - B1 ** step)) / ((v / (1 - B2 ** step)).sqrt() + EPS)
        want = p - lr * (update + decay[k] * p)
        bound = 2.0 ** -23 * p.abs() + lr * (2.0 ** -19 * (1 + (B1 * m0.abs() + (1 - B1) * g.abs()) / m.abs().clamp(min=1e-30)).clamp(max=2.0 ** 12) * update.abs()
                                             + 2.0 ** -22 * decay[k] * p.abs()) + 1e-12
        if old["p"][k].dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * want.abs()
        assert ((new["p"][k].double() - want).abs() <= bound).all(), k
        if new["copy"] is not None:
            assert torch.equal(new["copy"][k], new["p"][k].bfloat16())
        if bits == 32:
            assert ((new["m"][k].double() - m).abs() <= 2.0 ** -22 * (m0.abs() + g.abs())).all()
            assert ((new["v"][k].double() - v).abs() <= 2.0 ** -22 * v + 1e-37).all()
            continue
        u = randoms(seed, step, base, n)
        base += -(-n // 256) * 256
        for name, x, low in (("m", m, 0.0), ("v", v.sqrt(), 2.0 ** -9)):
            if not n:
                continue
            top = runs(x.abs()).amax(1)
            assert torch.equal(new[name + "s"][k], (top / 448).float())
            scale = (top / 448).repeat_interleave(256)[:n]
            count, unit = steps_of(x, scale)
            raw = count + u[:, 0 if name == "m" else 1]
            q = (raw.floor() * unit).clamp(max=448.0)
            q = torch.where((x != 0) & (scale > 0), q.clamp(min=low), q)
            got = new[name][k].double()
            assert torch.equal(got.abs(), q)
            assert ((got == 0) | (torch.sign(got) == torch.sign(x))).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_steps(bits, param, grad, offset):
    from paper_2609_13645_b200 import binding as Bn
    t = make(SIZES, param, grad, bits, param == torch.float32, 7, offset)
    decay = [0.1 * (k % 3) for k in range(len(SIZES))]
    plan = plan_of(t, decay, bits)
    clip = torch.tensor([0.75], device="cuda")
    for step in (1, 2, 1000):
        old = clone(t)
        Bn.k_adamw(plan, LR, B1, B2, EPS, torch.tensor([step], device="cuda"), grad_scale=clip, seed=99)
        check(old, t, bits, decay, step, 0.75, 99)
        assert all(torch.equal(a, b) for a, b in zip(old["g"], t["g"]))


def test_the_same_bits_twice_and_for_every_grouping():
    """Moments in 32 bits do not depend on which tensors share a plan; in 8 bits a step repeats its bits."""
    from paper_2609_13645_b200 import binding as Bn
    step = torch.tensor([3], device="cuda")
    for bits in (32, 8):
        a = make(SIZES, torch.float32, torch.float32, bits, False, 1)
        b = clone(a)
        Bn.k_adamw(plan_of(a, 0.1, bits), LR, B1, B2, EPS, step, seed=5)
        if bits == 32:
            for k in range(len(SIZES)):
                one = {n: v[k:k + 1] if v else v for n, v in b.items()}
                Bn.k_adamw(plan_of(one, 0.1, bits), LR, B1, B2, EPS, step, seed=5)
        else:
            Bn.k_adamw(plan_of(b, 0.1, bits), LR, B1, B2, EPS, step, seed=5)
        for name in ("p", "m", "v", "ms", "vs"):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a[name], b[name]))


def test_it_is_the_models_update():
    """The step's own optimizer, ft_apply_update, on the same values: the same bits."""
    from paper_2609_13645_b200 import binding as Bn
    cfg = Bn.make_config(1, 256, 4, 4, 64, 688, 1024, 2, 128, lr=1e-3, beta1=B1, beta2=B2, weight_decay=0.1)
    model = Bn.Model(cfg, seed=3)
    rng = np.random.RandomState(0)
    names = [n for n, _ in model.params]
    tok = torch.from_numpy(rng.randint(0, 1024, (2, 128)).astype(np.int32)).cuda()
    model.forward_backward(tok, tok)
    get = lambda kind: [torch.from_numpy(model.get_param(n, kind)).cuda().view(-1) for n in names]  # noqa: E731
    t = dict(p=get(Bn.KIND_MASTER), g=get(Bn.KIND_GRAD), m=get(Bn.KIND_ADAM_M), v=get(Bn.KIND_ADAM_V), ms=None, vs=None, copy=None)
    model.apply_update()
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    decay = [0.1 if len(shape) == 2 else 0.0 for _, shape in model.params]
    Bn.k_adamw(plan_of(t, decay, 32), f32(1e-3), f32(B1), f32(B2), f32(1e-8), torch.tensor([1], device="cuda"))
    for k, n in enumerate(names):
        for kind, name in ((Bn.KIND_ADAM_M, "m"), (Bn.KIND_ADAM_V, "v"), (Bn.KIND_MASTER, "p")):
            want = torch.from_numpy(model.get_param(n, kind)).cuda().view(-1)
            # the bias corrections may be formed otherwise: one rounding of the update, which the learning rate scales
            assert float((t[name][k] - want).abs().max()) <= (2e-10 if name == "p" else 0.0), (n, name)
    model.close()


def test_eight_bits_keep_the_mean_of_slow_moments():
    """Under a constant gradient m and v go to g and g^2 as in 32 bits, through steps far smaller than a code's."""
    from paper_2609_13645_b200 import binding as Bn
    n = 1 << 16
    p, g = [torch.zeros(n, device="cuda")], [torch.full((n,), 0.5, device="cuda")]
    g[0][::256] = 1.0  # sets the scale
    m8, v8 = [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)], [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)]
    ms, vs = [torch.zeros(n // 256, device="cuda")], [torch.zeros(n // 256, device="cuda")]
    plan = Bn.AdamWPlan(p, g, m8, v8, m_scales=ms, v_scales=vs)
    b1, b2, step = 0.95, 0.95, torch.zeros(1, dtype=torch.int64, device="cuda")
    for t in range(1, 101):
        step += 1
        Bn.k_adamw(plan, 0.0, b1, b2, 1e-8, step, seed=1)
    rest = torch.arange(n, device="cuda") % 256 != 0
    m = unpack(m8[0], ms[0])[rest]
    # m is a sum of roundings that keep the mean: the mean over 65280 elements is within 6 standard errors of the exact one, an
    # element's own deviation being under a code's step (1/16 of its value) times the root of the 1 / (1 - b1^2) steps it remembers
    want = 0.5 * (1 - b1 ** 100)
    assert abs(float(m.mean()) - want) < 6 * (0.5 / 8) * (1 / (1 - b1 * b1)) ** 0.5 / rest.sum().item() ** 0.5 + want * 1e-5
    r = unpack(v8[0], vs[0])[rest]
    # sqrt(v) keeps its mean in the rounding; the next step squares it, which adds its variance: at most a step's square
    want = 0.5 * (1 - b2 ** 100) ** 0.5
    assert abs(float(r.mean()) - want) < 0.1 * want and float((r == 0).sum()) == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_gradients_are_seen(bad):
    from paper_2609_13645_b200 import binding as Bn
    for bits in (32, 8):
        t = make([1000], torch.float32, torch.float32, bits, False, 3)
        t["g"][0][300] = bad
        old = clone(t)
        Bn.k_adamw(plan_of(t, 0.0, bits), LR, B1, B2, EPS, torch.tensor([2], device="cuda"), seed=1)
        assert not torch.isfinite(t["p"][0][300])
        others = torch.arange(1000, device="cuda") != 300
        assert torch.isfinite(t["p"][0][others]).all()
        m = t["m"][0].double() if bits == 32 else unpack(t["m"][0], t["ms"][0])
        run = (torch.arange(1000, device="cuda") // 256 == 1) if bits == 8 else ~others
        assert not torch.isfinite(m[run]).any() and torch.isfinite(m[~run]).all()
        assert not torch.equal(old["p"][0], t["p"][0])


def test_replays_read_step_rate_and_scale():
    from paper_2609_13645_b200 import binding as Bn
    for bits in (32, 8):
        t = make([700, 3], torch.float32, torch.bfloat16, bits, True, 2)
        plan = plan_of(t, 0.1, bits)
        step, lr, clip = torch.tensor([1], device="cuda"), torch.tensor([1e-2], device="cuda"), torch.tensor([1.0], device="cuda")
        call = lambda: Bn.k_adamw(plan, 123.0, B1, B2, EPS, step, lr_tensor=lr, grad_scale=clip, seed=8)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for s, rate, c in ((5, 3e-3, 0.5), (6, 2e-2, 0.25)):
            step.fill_(s), lr.fill_(rate), clip.fill_(c)
            old = clone(t)
            graph.replay()
            check(old, t, bits, [0.1, 0.1], s, c, 8, lr=float(lr[0]))


@pytest.mark.parametrize("bits", [32, 8])
def test_elements_past_32_bits(bits):
    """The last elements of a tensor of more than 2^31, and a tensor behind it."""
    from paper_2609_13645_b200 import binding as Bn
    far, last = 1 << 31, 1000
    t = make([last, 300], torch.bfloat16, torch.bfloat16, bits, False, 21)
    big = {}
    for name, v in t.items():
        if v is not None and len(v):
            skipped = far // 256 if name in ("ms", "vs") else far
            big[name] = torch.zeros(skipped + v[0].numel(), dtype=v[0].dtype, device="cuda")
            big[name][skipped:] = v[0]
    whole = {name: [big[name], v[1]] if v else v for name, v in t.items()}
    Bn.k_adamw(plan_of(whole, 0.1, bits), LR, B1, B2, EPS, torch.tensor([4], device="cuda"), seed=3)
    new = {name: [v[0][-t[name][0].numel():], v[1]] if v else v for name, v in whole.items()}
    first = {name: v[:1] if v else v for name, v in new.items()}
    check({name: v[:1] if v else v for name, v in t.items()}, first, bits, [0.1], 4, 1.0, 3, base=far)
    assert not big["p"][:far].any() and not big["m"][:far].view(torch.uint8).any()


def test_two_plans_on_two_streams():
    """Steps that run at the same time, and in other orders, give the bits of steps one after the other."""
    from paper_2609_13645_b200 import binding as Bn
    step, streams = torch.tensor([2], device="cuda"), [torch.cuda.Stream() for _ in range(2)]
    for bits in (32, 8):
        a = [make(SIZES + [1 << 20], torch.float32, torch.float32, bits, True, s) for s in (1, 2)]
        b = [clone(t) for t in a]
        plans = [plan_of(t, 0.1, bits) for t in b]
        for t in a:
            Bn.k_adamw(plan_of(t, 0.1, bits), LR, B1, B2, EPS, step, seed=5)
        torch.cuda.synchronize()
        for plan, stream in zip(plans, streams):
            with torch.cuda.stream(stream):
                Bn.k_adamw(plan, LR, B1, B2, EPS, step, seed=5)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            for name in ("p", "m", "v", "ms", "vs", "copy"):
                assert all(torch.equal(u.view(torch.uint8), w.view(torch.uint8)) for u, w in zip(x[name], y[name]))
