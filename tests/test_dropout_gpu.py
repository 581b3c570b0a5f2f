"""Dropout with a residual against its definition: the mask bit for bit, the values to one rounding, which is off by at most
half a step, torch.finfo(t).eps / 2 of the value: 2^-8 in bf16 (8 significant bits), 2^-24 in fp32."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

M64 = (1 << 64) - 1


def _mix(z):
    z = z + np.uint64(0x9E3779B97F4A7C15)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def keep_mask(rows, h, p, seed, site, step):
    n = rows * h
    with np.errstate(over="ignore"):
        one = lambda v: np.array([v & M64], dtype=np.uint64)  # noqa: E731
        key = _mix(_mix(one(seed ^ ((site + 1) * 0xD1B54A32D192ED03))) ^ one(step * 0xA24BAED4963EE407))
        i = np.arange(n, dtype=np.uint64)
        word = _mix(key ^ (i // np.uint64(4) * np.uint64(0x8CB92BA72F3D8DD7)))
        bits = (word >> (np.uint64(16) * (i % np.uint64(4)))) & np.uint64(0xFFFF)
    t = min(65535, int(np.floor(float(np.float32(p)) * 65536 + 0.5)))
    return torch.from_numpy((bits >= np.uint64(t)).reshape(rows, h)).cuda(), t


def _rows(g, rows, h, dtype, pad=0, offset=0):
    return torch.randn(rows, h + pad + offset, generator=g, device="cuda").to(dtype)[:, offset:offset + h]


@pytest.mark.parametrize("rows,h,pad,offset", [(1, 1, 0, 0), (1, 3, 0, 0), (5, 7, 0, 0), (3, 8, 8, 0), (64, 100, 0, 0), (33, 129, 3, 0),
                                               (17, 260, 4, 0), (40, 514, 2, 0), (129, 2048, 0, 0), (50, 1000, 5, 1), (1, 40001, 0, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999])
@pytest.mark.parametrize("resid", [True, False])
def test_matches_the_definition(rows, h, pad, offset, dtype, p, resid):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    x = _rows(g, rows, h, dtype, pad, offset)
    r = _rows(g, rows, h, dtype, pad, offset) if resid else None
    out = torch.full((rows, h + pad + offset), 3.0, dtype=dtype, device="cuda")
    y = out[:, offset:offset + h]
    step = torch.tensor([11], dtype=torch.int64, device="cuda")
    Bn.k_dropout_add(x, r, y, p, 0xFEDCBA9876543210, 3, step=step, scale=0.75)
    keep, t = keep_mask(rows, h, p, 0xFEDCBA9876543210, 3, 11)
    kept = torch.where(keep, x.double() * 0.75 * 65536.0 / (65536 - t), torch.zeros((), dtype=torch.float64, device="cuda"))
    ref = kept if r is None else kept + r.double()
    u = torch.finfo(dtype).eps / 2
    # one rounding of the result; before it the product's and the sum's in fp32
    bound = u * ref.abs() * 1.001 + 2.0 ** -22 * (kept.abs() + ref.abs()) + 1e-38
    assert ((y.double() - ref).abs() <= bound).all()
    if r is None:
        assert torch.equal(y != 0, keep & (x != 0))
    if pad + offset:
        rest = torch.ones(h + pad + offset, dtype=torch.bool, device="cuda")
        rest[offset:offset + h] = False
        assert (out[:, rest] == 3).all()


def test_the_gradient_uses_the_forward_mask_and_the_stride_does_not_change_it():
    from paper_2609_13645_b200 import binding as Bn
    rows, h, p = 70, 333, 0.3
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dy = (_rows(g, rows, h, torch.float32) for _ in range(3))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    Bn.k_dropout_add(x, r, y, p, 5, 0, scale=2.0)
    Bn.k_dropout_add(dy, None, dx, p, 5, 0, scale=2.0)
    keep, t = keep_mask(rows, h, p, 5, 0, 0)
    assert torch.equal(dx != 0, keep)
    # d(sum(y dy)) / dx by differences: the map is linear in x
    v = torch.randn(rows, h, generator=g, device="cuda")
    y2 = torch.empty_like(y)
    Bn.k_dropout_add(x + v, r, y2, p, 5, 0, scale=2.0)
    a, b = float(((y2 - y).double() * dy.double()).sum()), float((dx.double() * v.double()).sum())
    assert abs(a - b) < 1e-4 * float(dx.double().norm())
    wide = torch.zeros(rows, h + 3, device="cuda")
    Bn.k_dropout_add(dy, None, wide[:, :h], p, 5, 0, scale=2.0)
    assert torch.equal(wide[:, :h], dx)


def test_seed_site_and_step_give_other_masks_of_the_right_rate():
    from paper_2609_13645_b200 import binding as Bn
    rows, h, p = 512, 1024, 0.1
    x = torch.ones(rows, h, device="cuda")
    masks = []
    for seed, site, step in ((1, 0, None), (2, 0, None), (1, 1, None), (1, 0, 1), (1, 0, 2)):
        y = torch.empty_like(x)
        s = None if step is None else torch.tensor([step], dtype=torch.int64, device="cuda")
        Bn.k_dropout_add(x, None, y, p, seed, site, step=s)
        masks.append(y != 0)
        n, q = rows * h, 6554 / 65536
        assert abs(int((~masks[-1]).sum()) - n * q) < 6 * (n * q * (1 - q)) ** 0.5
        assert abs(float(y.double().mean()) - 1.0) < 6 * (q / (1 - q) / n) ** 0.5
    for i in range(5):
        for j in range(i):
            both = float((masks[i] ^ masks[j]).double().mean())  # independent masks differ in 2 q (1 - q) of the places
            assert abs(both - 2 * q * (1 - q)) < 6 * (2 * q * (1 - q) / n) ** 0.5


def test_a_dropped_element_contributes_zero_whatever_its_value():
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 16, 64
    keep, _ = keep_mask(rows, h, 0.5, 9, 2, 0)
    x = torch.where(keep, 1.0, float("nan")).to(torch.bfloat16)
    x[0] = torch.where(keep[0], 1.0, float("inf")).to(torch.bfloat16)
    r = torch.full_like(x, 4.0)
    Bn.k_dropout_add(x, r, x, 0.5, 9, 2)  # in place
    assert torch.equal(x, torch.where(keep, 6.0, 4.0).to(torch.bfloat16))


def test_replays_read_the_step_on_the_device():
    from paper_2609_13645_b200 import binding as Bn
    rows, h = 64, 512
    x, y = torch.ones(rows, h, device="cuda", dtype=torch.bfloat16), torch.empty(rows, h, device="cuda", dtype=torch.bfloat16)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    Bn.k_dropout_add(x, None, y, 0.25, 77, 4, step=step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Bn.k_dropout_add(x, None, y, 0.25, 77, 4, step=step)
    for s in (3, 4):
        step.fill_(s)
        graph.replay()
        assert torch.equal(y != 0, keep_mask(rows, h, 0.25, 77, 4, s)[0])


@pytest.mark.parametrize("rows,h", [(1, 3), (5, 7), (3, 16), (40, 241), (700, 2047), (1500, 33)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_tensor_at_an_alignment_of_its_own(rows, h, dtype):
    from paper_2609_13645_b200 import binding as Bn
    g = torch.Generator(device="cuda").manual_seed(rows + h)

    def at(ld, offset):  # rows that begin `offset` elements into an allocation which ends with the last of them
        buf = torch.randn(offset + (rows - 1) * ld + h, generator=g, device="cuda").to(dtype)
        return torch.as_strided(buf, (rows, h), (ld, 1), offset)
    x, r, y = at(h + 3, 1), at(h + 8, 6), at(h + 1, 3)
    Bn.k_dropout_add(x, r, y, 0.25, 11, 1, scale=0.5)
    keep, t = keep_mask(rows, h, 0.25, 11, 1, 0)
    want = r.double() + x.double() * keep * (0.5 * 65536.0 / (65536.0 - t))
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22
    assert ((y.double() - want).abs() <= eps * want.abs() + 2.0 ** -22 * (r.double().abs() + x.double().abs())).all()
    x2 = x.clone()  # packed
    r2 = r.clone()
    out = torch.empty_like(x2)
    Bn.k_dropout_add(x2, r2, out, 0.25, 11, 1, scale=0.5)
    assert torch.equal(out, y)
    Bn.k_dropout_add(x, r, r, 0.25, 11, 1, scale=0.5)  # in place
    assert torch.equal(r, y)
