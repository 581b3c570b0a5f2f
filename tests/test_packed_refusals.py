"""What the operators for packed documents refuse, on the host: the binding's checks with tensors on the CPU and the C calls with
addresses that are never used."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_13645_b200 import binding as Bn

P = 1 << 20  # an address; none of these calls gets as far as using it


def refused(f, *a, **k):
    with pytest.raises(Bn.ForgeStepError) as e:
        f(*a, **k)
    assert e.value.status == Bn.FT_EINVAL


def test_bounds():
    L = Bn.lib()
    ok = (P, 3, 100, 50, 2 * P)
    for i, v in ((0, 0), (0, P + 1), (1, -1), (1, 2 ** 31 - 1), (2, 0), (2, -1), (2, (1 << 28) + 1), (3, 0), (4, 0), (4, 2 * P + 2), (4, P), (4, P - 1196)):
        assert L.ft_k_packed_bounds(*[v if j == i else x for j, x in enumerate(ok)], None) == Bn.FT_EINVAL, (i, v)
    cu = torch.zeros(3, dtype=torch.int32)
    refused(Bn.k_packed_bounds, cu, torch.empty(3, 4, dtype=torch.int32), 4)  # no CUDA tensors
    refused(Bn.k_packed_bounds, cu, torch.empty(3, 4, dtype=torch.int32), 0)
    refused(Bn.k_packed_bounds, cu, torch.empty(3, 4, dtype=torch.int32), 2 ** 31)
    refused(Bn.k_packed_bounds, cu, torch.empty(3, 4, dtype=torch.int32), 4, 0)


def test_attention():
    L, G = Bn.lib(), 1 << 30
    T, nh, nkv, d = 100, 4, 2, 64
    fwd = [G, 2 * G, 3 * G, 4 * G, T, nh, nkv, d]
    for i, v in ((0, 0), (1, 0), (2, 0), (3, 0), (0, G + 8), (1, 2 * G + 2), (2, 3 * G + 1), (3, 4 * G + 2), (4, 0), (4, -1), (4, (1 << 28) + 1),
                 (5, 0), (5, 3), (6, 0), (6, 8), (7, 96), (7, 0), (1, G), (1, G + 100 * 8 * 128 - 16), (2, 2 * G), (2, G), (1, 4 * G), (2, 4 * G + 16)):
        assert L.ft_k_attention_packed_fwd(*[v if j == i else x for j, x in enumerate(fwd)], None) == Bn.FT_EINVAL, (i, v)
    size = L.ft_k_attention_packed_scratch_bytes(T, nh, nkv, d, 50)
    assert size > 0 and L.ft_k_attention_packed_scratch_bytes(T, nh, nkv, d, 0) == 0 and L.ft_k_attention_packed_scratch_bytes(T, nh, 3, d, 5) == 0
    assert 4 * L.ft_k_attention_packed_scratch_bytes(4096, 16, 8, 128, 100) < L.ft_k_attention_packed_scratch_bytes(4096, 16, 8, 128, 4096)
    bwd = [G, 2 * G, 3 * G, 4 * G, 5 * G, 6 * G, 7 * G, 8 * G, 9 * G, size, T, nh, nkv, d, 50]
    for i, v in ((0, 0), (1, 0), (2, 0), (3, 0), (4, 0), (5, 0), (8, 0), (0, G + 8), (6, 7 * G + 4), (6, 0), (7, 0), (8, 9 * G + 128), (10, 0), (11, 3),
                 (13, 32), (14, 0), (4, G), (4, 2 * G), (4, 3 * G), (4, 4 * G), (4, 6 * G), (4, 7 * G), (8, G), (8, 5 * G), (8, 6 * G), (8, 8 * G)):
        assert L.ft_k_attention_packed_bwd(*[v if j == i else x for j, x in enumerate(bwd)], None) == Bn.FT_EINVAL, (i, v)
    assert L.ft_k_attention_packed_bwd(*[size - 1 if j == 9 else x for j, x in enumerate(bwd)], None) == Bn.FT_ENOMEM
    for bad in ((0, 4, 2, 64), (10, 3, 2, 64), (10, 4, 2, 80), (2 ** 31, 4, 2, 64)):
        refused(Bn.attention_packed_scratch_bytes, *bad)
        refused(Bn.k_attention_packed_fwd, *[torch.zeros(1)] * 4, *bad)


def test_rotary():
    L, G = Bn.lib(), 1 << 30
    ok = [G, 512, 2 * G, 512, 3 * G, 4 * G, 5 * G, 64, 10, 4, 128, 128, 0, 0, 0]
    for i, v in ((0, 0), (2, 0), (5, 0), (6, 0), (1, 511), (3, 511), (0, G + 1), (2, 2 * G + 1), (4, 3 * G + 2), (5, 4 * G + 2), (7, 0), (8, 0), (9, 0), (9, -1),
                 (10, 0), (10, 127), (11, 0), (11, 3), (11, 130), (11, -2), (12, 2), (13, 2), (14, 2), (14, -1)):
        assert L.ft_k_rotary(*[v if j == i else x for j, x in enumerate(ok)], None) == Bn.FT_EINVAL, (i, v)
    rows = [v for v in ok]
    rows[4], rows[8] = None, 65  # more rows than positions
    assert L.ft_k_rotary(*rows, None) == Bn.FT_EINVAL
    same = [v for v in ok]
    same[2], same[3] = G, 520  # in place with another stride
    assert L.ft_k_rotary(*same, None) == Bn.FT_EINVAL
    # y over part of x, its tables or its positions (in bf16: rows of 1024 bytes)
    for i, v in ((2, G + 2), (2, G + 1024 * 9 + 1022), (0, 2 * G + 1022), (2, 4 * G - 2), (2, 5 * G + 64 * 256 - 2), (2, 3 * G + 38)):
        assert L.ft_k_rotary(*[v if j == i else x for j, x in enumerate(ok)], None) == Bn.FT_EINVAL, (i, v)
    wide = [v for v in ok]
    wide[1] = wide[3] = 1500  # rows of 3000 bytes of which x has the first 1024
    for v in (G + 1022, G + 3000 * 2 + 2, G + 3000 - 1022):
        assert L.ft_k_rotary(*[v if j == 2 else x for j, x in enumerate(wide)], None) == Bn.FT_EINVAL, v
    assert L.ft_k_rotary(*[{2: G + 1024, 3: 1540}.get(j, x) for j, x in enumerate(wide)], None) == Bn.FT_EINVAL  # another stride
    fp32 = [v for v in ok]
    fp32[14], fp32[0] = 1, G + 2
    assert L.ft_k_rotary(*fp32, None) == Bn.FT_EINVAL
    tab = [G, 2 * G, 3 * G, 100, 64, 1e4, 1.0]
    for i, v in ((0, 0), (1, 0), (0, G + 2), (2, 3 * G + 1), (3, 0), (4, 0), (4, 3), (4, 8194), (5, 0.0), (5, -1.0), (5, float("inf")), (5, float("nan")), (6, float("inf")),
                 (1, G + 12796), (2, G + 8), (2, 2 * G)):
        assert L.ft_k_rotary_tables(*[v if j == i else x for j, x in enumerate(tab)], None) == Bn.FT_EINVAL, (i, v)
    x, cos = torch.zeros(4, 8), torch.zeros(4, 2)
    refused(Bn.k_rotary, x, x, cos, cos, 2, 4)
    refused(Bn.k_rotary, x.half(), x, cos, cos, 2, 4)
    refused(Bn.k_rotary_tables, cos, cos)


def tensors(*rows):
    return (Bn.FtAdamWTensor * len(rows))(*[Bn.FtAdamWTensor(*r) for r in rows])


def test_adamw_plan():
    L, G = Bn.lib(), 1 << 30
    size = lambda t, p=1, g=1, b=32: L.ft_k_adamw_plan_bytes(t, len(t), p, g, b)  # noqa: E731
    ok = [G, 2 * G, 3 * G, 4 * G, None, None, 5 * G, 1000, 0.1]
    assert size(tensors(ok)) > 0
    eight = [G, 2 * G, 3 * G, 4 * G, 6 * G, 7 * G, 5 * G, 1000, 0.1]
    assert size(tensors(eight), b=8) > 0 and size(tensors(ok[:6] + [None] + ok[7:]), p=0) > 0
    assert size(tensors(eight)) == 0 and size(tensors(ok), b=8) == 0 and size(tensors(ok), p=0) == 0 and size(tensors(ok), b=16) == 0
    assert size(tensors(ok), p=2) == 0 and size(tensors(ok), g=-1) == 0 and L.ft_k_adamw_plan_bytes(tensors(ok), 0, 1, 1, 32) == 0
    assert L.ft_k_adamw_plan_bytes(None, 1, 1, 1, 32) == 0
    for i, v in ((0, None), (1, None), (2, None), (3, None), (0, G + 2), (1, 2 * G + 1), (2, 3 * G + 2), (6, 5 * G + 1), (7, -1), (7, 1 << 41), (8, float("nan")),
                 (0, 3 * G), (0, 3 * G - 3996), (2, 4 * G + 3996), (6, G), (1, G), (1, 4 * G - 400), (1, 5 * G + 1996)):
        assert size(tensors([v if j == i else x for j, x in enumerate(ok)])) == 0, (i, v)
    for i, v in ((4, None), (5, None), (4, 6 * G + 2), (4, 7 * G + 12), (5, 3 * G)):
        assert size(tensors([v if j == i else x for j, x in enumerate(eight)]), b=8) == 0, (i, v)
    far = [8 * v if isinstance(v, int) and v >= G else v for v in ok]
    assert size(tensors(ok, far)) > size(tensors(ok)) and size(tensors(ok, ok)) == 0  # the same tensor twice
    nothing = [None] * 7 + [0, 0.0]
    assert size(tensors(nothing)) > 0 and size(tensors(ok, nothing)) > 0
    n = size(tensors(ok))
    host = np.zeros(n // 8 + 1, dtype=np.uint64)
    assert L.ft_k_adamw_plan(tensors(ok), 1, 1, 1, 32, host.ctypes.data, n - 1) == Bn.FT_ENOMEM
    assert L.ft_k_adamw_plan(tensors(ok), 1, 1, 1, 32, host.ctypes.data + 4, n) == Bn.FT_EINVAL
    assert L.ft_k_adamw_plan(tensors(ok), 1, 1, 1, 32, None, n) == Bn.FT_EINVAL
    assert L.ft_k_adamw_plan(tensors(ok), 1, 1, 1, 32, host.ctypes.data, n) == Bn.FT_OK
    call = [host.ctypes.data, G, n, 1e-3, 0.9, 0.95, 1e-8, 2 * G, None, None, 0]
    for i, v in ((0, None), (1, None), (7, None), (1, G + 8), (2, n - 1), (2, 0), (3, float("nan")), (4, 1.0), (4, -0.1), (5, 1.5), (5, float("nan")), (6, -1.0), (7, 2 * G + 4),
                 (8, 2 * G + 2), (9, 2 * G + 1)):
        assert L.ft_k_adamw(*[v if j == i else x for j, x in enumerate(call)], None) == Bn.FT_EINVAL, (i, v)
    host[0] = 0  # not a plan
    assert L.ft_k_adamw(*call, None) == Bn.FT_EINVAL
    t = [torch.zeros(10)]
    refused(Bn.AdamWPlan, t, t, t, t)  # no CUDA tensors
    refused(Bn.AdamWPlan, [], [], [], [])
    refused(Bn.AdamWPlan, t, t, t, t + t)
    refused(Bn.AdamWPlan, t, t, t, t, weight_decay=[0.1, 0.2])
    refused(Bn.AdamWPlan, [t[0].half()], t, t, t)
    refused(Bn.AdamWPlan, t, t, [t[0].bfloat16()], t)
    refused(Bn.AdamWPlan, t, t, t, t, m_scales=t)


def test_an_empty_plan_steps_over_nothing():
    L = Bn.lib()
    t = tensors([None] * 7 + [0, 0.0])
    n = L.ft_k_adamw_plan_bytes(t, 1, 1, 1, 32)
    host = np.zeros(n // 8 + 1, dtype=np.uint64)
    assert L.ft_k_adamw_plan(t, 1, 1, 1, 32, host.ctypes.data, n) == Bn.FT_OK
    assert L.ft_k_adamw(host.ctypes.data, P, n, 1e-3, 0.9, 0.95, 1e-8, P, None, None, 0, None) == Bn.FT_OK
