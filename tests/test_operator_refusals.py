"""What the decoder-block operators refuse, through the C entry points (which validate before they touch the device, so this
runs without one) and through the binding's checks of tensors."""
import ctypes as C

import pytest
import torch

from paper_2609_13645_b200 import binding as B
from paper_2609_13645_b200 import build

P = 1 << 20  # an aligned address that nothing dereferences: every call below is refused first
GIB = 1 << 30


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


ATT = dict(B=2, S=200, nh=4, nkv=2, d=64, window=50, sinks=2)


def _att(**kw):
    a = dict(ATT, **kw)
    return [a[k] for k in ("B", "S", "nh", "nkv", "d", "window", "sinks")]


BAD_ATT = [dict(B=0), dict(S=0), dict(S=-1), dict(nh=0), dict(nkv=0), dict(nh=3), dict(d=96), dict(d=0), dict(window=0), dict(window=-5),
           dict(sinks=-1), dict(S=2 ** 31 - 1), dict(B=2 ** 31 - 1), dict(nh=2 ** 31 - 2), dict(B=-2 ** 31)]


@pytest.mark.parametrize("bad", BAD_ATT)
def test_attention_window_shapes(L, bad):
    assert L.ft_k_attention_window_scratch_bytes(*_att(**bad)) == 0
    assert L.ft_k_attention_window_bwd(P, P, P, P, P, None, None, P, GIB, *_att(**bad), None) == B.FT_EINVAL


def test_attention_window_pointers_and_scratch(L):
    need = L.ft_k_attention_window_scratch_bytes(*_att())
    assert need >= 4 * 2 * 4 * 200
    good = [P, P, P, P, P, P, P, P]
    for i in (0, 1, 2, 3, 4, 7):
        assert L.ft_k_attention_window_bwd(*(good[:i] + [None] + good[i + 1:]), GIB, *_att(), None) == B.FT_EINVAL
    for i in (0, 1, 2, 4, 5, 6, 7):  # misaligned
        assert L.ft_k_attention_window_bwd(*(good[:i] + [P + 8] + good[i + 1:]), GIB, *_att(), None) == B.FT_EINVAL
    assert L.ft_k_attention_window_bwd(*good, need - 1, *_att(), None) == B.FT_ENOMEM
    assert L.ft_k_attention_window_bwd(*good, 0, *_att(), None) == B.FT_ENOMEM
    for i in range(3):
        assert L.ft_k_attention_window_fwd(*([P, P, P][:i] + [None] + [P, P, P][i + 1:]), *_att(), None) == B.FT_EINVAL
    assert L.ft_k_attention_window_fwd(P + 2, P, P, *_att(), None) == B.FT_EINVAL
    assert L.ft_k_attention_window_fwd(P, P + 4, P, *_att(), None) == B.FT_EINVAL


def test_attention_window_scratch_grows_with_what_is_cut(L):
    """A long sequence's sink block is cut into parts; a mask that covers the sequence is plain causal attention."""
    plain = L.ft_k_attention_window_scratch_bytes(*_att(S=16384, nh=16, nkv=8, d=128, window=1024, sinks=0))
    cut = L.ft_k_attention_window_scratch_bytes(*_att(S=16384, nh=16, nkv=8, d=128, window=1024, sinks=4))
    assert cut > plain and cut < 2 ** 32
    over = L.ft_k_attention_window_scratch_bytes(*_att(window=2 ** 31 - 1, sinks=2 ** 31 - 1))
    assert over == L.ft_k_attention_window_scratch_bytes(*_att(window=200, sinks=0)) > 0
    # however the sinks and the window are chosen, the parts stay a bounded number
    for window in (1, 7, 4096):
        for sinks in (0, 1, 65536, 131072):
            assert 0 < L.ft_k_attention_window_scratch_bytes(1, 131072, 8, 1, 128, window, sinks) < 2 ** 33


def _ln_fwd(L, **kw):
    a = dict(x=P, ldx=64, gain=P, bias=P, y=P, ldy=64, mean=P, rstd=P, rows=4, h=64, eps=1e-5, dtype=0)
    a.update(kw)
    return L.ft_k_layernorm_fwd(*a.values(), None)


def _ln_bwd(L, **kw):
    a = dict(dy=P, lddy=64, x=P, ldx=64, mean=P, rstd=P, gain=P, resid=P, ldr=64, dx=P, lddx=64, dgain=P, dbias=P, scratch=P, bytes=GIB,
             rows=4, h=64, dtype=0)
    a.update(kw)
    return L.ft_k_layernorm_bwd(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(gain=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(rows=0), dict(rows=-3),
                                 dict(h=0), dict(h=16385), dict(ldx=63), dict(ldy=63), dict(dtype=2), dict(dtype=-1), dict(x=P + 1),
                                 dict(y=P + 2, dtype=1), dict(eps=float("nan")), dict(eps=-1.0)])
def test_layernorm_forward(L, bad):
    assert _ln_fwd(L, **bad) == B.FT_EINVAL


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(gain=None), dict(dx=None),
                                 dict(dgain=None), dict(scratch=None), dict(rows=0), dict(h=0), dict(h=16385), dict(lddy=1), dict(ldx=63),
                                 dict(lddx=0), dict(ldr=63), dict(dtype=3), dict(dx=P + 1), dict(scratch=P + 4)])
def test_layernorm_backward(L, bad):
    assert _ln_bwd(L, **bad) == B.FT_EINVAL


def test_layernorm_scratch(L):
    assert L.ft_k_layernorm_scratch_bytes(0, 64) == 0 and L.ft_k_layernorm_scratch_bytes(4, 16385) == 0
    need = L.ft_k_layernorm_scratch_bytes(4, 64)
    assert need >= 2 * 64 * 4 and _ln_bwd(L, bytes=need - 1) == B.FT_ENOMEM
    assert L.ft_k_layernorm_scratch_bytes(2 ** 31 - 1, 16384) < 2 ** 27


def _drop(L, **kw):
    a = dict(x=P, ldx=64, resid=P, ldr=64, y=P, ldy=64, rows=4, h=64, p=0.1, scale=1.0, seed=1, site=0, step=P, dtype=0)
    a.update(kw)
    return L.ft_k_dropout_add(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(rows=0), dict(h=-1), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")),
                                 dict(scale=float("inf")), dict(scale=float("nan")), dict(site=-1), dict(dtype=2), dict(ldx=63), dict(ldy=63),
                                 dict(ldr=10), dict(x=P + 1), dict(y=P + 2, dtype=1), dict(step=P + 4)])
def test_dropout(L, bad):
    assert _drop(L, **bad) == B.FT_EINVAL


def _refused(call):
    with pytest.raises(B.ForgeStepError) as e:
        call()
    assert e.value.status == B.FT_EINVAL


def test_the_binding_refuses_host_tensors_and_bad_shapes(L):
    """Host tensors are refused by name instead of being handed to a kernel; shapes before anything else."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    _refused(lambda: B.k_attention_window_fwd(bf(200, 512), bf(200, 256), f(800), 1, 200, 4, 2, 64, 50, 2))
    _refused(lambda: B.k_layernorm_fwd(bf(4, 64), bf(64), None, bf(4, 64), f(4), f(4)))
    _refused(lambda: B.k_layernorm_fwd(torch.zeros(4, 64, dtype=torch.float16), bf(64), None, bf(4, 64), f(4), f(4)))
    _refused(lambda: B.k_dropout_add(bf(4, 64), None, bf(4, 64), 0.1, 1, 0))
    for bad in (dict(window=0), dict(sinks=-1), dict(nh=3), dict(d=80), dict(S=0)):
        _refused(lambda: B.attention_window_scratch_bytes(*_att(**bad)))


def test_attention_window_buffers_that_overlap(L):
    need = L.ft_k_attention_window_scratch_bytes(*_att())
    T, row = 2 * 200, (4 + 2 * 2) * 64 * 2
    apart = [P + i * GIB for i in range(6)]  # qkv, o, dO, lse, dqkv, scratch

    def bwd(p):
        return L.ft_k_attention_window_bwd(p[0], p[1], p[2], p[3], p[4], None, None, p[5], need, *_att(), None)
    for out in (4, 5):
        for other in range(6):
            if other != out:
                for shift in (0, 256, -256):
                    p = list(apart)
                    p[out] = p[other] + shift
                    assert bwd(p) == B.FT_EINVAL, (out, other, shift)
    q = P
    for o, lse in ((q, q + GIB), (q + GIB, q), (q + GIB, q + GIB), (q + T * row - 16, q + GIB), (q + GIB, q + T * row - 4)):
        assert L.ft_k_attention_window_fwd(q, o, lse, *_att(), None) == B.FT_EINVAL


def test_outputs_over_inputs_of_another_stride(L):
    Q = P + GIB
    assert L.ft_k_layernorm_fwd(P, 64, Q, None, P, 72, Q, Q, 8, 64, 1e-5, 0, None) == B.FT_EINVAL
    bwd = lambda dy, lddy, x, r, ldr, dx, lddx: L.ft_k_layernorm_bwd(dy, lddy, x, 64, Q, Q, Q, r, ldr, dx, lddx, Q, Q, Q, GIB, 8, 64, 0, None)  # noqa: E731
    assert bwd(P, 64, Q, None, 0, P, 72) == B.FT_EINVAL
    assert bwd(Q, 64, Q, P, 64, P, 72) == B.FT_EINVAL
    assert bwd(Q, 64, P, None, 0, P, 72) == B.FT_EINVAL
    drop = lambda x, ldx, r, ldr, y, ldy: L.ft_k_dropout_add(x, ldx, r, ldr, y, ldy, 8, 64, 0.1, 1.0, 3, 0, None, 0, None)  # noqa: E731
    assert drop(P, 64, None, 0, P, 72) == B.FT_EINVAL and drop(Q, 64, P, 80, P, 72) == B.FT_EINVAL


def test_sizes_beyond_32_bits():
    wide = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="meta")  # noqa: E731
    for shape in ((2 ** 31, 1), (1, 2 ** 31)):
        _refused(lambda: B._rows_of(wide(*shape)))
    assert B._rows_of(wide(2 ** 31 - 1, 1)) == (2 ** 31 - 1, 1)
    for kw in (dict(B=2 ** 32 + 2), dict(S=2 ** 32 + 200), dict(nh=2 ** 32 + 4)):
        _refused(lambda: B.attention_window_scratch_bytes(*_att(**kw)))
    assert B.layernorm_scratch_bytes(2 ** 32 + 5, 64) == 0 and B.layernorm_scratch_bytes(5, 2 ** 32 + 64) == 0


@pytest.mark.gpu
def test_the_binding_refuses_tensors_of_another_layout():
    dev = "cuda"
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    f = lambda *s: torch.zeros(*s, device=dev)  # noqa: E731
    S, nh, nkv, d = 200, 4, 2, 64
    qkv, o, lse = bf(S, (nh + 2 * nkv) * d), bf(S, nh * d), f(nh, S)
    call = lambda q=qkv, o=o, l=lse, **kw: B.k_attention_window_fwd(q, o, l, 1, S, nh, nkv, d, kw.get("window", 50), kw.get("sinks", 2))  # noqa: E731,E741
    call()
    _refused(lambda: call(q=qkv.float()))
    _refused(lambda: call(q=bf(S, 2 * (nh + 2 * nkv) * d)[:, ::2]))
    _refused(lambda: call(o=bf(S, nh * d - 1)))
    _refused(lambda: call(l=lse.double()))
    _refused(lambda: call(o=o.cpu()))
    need = B.attention_window_scratch_bytes(1, S, nh, nkv, d, 50, 2)
    bwd = lambda s, **kw: B.k_attention_window_bwd(qkv, o, o, lse, bf(*qkv.shape), s, 1, S, nh, nkv, d, 50, 2, **kw)  # noqa: E731
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8, device=dev)  # noqa: E731
    bwd(u8(need))
    _refused(lambda: bwd(u8(need), cos=f(S, d // 2)))
    _refused(lambda: bwd(u8(need), cos=f(S, d), sin=f(S, d)))
    _refused(lambda: bwd(u8(need + 8)[8:]))
    with pytest.raises(B.ForgeStepError) as e:
        bwd(u8(need - 1))
    assert e.value.status == B.FT_ENOMEM
    x, g, m = bf(8, 64), bf(64), f(8)
    B.k_layernorm_fwd(x, g, None, bf(8, 64), m, f(8))
    _refused(lambda: B.k_layernorm_fwd(x.t(), bf(8), None, bf(64, 8), f(64), f(64)))
    _refused(lambda: B.k_layernorm_fwd(x[0], g, None, bf(64), f(1), f(1)))
    _refused(lambda: B.k_layernorm_fwd(x[:1].expand(8, 64), g, None, bf(8, 64), m, f(8)))
    _refused(lambda: B.k_layernorm_fwd(x, f(64), None, bf(8, 64), m, f(8)))
    _refused(lambda: B.k_layernorm_fwd(x, g, None, bf(8, 64), f(7), f(8)))
    _refused(lambda: B.k_layernorm_bwd(x, x, m, m, g, None, bf(8, 64), f(64), None, u8(16)[:0]))
    _refused(lambda: B.k_dropout_add(x, bf(8, 63), bf(8, 64), 0.1, 1, 0))
    _refused(lambda: B.k_dropout_add(x, None, bf(8, 64), 1.0, 1, 0))
    _refused(lambda: B.k_dropout_add(x, None, bf(8, 64), 0.1, 1, 2 ** 32))
    _refused(lambda: B.k_dropout_add(x, None, bf(8, 64), 0.1, 1, -1))
    _refused(lambda: B.k_attention_window_bwd(qkv, o, o, lse, qkv, u8(need), 1, S, nh, nkv, d, 50, 2))
    _refused(lambda: call(o=qkv.view(-1)[:S * nh * d]))
    _refused(lambda: B.k_dropout_add(x, None, bf(8, 64), 0.1, 1, 0, step=torch.zeros(1, dtype=torch.int32, device=dev)))
    _refused(lambda: B.k_dropout_add(x, None, bf(8, 64), 0.1, 1, 0, step=torch.zeros(1, dtype=torch.int64)))
