"""Buffers that the decoder-block operators refuse by their place alone: tables that a gradient or scratch would overwrite, and
fp32 buffers that do not start at an fp32 element.  Nothing below is launched, so no device is needed."""
import pytest

from paper_2609_13645_b200 import binding as B
from paper_2609_13645_b200 import build

P, GIB = 1 << 20, 1 << 30  # an aligned address that nothing dereferences
SHAPE = (2, 200, 4, 2, 64, 50, 2)  # B, S, heads, kv heads, head dim, window, sinks


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


def test_rotation_tables_must_not_overlap_a_gradient_or_the_scratch(L):
    need, table = L.ft_k_attention_window_scratch_bytes(*SHAPE), 200 * 32 * 4
    apart = [P + i * GIB for i in range(8)]  # qkv, o, dO, lse, dqkv, cos, sin, scratch
    for t in (5, 6):
        for out, size in ((4, 2 * 200 * 8 * 64 * 2), (7, need)):
            for at in (0, 256, size - 16, 16 - table):
                p = list(apart)
                p[t] = p[out] + at
                assert L.ft_k_attention_window_bwd(*p, need, *SHAPE, None) == B.FT_EINVAL, (t, out, at)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_fp32_buffers_start_at_an_element(L, shift):
    q, need = P + shift, L.ft_k_attention_window_scratch_bytes(*SHAPE)
    a = [P + i * GIB for i in range(8)]
    assert L.ft_k_attention_window_fwd(a[0], a[1], a[2] + shift, *SHAPE, None) == B.FT_EINVAL
    assert L.ft_k_attention_window_bwd(a[0], a[1], a[2], a[3] + shift, a[4], None, None, a[7], need, *SHAPE, None) == B.FT_EINVAL
    fwd = lambda mean, rstd: L.ft_k_layernorm_fwd(a[0], 64, a[1], None, a[2], 64, mean, rstd, 4, 64, 1e-5, 0, None)  # noqa: E731
    assert fwd(q, a[4]) == B.FT_EINVAL and fwd(a[3], q) == B.FT_EINVAL
    ok = dict(mean=a[2], rstd=a[3], dgain=a[5], dbias=a[6])
    for name in ok:
        b = dict(ok, **{name: q})
        assert L.ft_k_layernorm_bwd(a[0], 64, a[1], 64, b["mean"], b["rstd"], a[4], None, 0, a[7], 64, b["dgain"], b["dbias"], a[7] + GIB,
                                    GIB, 4, 64, 0, None) == B.FT_EINVAL, name


def test_dropout_whose_factor_passes_fp32(L):
    """scale / (1 - p') is one fp32 number: beyond its range an element of 0 would become 0 * inf."""
    drop = lambda p, scale: L.ft_k_dropout_add(P, 64, None, 0, P + GIB, 64, 4, 64, p, scale, 1, 0, None, 0, None)  # noqa: E731
    assert drop(0.5, 3e38) == B.FT_EINVAL and drop(0.99999, -1e36) == B.FT_EINVAL
