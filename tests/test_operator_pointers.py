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
