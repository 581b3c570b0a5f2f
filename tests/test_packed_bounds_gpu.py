"""The bounds of packed documents at the ends of what offsets can be."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("only", [3, 10, 2 ** 31 - 1, 0, -1])
def test_no_documents(only):
    """One offset is a list of no documents: all rows are nobody's and nothing in front of the offset is read, also where it is not 0,
    which is reported."""
    from paper_2609_13645_b200 import binding as Bn
    T = 10
    around = torch.tensor([1, only, 1], dtype=torch.int32, device="cuda")  # what a read beside the offset would find
    bounds = torch.full((3, T), -1, dtype=torch.int32, device="cuda")
    Bn.k_packed_bounds(around[1:2], bounds, T, 6)
    if only == 0:
        Bn.k_status()
    else:
        with pytest.raises(Bn.ForgeStepError) as e:
            Bn.k_status()
        assert e.value.status == Bn.FT_EINVAL
        Bn.k_status()
    want = np.zeros((3, T), dtype=np.int32)
    want[0] = T
    assert np.array_equal(bounds.cpu().numpy(), want)


def bounds_of_row(cu, n, T, t, read):
    """The kernel's index arithmetic for one row, each read of the offsets through `read`."""
    total = min(max(read(cu, n), 0), T) if n > 0 else 0
    if t >= total:
        return T, total, 0
    lo, hi = 0, n
    while lo < hi:
        mid = (lo + hi) >> 1
        if read(cu, mid + 1) > t:
            hi = mid
        else:
            lo = mid + 1
    i = min(lo, n - 1)
    start = min(max(read(cu, i), 0), t)
    return start, min(max(read(cu, i + 1), t + 1), total), t - start


@pytest.mark.parametrize("seed", range(3))
def test_any_offsets_are_read_within_their_list(seed):
    """Lists of any values, most of them refused: the reads that the arithmetic makes stay inside the list (checked here on the host
    before the call), the bounds are what it says, and the refusal is what the rules say."""
    from paper_2609_13645_b200 import binding as Bn
    g = np.random.RandomState(seed)
    T, longest = 37, 20
    for _ in range(60):
        n = int(g.randint(0, 6))
        cu = g.randint(-5, 50, n + 1) if g.rand() < 0.5 else np.sort(g.randint(0, T + 1, n + 1))
        if g.rand() < 0.5:
            cu[0] = 0

        def read(c, i):
            assert 0 <= i < len(c)
            return int(c[i])
        want = np.array([bounds_of_row(cu, n, T, t, read) for t in range(T)], dtype=np.int32).T
        good = cu[0] == 0 and cu[-1] <= T and all(0 <= b - a <= longest for a, b in zip(cu[:-1], cu[1:]))
        bounds = torch.full((3, T), -1, dtype=torch.int32, device="cuda")
        Bn.k_packed_bounds(torch.from_numpy(cu.astype(np.int32)).cuda(), bounds, T, longest)
        if good:
            Bn.k_status()
        else:
            with pytest.raises(Bn.ForgeStepError):
                Bn.k_status()
        assert np.array_equal(bounds.cpu().numpy(), want)
