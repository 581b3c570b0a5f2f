"""Lists of tensors with gaps are refused like any other mistake in a plan."""
import pytest
import torch

from paper_2609_13645_b200 import binding as Bn


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("where", [0, 1])
def test_a_missing_tensor(which, where):
    lists = [[torch.zeros(10), torch.zeros(10)] for _ in range(4)]
    lists[which][where] = None  # a parameter without a gradient, for one
    with pytest.raises(Bn.ForgeStepError) as e:
        Bn.AdamWPlan(*lists)
    assert e.value.status == Bn.FT_EINVAL
