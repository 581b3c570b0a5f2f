"""A plan that is dropped while its step still runs on a stream of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
def test_a_dropped_plan_keeps_its_memory_until_its_step_is_through(captured):
    """The step waits on a side stream; meanwhile nothing may get the plan's memory, which the kernel reads addresses from."""
    from paper_2609_13645_b200 import binding as Bn
    n, side = 1 << 16, torch.cuda.Stream()
    p, g, m, v = (torch.ones(n, device="cuda") for _ in range(4))
    step = torch.tensor([1], device="cuda")
    Bn.k_adamw(Bn.AdamWPlan([p], [g], [m], [v]), 1e-2, 0.9, 0.95, 1e-8, step)  # the kernel is loaded, which may wait for the GPU
    torch.cuda._sleep(1000)
    torch.cuda.synchronize()
    p.fill_(1.0)
    plan = Bn.AdamWPlan([p], [g], [m], [v])
    if captured:  # the plan has met the stream in a capture before
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            Bn.k_adamw(plan, 1e-2, 0.9, 0.95, 1e-8, step)
        graph.replay()
        torch.cuda.synchronize()
    address, size = plan.device.data_ptr(), plan.device.numel()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # cycles: about a tenth of a second
        Bn.k_adamw(plan, 1e-2, 0.9, 0.95, 1e-8, step)
        done = torch.cuda.Event()
        done.record()
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(8)]  # not written
    assert not done.query()
    assert all(not t.data_ptr() <= address < t.data_ptr() + max(size, 512) for t in others)
    torch.cuda.synchronize()
    assert not torch.equal(p, torch.ones_like(p))
