"""A plan that is made anew: not within a capture, where nothing can be allocated, and without taking from captured steps what they read."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_capture_that_would_need_another_plan():
    """refused before anything is done: object and capture go on"""
    from paper_2305_01515_amd.dense import AdamW
    start = torch.randn(1000, generator=torch.Generator().manual_seed(0)).cuda()
    p, q = start.clone(), start.clone()
    one, two = AdamW([p], lr=1e-2), AdamW([q], lr=1e-2)
    g = torch.randn(1000, generator=torch.Generator().manual_seed(1)).cuda()
    half = g.half()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError):
            one.step([half])  # gradients of another type
        assert one.step_count == 0
        h = g * 2
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, g * 2) and torch.equal(p, start)
    for _ in range(2):
        one.step([g])
        two.step([g])
    assert torch.equal(p, q)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError):
            AdamW([p])


def test_captured_steps_outlive_their_plan():
    from paper_2305_01515_amd.dense import AdamW
    start = torch.randn(5000, generator=torch.Generator().manual_seed(2)).cuda()
    p, q = start.clone(), start.clone()
    one, two = AdamW([p], lr=1e-2), AdamW([q], lr=1e-2)
    g = torch.randn(5000, generator=torch.Generator().manual_seed(3)).cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step([g])
    handle = one._h.value
    one.step_count = 0
    one.step([g.bfloat16()])  # a plan of its own
    assert one._h.value != handle and [h.value for h in one._kept] == [handle]
    two.step([g.bfloat16()])
    for _ in range(3):
        graph.replay()
        two.step_count = 0
        two.step([g])
    torch.cuda.synchronize()
    assert torch.equal(p, q)
    for k in one.states:
        assert torch.equal(one.states[k], two.states[k])
    one.close()
    assert not one._kept and not one._h


def test_a_plan_that_cannot_be_made_leaves_the_old_one():
    from paper_2305_01515_amd.dense import AdamW
    from paper_2305_01515_amd.tbe import TbeError
    p = torch.zeros(100).cuda()
    opt = AdamW([p], lr=1.0, weight_decay=0.0)
    opt._decay = [float("nan")]
    with pytest.raises(TbeError):
        opt.step([torch.ones(100).cuda().half()])
    opt._decay = [0.0]
    opt.step([torch.ones(100).cuda()])
    assert bool((p < -0.9).all())
