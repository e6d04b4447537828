"""What the operators tell autograd: gradients of gradients raise (they are not there), what is written in place counts as changed, what a
backward needs may not have changed since."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def scan_call():
    from paper_2305_01515_amd.dense import Scan
    g = torch.Generator().manual_seed(0)
    x, u = (torch.randn(10, 8, generator=g).cuda().requires_grad_() for _ in range(2))
    h0, off = torch.randn(2, 8, generator=g).cuda().requires_grad_(), torch.tensor([0, 4, 10]).cuda()
    plan = Scan(8, torch.float32, 2, 10)
    return plan, (x, u, off, h0), lambda: plan(x, u, off, h0)[0]


def bias_call(**where):
    from paper_2305_01515_amd.dense import RelativeBias
    g = torch.Generator().manual_seed(0)
    table, scores = torch.randn(6, 2, generator=g).cuda().requires_grad_(), torch.randn(3, 2, 4, 5, generator=g).cuda().requires_grad_()
    plan = RelativeBias(2, [1, 3], bidirectional=True)
    return plan, (table, scores), lambda: plan(table, scores, **where)


@pytest.mark.parametrize("call", [scan_call, bias_call])
def test_gradients_of_gradients_raise(call):
    _, args, run = call()
    leaves = [t for t in args if t.requires_grad]
    # a penalty on the gradient: of the loss's square, so that the gradient depends on the inputs by the operator and by its output
    grads = torch.autograd.grad((run() ** 2).sum(), leaves, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (run().sum() + sum((x ** 2).sum() for x in grads)).backward()  # beside a loss that has a gradient
    first = torch.autograd.grad((run() ** 2).sum(), leaves)
    for a, b in zip(grads, first):
        assert torch.equal(a, b)


def test_a_weight_that_a_graph_holds_may_not_be_stepped():
    from paper_2305_01515_amd.dense import AdamW
    w, other = (torch.nn.Parameter(torch.randn(4, 4).cuda()) for _ in range(2))
    x = torch.randn(4, 4).cuda().requires_grad_()
    opt = AdamW([w, other])
    loss, fine = (x @ w).sum(), (x @ other).sum()
    opt.step([torch.ones(4, 4).cuda(), None])
    fine.backward()  # that one has been left as it is
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    loss = (x @ w).sum()
    opt.step([torch.ones(4, 4).cuda()] * 2)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()


def test_outputs_and_states_that_were_given():
    """what an earlier product saved has been written over: its backward raises"""
    plan, (x, u, off, h0), _ = scan_call()
    w = torch.randn(8, 8).cuda().requires_grad_()
    y, state = torch.randn(10, 8).cuda(), torch.randn(12, 8).cuda()
    loss = (y @ w).sum()
    plan.forward(x.detach(), u.detach(), off, y=y)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    loss = (state @ w).sum()
    plan.step(state, x.detach(), u.detach())
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    loss = (y @ w).sum()
    plan.step(state, x.detach(), u.detach(), y=y)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    bias, (table, scores), _ = bias_call()
    out = torch.randn(3, 2, 4, 5).cuda()
    loss = (out * scores).sum()
    bias.forward(table.detach(), scores=scores.detach(), out=out)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()


def test_under_inference_mode():
    from paper_2305_01515_amd.dense import AdamW
    plan, (x, u, off, h0), _ = scan_call()
    bias, (table, scores), _ = bias_call()
    w = torch.ones(5).cuda()
    opt = AdamW([w])
    with torch.inference_mode():
        state, y, out = torch.zeros(10, 8).cuda(), torch.empty(10, 8).cuda(), torch.empty(3, 2, 4, 5).cuda()
        plan.step(state, x, u, y=y)
        assert torch.equal(y, state) and bool((state != 0).any())
        plan.forward(x, u, off, y=y)
        bias.forward(table, scores=scores, out=out)
        opt.step([torch.ones(5).cuda()])
    assert bool((w < 1).all())


@pytest.mark.parametrize("name", ["q_pos", "k_pos", "key_lengths"])
def test_positions_and_lengths_that_change_before_the_backward(name):
    """a buffer that holds the next batch's by then: the gradient would be that of other buckets"""
    where = dict(q_pos=torch.arange(4).expand(3, 4).contiguous().cuda(), k_pos=torch.arange(5).expand(3, 5).contiguous().cuda(),
                 key_lengths=torch.tensor([5, 2, 0]).cuda())
    _, leaves, run = bias_call(mask_value=0.0, scale=0.5, **where)
    first = torch.autograd.grad(run().square().sum(), leaves)
    again = torch.autograd.grad(run().square().sum(), leaves)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    loss = run().sum()
    where[name].add_(1)
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
