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
