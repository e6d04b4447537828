"""An output in an input's memory is refused: a chunk that has heard nothing goes through the rows before it again, which would be outputs by then."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_outputs_in_the_inputs_memory():
    from paper_2305_01515_amd import dense
    from paper_2305_01515_amd.tbe import TbeError
    g = torch.Generator().manual_seed(0)
    x, u, dy = (torch.randn(10, 8, generator=g).cuda() for _ in range(3))
    off = torch.tensor([0, 4, 10]).cuda()
    plan = dense.Scan(8, torch.float32, 2, 10)
    want, _, saved = plan.forward(x, u, off, save=True)
    for t in (x, u):
        kept = t.clone()
        with pytest.raises(TbeError) as e:
            plan.forward(x, u, off, y=t)
        assert e.value.code == -1 and torch.equal(t, kept)
    assert torch.equal(plan.forward(x, u, off)[0], want)
    a = [t.data_ptr() for t in (x, u, dy, torch.empty_like(x))]
    call = lambda dx, du: dense._lib().tbe_scan_backward(plan._h, a[0], 8, a[1], 8, off.data_ptr(), 2, 10, None, 0, saved.data_ptr(), a[2], 8, None, dx, 8,  # noqa: E731
                                                         du, 8, None, torch.cuda.current_stream().cuda_stream)
    for k in range(3):
        assert call(a[k], a[3]) == call(a[3], a[k]) == -1
    empty = torch.empty(0, 8).cuda()
    plan.forward(empty, empty, torch.tensor([0, 0]).cuda(), y=empty)
    plan.check()
