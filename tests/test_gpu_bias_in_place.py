"""Output (gradient of the scores) in the scores' (the gradient's) own memory: with the same strides, or refused."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu


def call():
    from paper_2305_01515_amd.dense import RelativeBias
    g = torch.Generator().manual_seed(0)
    return RelativeBias(2, [1, 3]), torch.randn(3, 2, generator=g).cuda(), torch.randn(3, 2, 4, 8, generator=g).cuda()


def test_other_strides_are_refused():
    from paper_2305_01515_amd.tbe import TbeError
    plan, table, scores = call()
    kept = scores.clone()
    for other in (scores.as_strided((3, 2, 4, 8), (64, 8, 16, 1)), scores.as_strided((3, 2, 4, 8), (8, 24, 48, 1))):
        with pytest.raises(TbeError) as e:
            plan.forward(table, scores=scores, out=other)
        assert e.value.code == -1
        with pytest.raises(TbeError):
            plan.forward(table, scores=other, out=scores)
    assert torch.equal(scores, kept)
    want = plan.forward(table, scores=scores)
    plan.forward(table, scores=scores, out=scores)
    assert torch.equal(scores, want)


def test_strides_of_single_places_do_not_count():
    plan, table, scores = call()
    one = scores[:1, :, :1]  # a sample, a query: whatever their strides
    want = plan.forward(table, scores=one.contiguous())
    plan.forward(table, scores=one, out=one.as_strided((1, 2, 1, 8), (7, one.stride(1), 5, 1)))
    assert torch.equal(one, want)


def test_outputs_whose_elements_share_memory_are_refused():
    plan, table, scores = call()
    for out in (torch.zeros(1, 2, 4, 8).cuda().expand(3, 2, 4, 8), torch.zeros(3, 1, 4, 8).cuda().expand(3, 2, 4, 8), torch.zeros(3, 2, 1, 8).cuda().expand(3, 2, 4, 8)):
        with pytest.raises(ValueError):
            plan.forward(table, scores=scores, out=out)


def test_gradient_in_place():
    from paper_2305_01515_amd.dense import BiasShape, BiasStrides, _lib
    plan, table, dout = call()
    shape = BiasShape(3, 4, 8, 0, None, None, 0, 0, None, 0, 0)
    kept = dout.clone()
    same, other = BiasStrides(*dout.stride()[:3]), BiasStrides(64, 8, 16)
    p, s = dout.data_ptr(), torch.cuda.current_stream().cuda_stream
    assert _lib().tbe_bias_backward(plan._h, C.byref(shape), p, C.byref(same), None, 0.5, p, C.byref(other), s) == -1
    assert torch.equal(dout, kept)
    assert _lib().tbe_bias_backward(plan._h, C.byref(shape), p, C.byref(same), None, 0.5, p, C.byref(same), s) == 0
    assert torch.equal(dout, kept * 0.5)
