"""The first step on another stream than the constructor's waits for what the constructor enqueued there: zeros of the states, fp32 copies."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_on_another_stream(bits):
    from paper_2305_01515_amd.dense import AdamW
    n, g = 50_000, torch.Generator().manual_seed(bits)
    start, grad = torch.randn(n, generator=g).bfloat16().cuda(), torch.randn(n, generator=g).bfloat16().cuda()
    p, q = start.clone(), start.clone()
    want = AdamW([q], lr=1e-2, state_bits=bits, master=True)
    want.step([grad])
    a = torch.randn(8192, 8192, device="cuda").bfloat16()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        poison = [torch.full((1 << 18,), 7.0, device="cuda") for _ in range(8)]  # what the constructor gets as memory for states holds no zeros
        del poison
        for _ in range(40):  # some 40 ms in front of what the constructor enqueues
            a @ a
        opt = AdamW([p], lr=1e-2, state_bits=bits, master=True)
    with torch.cuda.stream(two):
        opt.step([grad])
    torch.cuda.synchronize()
    assert torch.equal(p, q) and torch.equal(opt.master[0], want.master[0])
    for k in opt.states:
        assert torch.equal(opt.states[k], want.states[k])
