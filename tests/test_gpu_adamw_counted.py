"""Steps whose number is counted on the GPU: replays of a captured one are the steps 1, 2, 3, ... that eager calls take.

Bars.  The moving averages and their codes go by the gradients, the betas and the step's random key: the same bits.  Weights go by two factors
of the step's number besides, which host and GPU compute in double and round to fp32: two of them may differ in the last bit, an update by 2 eps
of itself, a weight after n steps by what n such updates and as many roundings of the weight add."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
SIZES = [300, 5, 4097, 70_001]
LR = 1e-2


def make(bits, capturable, seed=1, sizes=SIZES, **kw):
    from paper_2305_01515_amd.dense import AdamW
    g = torch.Generator().manual_seed(seed)
    params = [torch.randn(n, generator=g).cuda() for n in sizes]
    return AdamW(params, lr=LR, weight_decay=0.01, state_bits=bits, seed=5, capturable=capturable, **kw)


def gradients(count, sizes=SIZES):
    g = torch.Generator().manual_seed(9)
    return [[torch.randn(n, generator=g).cuda() * (10.0 ** -(k % 3)) for n in sizes] for k in range(count)]


def compare(counted, eager, steps):
    assert counted.step_count == eager.step_count == steps
    for k in eager.states:
        assert torch.equal(counted.states[k], eager.states[k]), k
    for p, q in zip(counted.params, eager.params):
        # |m| / sqrt(v) of bias-corrected averages is at most sqrt of the steps here (one gradient with zeros around it)
        bar = steps * (2 * EPS * (q.abs().max() + 1) + 4 * EPS * LR * (steps ** 0.5 + 1))
        assert (p.double() - q.double()).abs().max() <= bar


@pytest.mark.parametrize("bits", [32, 8])
def test_eager_steps(bits):
    one, two = make(bits, True), make(bits, False)
    for k, gs in enumerate(gradients(6)):
        one.step(gs)
        two.step(gs)
        compare(one, two, k + 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_replays_are_the_steps_of_eager_calls(bits):
    """captured once, replayed with eager work, eager steps and synchronizations between the replays"""
    one, two = make(bits, True), make(bits, False)
    grads = gradients(9)
    held = [torch.empty_like(g) for g in grads[0]]
    one.step(grads[0])
    two.step(grads[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(held)
    compare(one, two, 1)  # capturing is no step
    for k, gs in enumerate(grads[1:], 1):
        two.step(gs)
        if k == 4:
            one.step(gs)
        else:
            for h, g in zip(held, gs):
                h.copy_(g)
            graph.replay()
        if k % 2:
            torch.cuda.synchronize()
            float(sum(h.sum() for h in held))
        compare(one, two, k + 1)


def test_draws_of_replays_differ():
    """no gradient, beta2 = 0.99: sqrt(v) falls by half a percent a step, a tenth of a code's gap, which only draws that differ follow"""
    from paper_2305_01515_amd.dense import AdamW
    p = torch.zeros(64 * 256).cuda()
    opt = AdamW([p], lr=0.0, betas=(0.9, 0.99), weight_decay=0.0, state_bits=8, seed=5, capturable=True)
    g = torch.randn(p.shape, generator=torch.Generator().manual_seed(1)).cuda()
    value = lambda: float((opt.states["v"].view(torch.float8_e4m3fn).float().view(-1, 256) * opt.states["v_scale"][:, None]).double().mean())  # noqa: E731
    opt.step([g])
    before = value()
    g.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
    for _ in range(40):
        graph.replay()
    assert abs(value() / before / 0.99 ** 20 - 1) < 0.006  # 6 standard deviations of the mean of 16384 elements off by 1/8 at most
    assert opt.step_count == 41


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes(bits):
    """two launches, one step"""
    sizes = [1 + 37 * (k % 11) for k in range(300)]
    one, two = make(bits, True, sizes=sizes), make(bits, False, sizes=sizes)
    for gs in gradients(2, sizes):
        gs[7] = gs[299] = None
        one.step(gs)
        two.step(gs)
    compare(one, two, 2)


def test_the_number_in_the_states():
    grads = gradients(5)
    one, two = make(8, True), make(8, False)
    for gs in grads[:2]:
        one.step(gs)
        two.step(gs)
    # put into a new object, with the number among the states
    three = make(8, True, seed=2, states={k: v.clone() for k, v in one.states.items()})
    for p, q in zip(three.params, one.params):
        p.copy_(q)
    three.step(grads[2])
    two.step(grads[2])
    compare(three, two, 3)
    three.step_count, two.step_count = 7, 7
    three.step(grads[3])
    two.step(grads[3])
    compare(three, two, 8)
    one.states["step"].fill_(-5)
    one.step(grads[2])
    assert one.step_count == 1
    other = make(8, True, step=4)
    assert other.step_count == 4
    for bad in (torch.zeros(1).cuda(), torch.zeros(2, dtype=torch.int64).cuda(), torch.zeros(1, dtype=torch.int64)):
        other.states["step"] = bad
        with pytest.raises(ValueError):
            other.step(grads[0])


def test_a_captured_step_with_a_number_from_the_host_warns():
    opt = make(32, False)
    gs = gradients(1)[0]
    torch.cuda.synchronize()
    with pytest.warns(UserWarning, match="capturable"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            opt.step(gs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    import warnings
    with warnings.catch_warnings(), torch.cuda.stream(side):
        warnings.simplefilter("error")
        opt.step(gs)
    torch.cuda.synchronize()
    assert np.isfinite(opt.params[0].cpu().numpy()).all()
