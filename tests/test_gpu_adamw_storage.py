"""A step updates the parameters, copies and states that the object has then, not the memory that they had when it was made.  (What was there before is kept
here, so that nothing else gets its place.)"""
import copy

import pytest
import torch

pytestmark = pytest.mark.gpu
SIZES = [300, 5, 1000]


def both(bits, dtype=torch.bfloat16, master=True):
    """two optimizers in the same state, after a step, and the next gradients"""
    from paper_2305_01515_amd.dense import AdamW
    g = torch.Generator().manual_seed(bits)
    start = [torch.randn(n, generator=g).to(dtype) for n in SIZES]
    grads = [[torch.randn(n, generator=g).to(dtype).cuda() for n in SIZES] for _ in range(3)]
    pair = [AdamW([torch.nn.Parameter(p.cuda()) for p in start], lr=1e-2, state_bits=bits, seed=3, master=master) for _ in range(2)]
    for opt in pair:
        opt.step(grads[0])
    return (*pair, grads)


def same(a, b):
    for x, y in zip(a.params + [w for w in a.master if w is not None] + list(a.states.values()), b.params + [w for w in b.master if w is not None] + list(b.states.values())):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_with_another_storage(bits):
    one, two, grads = both(bits)
    kept = [p.data for p in one.params]
    old = [k.clone() for k in kept]
    for p in one.params:
        p.data = p.data.clone()  # as model.cpu().cuda(), or a loader that assigns
    for gs in grads[1:]:
        one.step(gs)
        two.step(gs)
    same(one, two)
    for k, o in zip(kept, old):
        assert torch.equal(k, o)


@pytest.mark.parametrize("bits", [32, 8])
def test_replaced_states_and_copies(bits):
    one, two, grads = both(bits)
    kept = dict(one.states), list(one.master)
    old = copy.deepcopy(kept)
    for k in one.states:
        one.states[k] = one.states[k].clone()
    one.master[1] = one.master[1].clone()
    for gs in grads[1:]:
        one.step(gs)
        two.step(gs)
    same(one, two)
    for k in kept[0]:
        assert torch.equal(kept[0][k], old[0][k])
    assert torch.equal(kept[1][1], old[1][1])


def test_a_checkpoint_put_into_the_states():
    """the states of one run into another run's object, by assignment: it goes on as that one"""
    one, two, grads = both(8)
    kept = dict(two.states)
    one.step(grads[1])
    two.states.update({k: v.clone() for k, v in one.states.items()})
    for p, q in zip(two.params, one.params):
        p.data = q.data.clone()
    two.master = [w.clone() for w in one.master]
    two.step_count = one.step_count
    one.step(grads[2])
    two.step(grads[2])
    same(one, two)
    assert kept


def test_parameters_of_another_type():
    """a model turned to 16 bits after the object was made: its weights are read and written as what they are"""
    from paper_2305_01515_amd.dense import AdamW
    one, _, grads = both(32, torch.float32, None)
    kept = [p.data for p in one.params]
    two = AdamW([torch.nn.Parameter(p.data.bfloat16()) for p in one.params], lr=1e-2, seed=3, step=1, states={k: v.clone() for k, v in one.states.items()},
                grad_dtypes=[torch.float32] * 3)
    for p in one.params:
        p.data = p.data.bfloat16()
    one.step(grads[1])
    two.step(grads[1])
    assert one.params[0].dtype == torch.bfloat16
    same(one, two)
    assert len(kept) == 3


def test_what_is_refused():
    one, _, grads = both(8)
    saved = [p.data for p in one.params]
    for bad in (torch.zeros(2000).bfloat16().cuda(), saved[0].cpu(), torch.zeros(600).bfloat16().cuda()[::2]):
        one.params[0].data = bad
        with pytest.raises(ValueError):
            one.step([torch.zeros_like(bad), *grads[1][1:]] if bad.shape != saved[0].shape else grads[1])
        one.params[0].data = saved[0]
    for name, bad in (("m", one.states["m"][:-1]), ("v_scale", one.states["v_scale"].cpu()), ("v", one.states["v"].float())):
        good = one.states[name]
        one.states[name] = bad
        with pytest.raises(ValueError):
            one.step(grads[1])
        one.states[name] = good
    one.master.append(None)
    with pytest.raises(ValueError):
        one.step(grads[1])
    one.master.pop()
    assert one.step_count == 1
    one.step(grads[1])
