"""What a call of the norm, the short convolution or the selective scan writes may not overlap what it reads: refused before anything is enqueued, wherever the
strides tell; columns side by side in one piece of memory, and what the header allows in place, go on."""
import pytest
import torch

from rows_util import offsets

pytestmark = pytest.mark.gpu
ROWS, DIM = 24, 8


def room(columns, dtype=torch.float32):
    g = torch.Generator().manual_seed(columns)
    return torch.randn(2 * ROWS, columns, generator=g).to(dtype).cuda()


def refused(call):
    from paper_2305_01515_amd.tbe import TbeError
    with pytest.raises(TbeError, match="overlaps|in place of an input"):
        call()


def test_norm():
    from paper_2305_01515_amd.dense import RMSNorm
    plan, w, store = RMSNorm(DIM, torch.float32, ROWS, residual_dtype=torch.float32), torch.ones(DIM, device="cuda"), room(3 * DIM)
    x, r, free = store[:ROWS, :DIM], store[:ROWS, DIM:2 * DIM], store[:ROWS, 2 * DIM:]
    want = plan.forward(x, w, r)
    one = room(DIM)
    for out in (store[:ROWS, 4:4 + DIM], store[1:ROWS + 1, :DIM], store[:ROWS, 12:12 + DIM], store.view(-1)[8:8 + ROWS * DIM].view(ROWS, DIM)):
        refused(lambda: plan.forward(x, w, r, out=out))
        refused(lambda: plan.forward(x, w, r, summed=out))
    refused(lambda: plan.forward(one[:ROWS], w, r, summed=one[1:ROWS + 1]))
    refused(lambda: plan.forward(x, w, r, out=free, summed=free))
    refused(lambda: plan.forward(x, one.view(-1)[4:4 + DIM], r, out=one[:ROWS]))
    refused(lambda: plan.quantise(x, w, r, codes=store.view(torch.float8_e4m3fn)[:ROWS, 20:20 + DIM]))
    out, _, _ = plan.forward(x, w, r, out=free)  # beside them
    assert torch.equal(out, want[0])
    r0 = r.clone()
    assert plan.forward(x, w, r, summed=r)[1] is r and torch.equal(r, want[1])
    r.copy_(r0)
    assert plan.forward(x, w, r, summed=x)[1] is x and torch.equal(x, want[1])


def test_conv():
    from paper_2305_01515_amd.dense import ShortConv
    store, w, off = room(3 * DIM), torch.ones(DIM, 3, device="cuda"), offsets([20, 4]).cuda()
    plan, x = ShortConv(DIM, 3, torch.float32, 2, ROWS), store[:ROWS, :DIM]
    want = plan.forward(x, off, w)[0]
    one = room(DIM)
    before = one.view(-1)[:2 * 2 * DIM].view(2, 2, DIM)
    for y in (x, store[:ROWS, 7:7 + DIM], store[2:ROWS + 2, :DIM], store.view(-1)[40:40 + ROWS * DIM].view(ROWS, DIM)):
        refused(lambda: plan.forward(x, off, w, y=y))
    refused(lambda: plan.forward(one[3:ROWS + 3], off, w, y=one[:ROWS]))
    refused(lambda: plan.forward(x, off, w, before=before, y=one[:ROWS]))
    refused(lambda: plan.forward(x, off, one.view(-1)[9:9 + 3 * DIM].view(DIM, 3), y=one[:ROWS]))
    assert torch.equal(plan.forward(x, off, w, y=store[:ROWS, 8:16])[0], want)  # beside it
    state = one.view(-1)[:ROWS * 2 * DIM].view(ROWS, 2, DIM)
    refused(lambda: plan.step(state, one[:ROWS], w))
    refused(lambda: plan.step(state, x, w, y=one[ROWS:]))
    refused(lambda: plan.step(state, store[:ROWS, :DIM], w, y=store[:ROWS, 4:4 + DIM]))
    a, b = state.clone(), state.clone()
    want = plan.step(a, x, w)
    assert torch.equal(plan.step(b, x, w, y=x), want) and torch.equal(a, b)  # in place


def test_ssm():
    from paper_2305_01515_amd.dense import SelectiveScan
    store, a, off = room(6 * DIM), -torch.ones(DIM, 8, device="cuda"), offsets([20, 4]).cuda()
    plan = SelectiveScan(DIM, 8, torch.float32, 2, ROWS)
    x, delta, b, c, z = (store[:ROWS, k * DIM:(k + 1) * DIM] for k in range(5))
    want = plan.forward(x, delta, a, b, c, off, z=z)[0]
    one = room(DIM)
    for y in (x, delta, b, c, z, store[:ROWS, 5:5 + DIM], store[4:ROWS + 4, 28:28 + DIM], store.view(-1)[40:40 + ROWS * DIM].view(ROWS, DIM)):
        refused(lambda: plan.forward(x, delta, a, b, c, off, z=z, y=y))
    refused(lambda: plan.forward(one[3:ROWS + 3], delta, a, b, c, off, y=one[:ROWS]))
    refused(lambda: plan.forward(x, delta, a, b, c, off, h0=one.view(-1)[:2 * DIM * 8].view(2, DIM, 8), y=one[:ROWS]))
    refused(lambda: plan.forward(x, delta, a, b, c, off, skip=one[5], y=one[:ROWS]))
    assert torch.equal(plan.forward(x, delta, a, b, c, off, z=z, y=store[:ROWS, 40:])[0], want)  # beside them
    states = room(DIM * 8)
    state = states[:ROWS].view(ROWS, DIM, 8)
    refused(lambda: plan.step(state, x, delta, a, b, c, y=states.view(-1)[8:8 + ROWS * DIM].view(ROWS, DIM)))
    refused(lambda: plan.step(state, states[:ROWS, 8:16], delta, a, b, c))
    for y in (b, c, store[:ROWS, 4:4 + DIM]):
        refused(lambda: plan.step(state, x, delta, a, b, c, z=z, y=y))
    one, two = state.clone(), state.clone()
    want = plan.step(one, x, delta, a, b, c, z=z)
    assert torch.equal(plan.step(two, x, delta, a, b, c, z=z, y=z), want) and torch.equal(one, two)  # in place
