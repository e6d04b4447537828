"""Rows, scores and weights whose places do not fit 32 bits: the same bits as from a compact copy."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def far(t, stride):
    """t's rows, `stride` elements apart"""
    room = torch.empty((t.shape[0] - 1) * stride + t.shape[1], dtype=t.dtype, device="cuda")
    v = room.as_strided(t.shape, (stride, 1))
    v.copy_(t)
    return v


@pytest.mark.parametrize("lengths", [[200, 0, 400, 1], [600], [3] * 200])
def test_scan_rows_far_apart(lengths):
    from paper_2305_01515_amd.dense import Scan
    n, dim, stride = sum(lengths), 64, 1 << 22  # 2.5 G elements
    g = torch.Generator().manual_seed(1)
    x, u, dy = (torch.randn(n, dim, generator=g).bfloat16().cuda() for _ in range(3))
    off = torch.tensor([0] + lengths).cumsum(0).cuda()
    plan = Scan(dim, torch.bfloat16, len(lengths), n)
    y, last, saved = plan.forward(x, u, off, save=True)
    want = plan.backward(x, u, off, saved, dy, last)
    fx, fu, fy = far(x, stride), far(u, stride), torch.empty((n - 1) * stride + dim, dtype=torch.bfloat16, device="cuda").as_strided((n, dim), (stride, 1))
    y2, last2, saved2 = plan.forward(fx, fu, off, y=fy, save=True)
    assert torch.equal(y, y2) and torch.equal(last, last2) and torch.equal(saved, saved2)
    got = plan.backward(fx, fu, off, saved2, far(dy, stride), last2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_scan_states_far_apart():
    from paper_2305_01515_amd.dense import Scan
    dim, slots, stride = 64, 700, 1 << 22  # 2.9 G elements of fp32
    g = torch.Generator().manual_seed(2)
    state, x, u = (torch.randn(k, dim, generator=g).cuda() for k in (slots, 9, 9))
    slot = torch.tensor([699, 0, 650, 3, 512, 511, 640, 1, 698]).cuda()
    plan = Scan(dim, torch.float32, 9, 9)
    wide = far(state, stride)
    assert torch.equal(plan.step(wide, x, u, slot), plan.step(state, x, u, slot))
    assert torch.equal(wide, state)


@pytest.mark.parametrize("times", [False, True])
@pytest.mark.parametrize("keys", [64, 61])
def test_scores_far_apart(keys, times):
    from paper_2305_01515_amd.dense import RelativeBias
    b, h, q = 3, 2, 40
    g = torch.Generator().manual_seed(3)
    scores, table = torch.randn(b, h, q, keys, generator=g).half().cuda(), torch.randn(10, h, generator=g).cuda()
    strides = (1 << 30, 1 << 29, 1 << 23, 1)
    room = torch.empty(2 * (1 << 30) + (1 << 29) + 39 * (1 << 23) + keys, dtype=torch.float16, device="cuda")
    wide = room.as_strided(scores.shape, strides)
    wide.copy_(scores)
    where = dict(causal=True, key_lengths=torch.tensor([keys, 5, 30]).cuda())
    if times:
        t = torch.randint(0, 9, (b, keys), generator=g).cumsum(1).cuda()
        where.update(q_pos=t[:, :q].contiguous(), k_pos=t)
    plan = RelativeBias(h, [1, 2, 5, 20], bidirectional=True)
    want, grads = plan.forward(table, scores=scores, **where), plan.backward(scores, want_dscores=True, **where)
    got = plan.backward(wide, want_dscores=True, **where)
    assert torch.equal(got[0], grads[0]) and torch.equal(got[1], grads[1])
    assert torch.equal(plan.forward(table, scores=wide, out=wide, **where), want)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_of_more_than_2_31_weights(bits):
    """all weights alike: what becomes of one becomes of all, but that codes are drawn for each"""
    from paper_2305_01515_amd.dense import AdamW
    n = (1 << 31) + 5000
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 0.25, dtype=torch.bfloat16, device="cuda")
    opt = AdamW([p], lr=0.125, weight_decay=0.0, state_bits=bits)
    opt.step([g])
    assert float(p.min()) == float(p.max()) == 0.875
    for k in "mv":
        s = opt.states[k]
        assert bool((s[:n] == s[0]).all()) and not bool(s[n:].any())


def test_rows_of_almost_2_31_keys():
    """the last pack of a row ends at key 2^31: what is behind the row is neither counted nor written"""
    from paper_2305_01515_amd.dense import RelativeBias
    keys = (1 << 31) - 1
    plan = RelativeBias(1, [1, 1 << 20, 1 << 30])
    dout = torch.zeros(2, 1, 1, keys, dtype=torch.bfloat16, device="cuda")
    ends = torch.arange(1, 21, dtype=torch.bfloat16, device="cuda")
    dout[0, 0, 0, -20:], dout[1, 0, 0, :20], dout[1, 0, 0, -20:] = ends, 2 * ends, 4 * ends
    dtable, dscores = plan.backward(dout, q_offset=keys - 1, want_dscores=True, scale=0.5)
    assert dtable[:, 0].tolist() == [100.0, 950.0, 0.0, 420.0]  # the newest key, the 19 before it, the first ones
    dout *= 0.5
    assert torch.equal(dscores, dout)
    assert plan.backward(dout, q_offset=keys - 1)[:, 0].tolist() == [50.0, 475.0, 0.0, 210.0]


def test_more_weights_than_one_launch_takes():
    """2^24 workgroups of 1024 elements have 2^32 lanes, one more than a grid may have"""
    from paper_2305_01515_amd.dense import AdamW
    n = (1 << 34) + 3000
    p, g = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 0.25, dtype=torch.bfloat16, device="cuda")
    opt = AdamW([p], lr=0.125, weight_decay=0.0, state_bits=8)
    opt.step([g])
    assert float(p.min()) == float(p.max()) == 0.875 and opt.step_count == 1
    for k in "mv":
        s = opt.states[k]
        for part in s[:n].split(1 << 31):
            assert bool((part == s[0]).all())
        assert not bool(s[n:].any())


@pytest.mark.parametrize("slots", [False, True])
def test_more_states_than_one_launch_takes(slots):
    """2^32 elements and more, a lane each, one more than a grid may have; the same bits as two halves"""
    from paper_2305_01515_amd.dense import Scan
    dim, n = 128, (1 << 25) + 77
    plan = Scan(dim, torch.bfloat16, 1, 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, u = (torch.empty(n, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    state = torch.empty(n, dim, device="cuda").normal_(generator=g)
    other, half = state.clone(), n // 2
    slot = torch.arange(n - 1, -1, -1, device="cuda") if slots else None
    y = plan.step(state, x, u, slot)
    plan.check()
    if slots:
        first, last = plan.step(other, x[:half], u[:half], slot[:half]), plan.step(other, x[half:], u[half:], slot[half:])
    else:
        first, last = plan.step(other[:half], x[:half], u[:half]), plan.step(other[half:], x[half:], u[half:])
    assert torch.equal(y[:half], first) and torch.equal(y[half:], last) and torch.equal(state, other)
    assert bool((y[-1] != 0).all())


def test_a_gradient_of_more_rows_than_a_launch_takes_is_refused():
    """2^22 workgroups of 1024 lanes: one more than a grid may have; the forward's have 512.  Nothing is enqueued."""
    import ctypes as C
    from paper_2305_01515_amd import dense
    dim, rows = 65535, 1 << 19
    plan = dense.Scan(dim, torch.float16, 1, rows)
    off, t = torch.tensor([0, rows]).cuda(), torch.zeros(8).cuda()
    a = t.data_ptr()
    args = (plan._h, a, dim, a, dim, off.data_ptr(), 1, rows, None, 0, a, a, dim, None, a + 8, dim, a + 16, dim, None, None)
    assert dense._lib().tbe_scan_backward(*args) == -5
    assert b"one launch" in dense._lib().tbe_last_error(None)
    torch.cuda.synchronize()
    assert not bool(t.any())
