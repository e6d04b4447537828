"""The short convolution over bags against its formula in 64 bits.

Bars.  eps = 2^-24.  v is a sum of width + 1 terms in any order: (width + 1) eps of their magnitudes.  A sigmoid is off by (|v| + 8) eps of itself, silu has a slope of at
most 1.1, its derivative one of at most 0.5 and an error of 3 (|v| + 8) (1 + |v|) eps of the sigmoid.  Sums over n rows add (n + 100) eps of
their magnitudes.  A result stored in 16 bits adds half a step of its own."""
import numpy as np
import pytest
import torch

from rows_util import EPS, RAGGED, TYPES, f64, near, offsets, placed, sigmoid

pytestmark = pytest.mark.gpu


def reference(lengths, x, w, bias, before, dy, dlast, silu):
    """{name: (value, bar)}, numpy float64, bag by bag"""
    (R, D), W, B = x.shape, w.shape[1], len(lengths)
    off = np.concatenate([[0], np.cumsum(lengths)])
    y, ey, dx, ex = (np.zeros((R, D)) for _ in range(4))
    last, dbefore, ebefore = (np.zeros((B, W - 1, D)) for _ in range(3))
    dw, mw, ew = (np.zeros((D, W)) for _ in range(3))
    db, mb, eb = (np.zeros(D) for _ in range(3))
    bias = np.zeros(D) if bias is None else bias
    for b in range(B):
        s = slice(off[b], off[b + 1])
        n = lengths[b]
        e = np.concatenate([np.zeros((W - 1, D)) if before is None else before[b], x[s]])
        last[b] = e[len(e) - (W - 1):]
        v = bias + sum(w[:, j] * e[j:j + n] for j in range(W))
        ev = (W + 1) * EPS * (np.abs(bias) + sum(np.abs(w[:, j] * e[j:j + n]) for j in range(W)))
        f = sigmoid(v)
        if silu:
            y[s], ey[s] = v * f, 1.1 * ev + (np.abs(v) + 10) * EPS * np.abs(v * f)
            slope = f * (1 + v * (1 - f))
            es = 0.5 * ev + 3 * (np.abs(v) + 8) * (1 + np.abs(v)) * EPS * f
        else:
            y[s], ey[s], slope, es = v, ev, 1.0, 0.0
        g, eg = dy[s] * slope, np.abs(dy[s]) * es + 2 * EPS * np.abs(dy[s] * slope)
        de, ee = np.zeros_like(e), np.zeros_like(e)
        for j in range(W):
            de[j:j + n] += w[:, j] * g
            ee[j:j + n] += np.abs(w[:, j]) * (eg + (W + 2) * EPS * np.abs(g))
            dw[:, j] += (g * e[j:j + n]).sum(0)
            mw[:, j] += np.abs(g * e[j:j + n]).sum(0)
            ew[:, j] += (eg * np.abs(e[j:j + n])).sum(0)
        db, mb, eb = db + g.sum(0), mb + np.abs(g).sum(0), eb + eg.sum(0)
        if dlast is not None:
            de[len(e) - (W - 1):] += dlast[b]
            ee[len(e) - (W - 1):] += EPS * (np.abs(de) + np.abs(ee))[len(e) - (W - 1):] + EPS * np.abs(dlast[b])
        dx[s], ex[s] = de[W - 1:], ee[W - 1:]
        dbefore[b], ebefore[b] = de[:W - 1], ee[:W - 1]
    many = (R + 100) * EPS
    return {"y": (y, ey), "last": last, "dx": (dx, ex), "dweight": (dw, ew + many * mw), "dbias": (db, eb + many * mb), "dbefore": (dbefore, ebefore)}


def inputs(rows, bags, dim, width, dtype, weights, seed):
    g = torch.Generator().manual_seed(seed)
    dt, wt = TYPES[dtype][0], TYPES[weights][0]
    t = {k: torch.randn(rows, dim, generator=g).to(dt) for k in ("x", "dy")}
    t |= {k: torch.randn(bags, width - 1, dim, generator=g).to(dt) for k in ("before", "dlast")}
    return t | {"weight": torch.randn(dim, width, generator=g).to(wt), "bias": torch.randn(dim, generator=g).to(wt)}


def run_and_compare(lengths, dim, width=4, dtype="f32", weights="f32", silu=True, leave=(), layout="plain", seed=0):
    from paper_2305_01515_amd.dense import ShortConv
    rows, bags = int(sum(lengths)), len(lengths)
    t = inputs(rows, bags, dim, width, dtype, weights, seed) | {k: None for k in leave}
    want = reference(lengths, *(f64(t[k]) for k in ("x", "weight", "bias", "before", "dy", "dlast")), silu)
    gpu = {k: placed(v, layout) if k in ("x", "dy") else None if v is None else v.cuda() for k, v in t.items()}
    plan, off = ShortConv(dim, width, TYPES[dtype][0], bags, rows, silu), offsets(lengths).cuda()
    y, last = plan.forward(gpu["x"], off, gpu["weight"], gpu["bias"], gpu["before"])
    got = plan.backward(gpu["x"], off, gpu["weight"], gpu["dy"], gpu["bias"], gpu["before"], gpu["dlast"])
    plan.check()
    near("y", y, *want["y"], dtype)
    assert np.array_equal(f64(last), want["last"])
    for name, v, kind in zip(("dx", "dweight", "dbias", "dbefore"), got, (dtype, "f32", "f32", dtype)):
        if v is None:
            assert name[1:] in leave
        else:
            near(name, v, *want[name], kind)
    return plan, gpu, off, (y, last, got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,width,layout,weights,silu,leave", [
    (64, 4, "plain", "f32", True, ()), (128, 4, "wide", "own", True, ("before",)), (1, 2, "plain", "f32", False, ()), (7, 3, "shifted", "own", True, ("bias",)),
    (33, 8, "plain", "f32", True, ()), (100, 5, "shifted", "f32", True, ("dlast",)), (16, 1, "plain", "f32", True, ("bias",)), (2500, 4, "plain", "f32", True, ()),
    (20, 6, "wide", "f32", False, ("before", "bias", "dlast")), (9, 7, "plain", "own", True, ())])
def test_ragged_bags(dim, width, layout, weights, silu, leave, dtype):
    run_and_compare(RAGGED, dim, width, dtype, dtype if weights == "own" else weights, silu, leave, layout, seed=dim)


@pytest.mark.parametrize("lengths", [[1], [0], [0, 0, 0], [3], [5000], [1] * 300, [2, 1, 0, 3, 1, 1, 2] * 30, [0] * 300 + [3] + [0] * 300, [4000, 0, 5000, 1], [4096, 4096],
                                     [16] * 40, [15, 1, 16, 17, 31]], ids=lambda v: f"{len(v)}x{max(v)}")
@pytest.mark.parametrize("width", [2, 4, 8])
def test_lengths(lengths, width):
    run_and_compare(lengths, 24, width, seed=len(lengths))
    run_and_compare(lengths, 3, width, "bf16", "bf16", seed=len(lengths) + 1)


def test_a_bag_in_two_parts():
    """what a bag's first part leaves is what its second goes on from: the same bits as in one"""
    from paper_2305_01515_amd.dense import ShortConv
    t = {k: v.cuda() for k, v in inputs(300, 3, 40, 4, "bf16", "f32", 1).items()}
    plan = ShortConv(40, 4, torch.bfloat16, 3, 300)
    y, last = plan.forward(t["x"], offsets([100, 2, 198]).cuda(), t["weight"], t["bias"], t["before"])
    first, second = [0, 1, 150], [100, 1, 48]
    at, parts = 0, [[], []]
    for n, m in zip(first, second):
        parts[0].append(t["x"][at:at + n])
        parts[1].append(t["x"][at + n:at + n + m])
        at += n + m
    y1, last1 = plan.forward(torch.cat(parts[0]), offsets(first).cuda(), t["weight"], t["bias"], t["before"])
    y2, last2 = plan.forward(torch.cat(parts[1]), offsets(second).cuda(), t["weight"], t["bias"], last1)
    assert torch.equal(last2, last)
    both = [v for n, m, a, b in zip(first, second, y1.split(first), y2.split(second)) for v in (a, b)]
    assert torch.equal(torch.cat(both), y)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,width", [(64, 4), (5, 2), (130, 8), (1, 1), (33, 3)])
def test_step_goes_on_where_bags_end(dim, width, dtype):
    from paper_2305_01515_amd.dense import ShortConv
    t = {k: v.cuda() for k, v in inputs(12, 12, dim, width, dtype, "f32", 3).items()}
    plan = ShortConv(dim, width, TYPES[dtype][0], 12, 12)
    y, last = plan.forward(t["x"], offsets([1] * 12).cuda(), t["weight"], t["bias"], t["before"])
    store = torch.full((20, width - 1, dim), 3.0, dtype=t["x"].dtype, device="cuda")
    slots = torch.arange(18, 6, -1, device="cuda")
    slots[3] = -1
    there = slots >= 0
    store[slots[there]] = t["before"][there]
    got = plan.step(store, t["x"], t["weight"], t["bias"], slots=slots)
    plan.check()
    assert torch.equal(got[there], y[there]) and (got[3] == 0).all() and torch.equal(store[slots[there]], last[there])
    untouched = [i for i in range(20) if i not in slots.tolist()]
    assert (store[untouched] == 3).all()


@pytest.mark.parametrize("dim,width,dtype", [(4096, 4, "f32"), (4096, 8, "f32"), (1024, 4, "bf16"), (8190, 3, "f16")])
def test_more_tiles_than_workgroups_of_the_backward(dim, width, dtype):
    """each walks a second tile, with the marks and the sums of the first one behind it"""
    rows = {1024: 9000, 4096: 1300, 8190: 1400}[dim]
    lengths = [rows - 320, 0, 1, 2, 7, 9, 300, 1]
    run_and_compare(lengths, dim, width, dtype, seed=dim + width)


def test_silu_over_its_range():
    """What the header says of a sigmoid, to the end of its range: v log2(e) is rounded (|v| eps of the exponential), log2(e) in 32 bits is 0.224 eps of itself too small
    (0.224 |v| eps); exponential, sum, quotient and product round to within some eps each.  So (1.25 |v| + 8) eps of the sigmoid and one of the product."""
    from paper_2305_01515_amd.dense import ShortConv
    v = torch.linspace(-86, 86, 1 << 22, dtype=torch.float64).float().view(-1, 64)
    plan = ShortConv(64, 1, torch.float32, 1, len(v))
    y, _ = plan.forward(v.cuda(), offsets([len(v)]).cuda(), torch.ones(64, 1, device="cuda"))
    d = f64(v)
    near("silu", y, d * sigmoid(d), (1.25 * np.abs(d) + 9) * EPS * np.abs(d * sigmoid(d)))


def test_more_elements_of_earlier_rows_than_a_launch_has_lanes():
    """2^32 of them and more: the gradient of an empty bag's earlier rows is that of its last ones, the others' what a call of these bags alone gives"""
    from paper_2305_01515_amd.dense import ShortConv
    bags, width, dim, rows = 9400, 8, 65536, 5
    assert bags * (width - 1) * dim > 1 << 32
    if torch.cuda.mem_get_info()[0] < 5 * bags * (width - 1) * dim * 2:
        pytest.skip("takes 35 GB")
    t = {k: v.cuda() for k, v in inputs(rows, 2, dim, width, "bf16", "f32", 21).items()}
    before, dlast = (torch.zeros(bags, width - 1, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dlast += torch.arange(bags, device="cuda")[:, None, None] % 251
    ends = torch.tensor([0, bags - 1], device="cuda")
    before[ends], dlast[ends] = t["before"], t["dlast"]
    few, many = ShortConv(dim, width, torch.bfloat16, 2, rows), ShortConv(dim, width, torch.bfloat16, bags, rows)
    want = few.backward(t["x"], offsets([2, 3]).cuda(), t["weight"], t["dy"], t["bias"], t["before"], t["dlast"])
    got = many.backward(t["x"], offsets([2] + [0] * (bags - 2) + [3]).cuda(), t["weight"], t["dy"], t["bias"], before, dlast)
    many.check()
    for v, w in zip(got[:3], want[:3]):
        assert torch.equal(v, w)
    assert torch.equal(got[3][ends], want[3])
    for k in range(1, bags - 1, 1000):
        assert torch.equal(got[3][k:min(k + 1000, bags - 1)], dlast[k:min(k + 1000, bags - 1)])


@pytest.mark.parametrize("lengths", [[17, 0, 40], []])
def test_each_gradient_of_the_weights_alone(lengths):
    """the C entry point takes null for either: the other one has the same bits as with it"""
    import ctypes as C

    from paper_2305_01515_amd import dense
    rows, bags = sum(lengths), len(lengths)
    t = {k: v.cuda() for k, v in inputs(rows, bags, 70, 4, "f32", "f32", 4).items()}
    plan, off = dense.ShortConv(70, 4, torch.float32, bags, rows), offsets(lengths).cuda()
    batch = plan._batch(t["x"], off, t["weight"], t["bias"], None)

    def grads(weight, bias):
        dx, dw, db = torch.empty_like(t["x"]), torch.full((70, 4), 7.0, device="cuda"), torch.full((70,), 7.0, device="cuda")
        assert dense._lib().tbe_conv_backward(plan._h, C.byref(batch), t["dy"].data_ptr(), 70, None, dx.data_ptr(), 70, dw.data_ptr() if weight else None,
                                              db.data_ptr() if bias else None, None, plan._stream()) == 0
        return dx, dw, db
    want = grads(True, True)
    assert rows or not (want[1].any() or want[2].any())
    for weight, bias in ((True, False), (False, True), (False, False)):
        dx, dw, db = grads(weight, bias)
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1] if weight else torch.full_like(dw, 7.0)) and torch.equal(db, want[2] if bias else torch.full_like(db, 7.0))


def test_an_infinity_stays_in_its_bag():
    from paper_2305_01515_amd.dense import ShortConv
    t = {k: v.cuda() for k, v in inputs(60, 3, 8, 4, "f32", "f32", 3).items()}
    plan, off = ShortConv(8, 4, torch.float32, 3, 60), offsets([20, 20, 20]).cuda()
    y, last = plan.forward(t["x"], off, t["weight"], t["bias"])
    clean = plan.backward(t["x"], off, t["weight"], t["dy"], t["bias"])[0]
    t["x"][39], t["dy"][39] = float("inf"), float("nan")
    y2, _ = plan.forward(t["x"], off, t["weight"], t["bias"])
    dx = plan.backward(t["x"], off, t["weight"], t["dy"], t["bias"])[0]
    rest = torch.arange(60, device="cuda") != 39
    assert torch.equal(y[rest], y2[rest]) and torch.equal(dx[:36], clean[:36]) and torch.equal(dx[40:], clean[40:])


def test_the_same_bits_again_and_in_graphs():
    plan, gpu, off, (y, last, got) = run_and_compare([700, 3, 0, 40, 129], 72, 4, dtype="bf16", seed=4)

    def both():
        y, last = plan.forward(gpu["x"], off, gpu["weight"], gpu["bias"], gpu["before"])
        return [y, last, *plan.backward(gpu["x"], off, gpu["weight"], gpu["dy"], gpu["bias"], gpu["before"], gpu["dlast"])]
    want = both()
    for v, w in zip(want, [y, last, *got]):
        assert torch.equal(v, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(4):
        for v in out:
            v.zero_()
        graph.replay()
        for v, w in zip(out, want):
            assert torch.equal(v, w)
        plan.forward(gpu["x"][:7], offsets([5, 2]).cuda(), gpu["weight"])
        torch.cuda.synchronize()


def test_gradients_through_autograd():
    from paper_2305_01515_amd.dense import ShortConv
    lengths, names = [5, 0, 2, 9], ("x", "weight", "bias", "before")
    t = inputs(16, 4, 6, 4, "f32", "f32", 8)

    def loss(v):
        want = reference(lengths, v["x"], v["weight"], v["bias"], v["before"], f64(t["dy"]), f64(t["dlast"]), True)
        return (want["y"][0] * f64(t["dy"])).sum() + (want["last"] * f64(t["dlast"])).sum()
    leaves = {k: t[k].cuda().requires_grad_() for k in names}
    plan = ShortConv(6, 4, torch.float32, 4, 16)
    y, last = plan(leaves["x"], offsets(lengths).cuda(), leaves["weight"], leaves["bias"], leaves["before"])
    ((y * t["dy"].cuda()).sum() + (last * t["dlast"].cuda()).sum()).backward()
    rs = np.random.RandomState(0)
    for k in names:
        way, v, step = rs.standard_normal(t[k].shape), {n: f64(t[n]) for n in names}, 1e-6
        slope = (loss(dict(v, **{k: v[k] + step * way})) - loss(dict(v, **{k: v[k] - step * way}))) / (2 * step)
        # differences: step^2 of the third derivative, and 2^-53 of the loss over the step; gradients: some hundred eps of their magnitudes
        assert abs(slope - (f64(leaves[k].grad) * way).sum()) <= 1e-5 * (np.abs(f64(leaves[k].grad) * way).sum() + 1), k
    y, _ = plan(leaves["x"], offsets(lengths).cuda(), leaves["weight"])
    y.sum().expand(()).backward()  # a gradient that is one number for all
    with pytest.raises(RuntimeError, match="once_differentiable"):
        y, _ = plan(leaves["x"], offsets(lengths).cuda(), leaves["weight"])
        g, = torch.autograd.grad((y ** 2).sum(), leaves["x"], create_graph=True)
        (g ** 2).sum().backward()


def test_what_is_refused():
    from paper_2305_01515_amd.dense import ShortConv
    from paper_2305_01515_amd.tbe import TbeError
    for bad in (dict(dim=0), dict(width=0), dict(width=9), dict(max_rows=-1)):
        with pytest.raises(TbeError):
            ShortConv(**{**dict(dim=64, width=4, dtype=torch.float32, max_bags=2, max_rows=9), **bad})
    with pytest.raises(ValueError):
        ShortConv(8, 4, torch.float64, 2, 9)
    plan, off = ShortConv(8, 4, torch.float32, 2, 9), offsets([4, 5]).cuda()
    t = {k: v.cuda() for k, v in inputs(9, 2, 8, 4, "f32", "f32", 1).items()}
    for x, o, w, b, e in ((t["x"].bfloat16(), off, t["weight"], None, None), (t["x"].t(), off, t["weight"], None, None), (t["x"], off.int(), t["weight"], None, None),
                          (t["x"], off, t["weight"].t().contiguous().t(), None, None), (t["x"], off, t["weight"], t["bias"].half(), None),
                          (t["x"], off, t["weight"], None, t["before"][:1]), (t["x"], off, t["weight"].double(), None, None)):
        with pytest.raises(ValueError):
            plan.forward(x, o, w, b, e)
    with pytest.raises(TbeError):
        plan.forward(t["x"], off, t["weight"], y=t["x"])
    with pytest.raises(TbeError):
        plan.forward(t["x"], offsets([3, 3, 3]).cuda(), t["weight"])
    for o in ([0, 6, 4], [1, 4, 9], [0, 4, 8]):
        plan.forward(t["x"], torch.tensor(o).cuda(), t["weight"])
        with pytest.raises(TbeError):
            plan.check()
        plan.backward(t["x"], torch.tensor(o).cuda(), t["weight"], t["dy"])
        with pytest.raises(TbeError):
            plan.check()
    plan.forward(t["x"], off, t["weight"])
    plan.check()
    state = torch.zeros(3, 3, 8, device="cuda")
    got = plan.step(state, t["x"][:2], t["weight"], slots=torch.tensor([1, 3]).cuda())
    with pytest.raises(TbeError):
        plan.check()
    assert (got[1] == 0).all() and (state[[0, 2]] == 0).all() and (state[1] != 0).any()
    with pytest.raises(TbeError):
        plan.step(state[:1], t["x"][:2], t["weight"])


def test_what_is_not_wanted_is_not_found():
    from paper_2305_01515_amd.dense import ShortConv
    t = {k: v.cuda() for k, v in inputs(300, 3, 40, 4, "bf16", "f32", 6).items()}
    plan, off = ShortConv(40, 4, torch.bfloat16, 3, 300), offsets([200, 0, 100]).cuda()
    y, last = plan.forward(t["x"], off, t["weight"])
    given = torch.full((300, 50), 5.0, dtype=torch.bfloat16, device="cuda")
    y2, none = plan.forward(t["x"], off, t["weight"], y=given[:, 3:43], want_last=False)
    assert none is None and torch.equal(y, y2) and (given[:, :3] == 5).all() and (given[:, 43:] == 5).all()
    for v, w in zip(plan.backward(t["x"], off, t["weight"], t["dy"]), plan.backward(t["x"], off, t["weight"], t["dy"], dlast=torch.zeros_like(last))):
        assert v is w is None or torch.equal(v, w)
