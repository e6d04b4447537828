"""The selective scan over bags against its formula in 64 bits, row by row.

Bars.  eps = 2^-24.  u = delta + bias is rounded once and its exponential is that of a rounded product, so D = softplus(u) is off by (2 |u| + 20) eps of
itself (e / (1 + e) is at most log(1 + e)).  A decay exp(D a) is off by |a| times that error and 2 (|D a| + 8) eps; where a bag is cut, the
decays' product is that of the sum of up to 128 D, which adds 128 eps |D a| a row.  A decay below the smallest normal number, 2^-126, becomes
zero (the hardware's power of two has no smaller results): LOST of what it is multiplied by.  M, the state that magnitudes would have, bounds what any order
of the sums adds: 4 eps M a row.  The error follows the recurrence of the state.  So does that of g, back.  A sum of n terms in any order adds n eps of
its magnitudes.  A result stored in 16 bits adds half a step of its own."""
import numpy as np
import pytest
import torch

from rows_util import EPS, RAGGED, TYPES, f64, near, offsets, placed, sigmoid

pytestmark = pytest.mark.gpu
LOST = 2.0 ** -126


def reference(lengths, x, delta, a, b, c, skip, bias, z, h0, dy, dlast, groups):
    """{name: (value, bar)}, numpy float64; b, c: [rows, groups, states]"""
    R, D = x.shape
    N, B, per = a.shape[1], len(lengths), D // groups
    u = delta + (0 if bias is None else bias)
    step = np.logaddexp(0, u)
    r_step = (2 * np.abs(u) + 20) * EPS
    silu = rz = fz = None
    if z is not None:
        fz = sigmoid(z)
        silu, rz = z * fz, (np.abs(z) + 10) * EPS
        dsilu, ez = fz * (1 + z * (1 - fz)), 3 * (np.abs(z) + 8) * (1 + np.abs(z)) * EPS * fz
    dv = dy if z is None else dy * silu
    edv = EPS * np.abs(dv) if z is None else np.abs(dv) * rz
    sk = np.zeros(D) if skip is None else skip
    out = {k: np.zeros((R, D)) for k in ("v", "ev", "x", "ex", "delta", "edelta")}
    last, elast, dh0, edh0 = (np.zeros((B, D, N)) for _ in range(4))
    da, eda, gwa = np.zeros((D, N)), np.zeros((D, N)), np.zeros((D, N))
    db, edb, dc, edc = (np.zeros((R, groups, N)) for _ in range(4))
    off = np.concatenate([[0], np.cumsum(lengths)])
    of = np.repeat(np.arange(groups), per)

    def decay(t):
        al = np.exp(step[t][:, None] * a)
        return al, np.abs(a) * step[t][:, None] * (r_step[t][:, None] + 128 * EPS) + 2 * (step[t][:, None] * np.abs(a) + 8) * EPS

    def share(v):
        return v.reshape(groups, per, N).sum(1)
    for k in range(B):
        h = np.zeros((D, N)) if h0 is None else h0[k].copy()
        M, e = np.abs(h), np.zeros((D, N))
        kept = []
        for t in range(off[k], off[k + 1]):
            bt, ct = b[t][of], c[t][of]
            al, ra = decay(t)
            w, W = al * h, al * M
            ew = al * e + ra * W + LOST * M
            into = (step[t] * x[t])[:, None] * bt
            h, M = w + into, W + np.abs(into)
            e = ew + (r_step[t][:, None] + 3 * EPS) * np.abs(into) + 4 * EPS * M
            kept.append((w, W, ew, h, M, e))
            V = (np.abs(ct) * M).sum(1) + np.abs(sk * x[t])
            out["v"][t] = (ct * h).sum(1) + sk * x[t]
            out["ev"][t] = (np.abs(ct) * e).sum(1) + (N + 4) * EPS * V
        last[k], elast[k] = h, e
        g = np.zeros((D, N)) if dlast is None else dlast[k].copy()
        G, e = np.abs(g), np.zeros((D, N))
        for t in range(off[k + 1] - 1, off[k] - 1, -1):
            w, W, ew, h, M, eh = kept[t - off[k]]
            bt, ct = b[t][of], c[t][of]
            al, ra = decay(t)
            gt = ct * dv[t][:, None] + g
            Gt = np.abs(ct * dv[t][:, None]) + G
            eg = e + np.abs(ct) * edv[t][:, None] + 4 * EPS * Gt
            gb, GB, egb = (gt * bt).sum(1), (Gt * np.abs(bt)).sum(1), (eg * np.abs(bt)).sum(1)
            out["x"][t] = sk * dv[t] + step[t] * gb
            out["ex"][t] = np.abs(sk) * edv[t] + step[t] * (egb + (N + 4) * EPS * GB + r_step[t] * GB) + 2 * EPS * (np.abs(sk * dv[t]) + step[t] * GB)
            s = sigmoid(u[t])
            all_ = (np.abs(a) * Gt * W).sum(1) + np.abs(x[t]) * GB
            ed = (np.abs(a) * (eg * W + Gt * ew)).sum(1) + np.abs(x[t]) * egb + (2 * N + 8) * EPS * all_
            out["delta"][t] = ((gt * w * a).sum(1) + x[t] * gb) * s
            out["edelta"][t] = s * (ed + r_step[t] * all_)
            da += gt * w * step[t][:, None]
            gwa += Gt * W * step[t][:, None]
            eda += step[t][:, None] * (eg * W + Gt * ew + r_step[t][:, None] * Gt * W)
            sx = (step[t] * x[t])[:, None]
            db[t], edb[t] = share(gt * sx), share(np.abs(sx) * (eg + (r_step[t][:, None] + (per + 8) * EPS) * Gt))
            dc[t], edc[t] = share(dv[t][:, None] * h), share(np.abs(dv[t])[:, None] * (eh + (per + 8) * EPS * M) + edv[t][:, None] * M)
            g, G, e = al * gt, al * Gt, al * eg + (ra * al + LOST) * Gt
        dh0[k], edh0[k] = g, e + 2 * EPS * G
    many = (R + 100) * EPS
    got = {"last": (last, elast), "dx": (out["x"], out["ex"]), "ddelta": (out["delta"], out["edelta"]), "da": (da, eda + many * gwa),
           "db": (db.reshape(R, groups * N), edb.reshape(R, groups * N)), "dc": (dc.reshape(R, groups * N), edc.reshape(R, groups * N)), "dh0": (dh0, edh0),
           "dskip": ((dv * x).sum(0), (edv * np.abs(x) + many * np.abs(dv * x)).sum(0)),
           "ddelta_bias": (out["delta"].sum(0), (out["edelta"] + many * (np.abs(out["delta"]) + out["edelta"])).sum(0))}
    if z is None:
        got["y"] = (out["v"], out["ev"])
    else:
        got["y"] = (out["v"] * silu, np.abs(silu) * out["ev"] + rz * np.abs(out["v"] * silu))
        got["dz"] = (dy * out["v"] * dsilu, np.abs(dy) * (np.abs(dsilu) * out["ev"] + (ez + 2 * EPS * np.abs(dsilu)) * (np.abs(out["v"]) + out["ev"])))
    return got


def inputs(rows, bags, dim, states, groups, dtype, seed, step=-2.0):
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype][0]
    t = {k: torch.randn(rows, dim, generator=g).to(dt) for k in ("x", "z", "dy")}
    t["delta"] = torch.randn(rows, dim, generator=g).to(dt)
    t |= {k: torch.randn(rows, groups * states, generator=g).to(dt) for k in ("b", "c")}
    t["a"] = -torch.rand(dim, states, generator=g) * states - 0.1
    t["skip"], t["delta_bias"] = torch.randn(dim, generator=g), torch.randn(dim, generator=g) * 0.5 + step
    t["h0"], t["dlast"] = torch.randn(bags, dim, states, generator=g), torch.randn(bags, dim, states, generator=g)
    return t


def run_and_compare(lengths, dim, states=16, groups=1, dtype="f32", leave=(), seed=0, layout="plain", step=-2.0, one_start=False):
    """leave: arguments that are None"""
    from paper_2305_01515_amd.dense import SelectiveScan
    rows, bags = int(sum(lengths)), len(lengths)
    t = inputs(rows, bags, dim, states, groups, dtype, seed, step)
    if one_start:
        t["h0"] = t["h0"][:1].expand(bags, dim, states)
    t |= {k: None for k in leave}
    want = reference(lengths, *(f64(t[k]) for k in ("x", "delta", "a")), *(f64(t[k]).reshape(rows, groups, states) for k in ("b", "c")),
                     *(f64(t[k]) for k in ("skip", "delta_bias", "z", "h0", "dy", "dlast")), groups)
    gpu = {k: placed(v, layout) if k in ("x", "z", "dy", "delta", "b", "c") else None if v is None else v.cuda() for k, v in t.items()}
    if one_start:
        gpu["h0"] = t["h0"][:1].cuda().expand(bags, dim, states)
    plan, off = SelectiveScan(dim, states, TYPES[dtype][0], bags, rows, groups), offsets(lengths).cuda()
    args = [gpu[k] for k in ("x", "delta", "a", "b", "c")] + [off]
    more = {k: gpu[k] for k in ("skip", "delta_bias", "z", "h0")}
    y, last, saved = plan.forward(*args, **more, save=True)
    got = plan.backward(*args, saved, gpu["dy"], gpu["dlast"], **more)
    plan.check()
    near("y", y, *want["y"], dtype)
    near("last", last, *want["last"])
    for k, v in got.items():
        near("d" + k, v, *want["d" + k], dtype if k in ("x", "delta", "b", "c", "z") else "f32")
    assert set(got) == {"x", "delta", "a", "b", "c"} | {k for k in ("skip", "delta_bias", "z", "h0") if t[k] is not None}
    return plan, args, more, gpu, (y, last, saved, got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,states,groups,layout,leave", [
    (64, 16, 1, "plain", ()), (1, 1, 1, "plain", ("z",)), (7, 3, 1, "wide", ("skip", "h0")), (130, 16, 1, "shifted", ("delta_bias",)),
    (33, 8, 1, "plain", ("dlast",)), (128, 16, 2, "wide", ("h0", "z")), (40, 64, 1, "plain", ()), (128, 24, 2, "shifted", ("skip", "delta_bias", "z", "h0", "dlast")),
    (300, 5, 1, "plain", ()), (256, 64, 4, "plain", ("z", "skip"))])
def test_ragged_bags(dim, states, groups, layout, leave, dtype):
    run_and_compare(RAGGED, dim, states, groups, dtype, leave, seed=dim, layout=layout)


@pytest.mark.parametrize("lengths", [[1], [0], [0, 0, 0], [64], [65], [5000], [1] * 300, [0] * 300 + [3] + [0] * 300, [1500, 0, 1100, 1], [2048, 2048], [65] * 9,
                                     [63, 700, 1, 700, 33, 96], [16] * 7, [15, 17, 81, 79]], ids=lambda v: f"{len(v)}x{max(v)}")
def test_lengths(lengths):
    run_and_compare(lengths, 24, 16, seed=len(lengths))
    run_and_compare(lengths, 10, 4, dtype="bf16", seed=len(lengths) + 1, leave=("z",), one_start=True)


@pytest.mark.parametrize("step", [-20.0, -6.0, 3.0, 20.0])
def test_small_and_large_steps(step):
    """decays of nearly one over thousands of rows, and of nothing"""
    run_and_compare([3000, 17, 200], 20, 16, seed=5, step=step)


def test_more_segments_than_are_read_at_once():
    """33500 rows are 1047 units in 17 segments, in both directions; with steps of 1e-4 the first segment's states are still there in the last one"""
    run_and_compare([33500, 0, 700], 3, 4, seed=8, step=-10.0)


def test_steps_and_decays_over_their_range():
    """What the header says of D and of the decays.  D = log(1 + exp(u)): u log2(e) is rounded, log2(e) in 32 bits is 0.224 eps of itself too small, together 1.224 |u| eps of
    the exponential, and no more of D; the other steps round to within some eps each.  A decay's exponent is rounded twice: 2.224 |D a| eps of the decay."""
    from paper_2305_01515_amd.dense import SelectiveScan
    u = torch.cat([torch.linspace(-85, 85, 1 << 18, dtype=torch.float64), torch.linspace(-18, -14, 1 << 16, dtype=torch.float64)]).float().view(-1, 64)
    rows = len(u)
    plan, off, ones = SelectiveScan(64, 1, torch.float32, rows, rows), torch.arange(rows + 1, device="cuda"), torch.ones(rows, 64, device="cuda")
    one, two = torch.ones(rows, 1, device="cuda"), torch.tensor([0, 1], device="cuda")
    _, last, _ = plan.forward(ones, u.cuda(), -ones[:1].view(64, 1), one, one, off)  # a row's state from zero with b = x = 1 is D
    d = f64(u)
    near("D", last.view(rows, 64), np.logaddexp(0, d), (1.25 * np.abs(d) + 8) * EPS * np.logaddexp(0, d))
    a = -torch.linspace(1e-3, 86, 1 << 16, dtype=torch.float64).float().view(1024, 64)
    step = [SelectiveScan(1024, n, torch.float32, 1, 1) for n in (1, 64)]
    x, delta, h0 = torch.zeros(1, 1024, device="cuda"), torch.full((1, 1024), 0.5413, device="cuda"), torch.ones(1, 1024, 64, device="cuda")
    _, D, _ = step[0].forward(x + 1, delta, a[:, :1].contiguous().cuda(), one[:1], one[:1], two)
    _, last, _ = step[1].forward(x, delta, a.cuda(), x[:, :64].contiguous(), x[:, :64].contiguous(), two, h0=h0)
    p = f64(D).reshape(1024, 1) * f64(a)
    near("decay", last[0], np.exp(p), (1.25 * np.abs(p) + 8) * 2 * EPS * np.exp(p))


def test_many_units_a_segment_and_wide_rows():
    """units of 64 rows (many elements) and of 128: the same numbers as rows of fewer elements have, which units of 32 rows go through"""
    from paper_2305_01515_amd.dense import SelectiveScan
    for rows, dim in ((3001, 11264), (1100, 65536)):
        lengths = [rows - 41, 0, 41]
        t = {k: v.cuda() for k, v in inputs(rows, 3, dim, 1, 1, "f32", 9).items()}
        off, got = offsets(lengths).cuda(), []
        for s in (slice(0, dim), slice(dim - 96, dim)):
            part = {k: v if k in ("b", "c") else v[s] if k in ("a", "skip", "delta_bias") else v[:, s].contiguous() for k, v in t.items()}
            plan = SelectiveScan(part["x"].shape[1], 1, torch.float32, 3, rows)
            args, more = [part[k] for k in ("x", "delta", "a", "b", "c")] + [off], {k: part[k].contiguous() for k in ("skip", "delta_bias", "z", "h0")}
            y, last, saved = plan.forward(*args, **more, save=True)
            g = plan.backward(*args, saved, part["dy"], part["dlast"], **more)
            got.append([y[:, -96:], last[:, -96:], g["x"][:, -96:], g["delta"][:, -96:], g["z"][:, -96:], g["a"][-96:], g["h0"][:, -96:]])
        for v, w in zip(*got):
            # both within the bars of the formula, which for these inputs (|D a| below 3, one state) are some hundred eps of the largest number
            assert (v - w).abs().max() <= 1000 * EPS * w.abs().max()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,states,leave", [(17, 16, ()), (65, 3, ("z",)), (129, 16, ()), (41, 64, ()), (70, 64, ("z",)), (130, 64, ()), (65, 32, ()), (129, 33, ("skip",)), (67, 50, ())])
def test_rows_that_end_within_a_wavefront_of_the_backward(dim, states, leave, dtype):
    """a wavefront there has 16, 8 or 4 elements: rows that leave one of them, or some, and whole wavefronts of a workgroup; bags that start in any row of 8, cut ones too"""
    run_and_compare([1, 2, 3, 4, 5, 0, 6, 7, 70, 1, 300], dim, states, dtype=dtype, leave=leave, seed=dim + states)


def test_groups_see_their_own():
    """groups = two scans beside each other"""
    from paper_2305_01515_amd.dense import SelectiveScan
    t = {k: v.cuda() for k, v in inputs(200, 2, 256, 8, 2, "f32", 3).items()}
    off = offsets([150, 50]).cuda()
    y, last, _ = SelectiveScan(256, 8, torch.float32, 2, 200, groups=2).forward(*(t[k] for k in ("x", "delta", "a", "b", "c")), off)
    for k in range(2):
        s, n = slice(128 * k, 128 * k + 128), slice(8 * k, 8 * k + 8)
        y1, last1, _ = SelectiveScan(128, 8, torch.float32, 2, 200).forward(t["x"][:, s], t["delta"][:, s], t["a"][s], t["b"][:, n], t["c"][:, n], off)
        assert torch.equal(y[:, s], y1) and torch.equal(last[:, s], last1)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,states,groups", [(64, 16, 1), (5, 3, 1), (128, 24, 2), (70, 64, 1), (1, 1, 1)])
def test_step_goes_on_where_bags_end(dim, states, groups, dtype):
    """bags of 1, 2, ... rows, and one more row each: what a pass over the longer bags gives"""
    from paper_2305_01515_amd.dense import SelectiveScan
    lengths = list(range(12))
    rows, bags = sum(lengths) + 12, 12
    t = {k: v.cuda() for k, v in inputs(rows, bags, dim, states, groups, dtype, 7).items()}
    longer = offsets([n + 1 for n in lengths]).cuda()
    newest = longer[1:] - 1
    old = torch.ones(rows, dtype=torch.bool, device="cuda")
    old[newest] = False
    plan = SelectiveScan(dim, states, TYPES[dtype][0], bags, rows, groups)
    more = {k: t[k] for k in ("skip", "delta_bias")}
    y, last, _ = plan.forward(*(t[k] for k in ("x", "delta", "a", "b", "c")), longer, z=t["z"], h0=t["h0"], **more)
    _, state, _ = plan.forward(t["x"][old], t["delta"][old], t["a"], t["b"][old], t["c"][old], offsets(lengths).cuda(), h0=t["h0"], **more)
    store = torch.full((bags + 5, dim + 1, states), 3.0, device="cuda")[:, :dim]  # slots that lie apart
    slots = torch.arange(bags + 4, 4, -1, device="cuda")
    slots[3] = -1
    store[slots[slots >= 0]] = state[slots >= 0]
    before = store.clone()
    got = plan.step(store, t["x"][newest], t["delta"][newest], t["a"], t["b"][newest], t["c"][newest], z=t["z"][newest], slots=slots, **more)
    plan.check()
    there = slots >= 0
    assert torch.equal(store[:5], before[:5]) and (got[3] == 0).all() and torch.equal(store[bags + 1], before[bags + 1])
    # the same operations on the same numbers, but for the order of the sum over states: (states + 4) eps of its magnitudes, and the gate's product
    assert (store[slots[there]] - last[there]).abs().max() <= 4 * EPS * last.abs().max()
    size = last.abs().amax((1, 2))[:, None] * states * t["c"].abs().max().float() * (1 + t["z"][newest].abs().float()) + 10
    assert ((got.float() - y[newest].float()).abs() <= ((states + 20) * EPS + 2 * TYPES[dtype][1]) * size)[there].all()


def test_rows_go_by_their_bag_alone():
    """an infinity in one bag stays there; empty bags keep their states"""
    from paper_2305_01515_amd.dense import SelectiveScan
    lengths = [200, 0, 70, 300]
    t = {k: v.cuda() for k, v in inputs(570, 4, 16, 16, 1, "f32", 2).items()}
    off, plan = offsets(lengths).cuda(), SelectiveScan(16, 16, torch.float32, 4, 570)
    call = lambda: plan.forward(*(t[k] for k in ("x", "delta", "a", "b", "c")), off, h0=t["h0"], save=True)  # noqa: E731
    y, last, _ = call()
    t["x"][230], t["x"][10, 3] = float("inf"), float("nan")
    y2, last2, saved = call()
    assert torch.equal(y[270:], y2[270:]) and torch.equal(last[3], last2[3]) and torch.equal(y[200:230], y2[200:230])
    other = torch.arange(16, device="cuda") != 3
    assert torch.equal(y[:200, other], y2[:200, other]) and torch.isnan(y2[10:200, 3]).all() and not torch.isfinite(y2[230:270]).any()
    assert torch.equal(last2[1], t["h0"][1])
    g = plan.backward(*(t[k] for k in ("x", "delta", "a", "b", "c")), off, saved, t["dy"], t["dlast"], h0=t["h0"])
    assert torch.isfinite(g["x"][270:]).all() and torch.equal(g["h0"][1], t["dlast"][1])


def test_the_same_bits_again_and_in_graphs():
    """calls of the same inputs, and replays of a captured forward and backward between eager work on other sizes of the same handle"""
    plan, args, more, gpu, (y, last, saved, got) = run_and_compare([700, 3, 0, 40, 129], 72, 16, dtype="bf16", seed=4)

    def both():
        y, last, saved = plan.forward(*args, **more, save=True)
        return [y, last, *plan.backward(*args, saved, gpu["dy"], gpu["dlast"], **more).values()]
    want = both()
    for v, w in zip(want, [y, last, *got.values()]):
        assert torch.equal(v, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        for v in out:
            v.zero_()
        graph.replay()
        for v, w in zip(out, want):
            assert torch.equal(v, w)
        short = offsets([5, 2]).cuda()
        rows = [t[:7] if i != 2 else t for i, t in enumerate(args[:5])]
        plan.forward(*rows, short)
        torch.cuda.synchronize()
    plan.check()


def test_gradients_through_autograd():
    """a loss of y and last, against the formula's gradients by differences in 64 bits"""
    from paper_2305_01515_amd.dense import SelectiveScan
    lengths, names = [5, 0, 9], ("x", "delta", "a", "b", "c", "skip", "delta_bias", "z", "h0")
    t = inputs(14, 3, 6, 5, 1, "f32", 8)
    wy, wl = t["dy"], t["dlast"]

    def loss(v):
        want = reference(lengths, v["x"], v["delta"], v["a"], v["b"][:, None], v["c"][:, None], v["skip"], v["delta_bias"], v["z"], v["h0"], f64(wy), f64(wl), 1)
        return (want["y"][0] * f64(wy)).sum() + (want["last"][0] * f64(wl)).sum()
    leaves = {k: t[k].cuda().requires_grad_() for k in names}
    plan = SelectiveScan(6, 5, torch.float32, 3, 14)
    y, last = plan(*(leaves[k] for k in names[:5]), offsets(lengths).cuda(), *(leaves[k] for k in names[5:]))
    ((y * wy.cuda()).sum() + (last * wl.cuda()).sum()).backward()
    rs = np.random.RandomState(0)
    for k in names:
        way, v = rs.standard_normal(t[k].shape), {n: f64(t[n]) for n in names}
        step = 1e-6
        up, down = loss(dict(v, **{k: v[k] + step * way})), loss(dict(v, **{k: v[k] - step * way}))
        slope, got = (up - down) / (2 * step), (f64(leaves[k].grad) * way).sum()
        # differences: step^2 of the third derivative, and 2^-53 of the loss over the step; gradients: some hundred eps of their magnitudes
        assert abs(slope - got) <= 1e-5 * (np.abs(f64(leaves[k].grad) * way).sum() + 1), k
    with pytest.raises(RuntimeError, match="once_differentiable"):
        y, _ = plan(*(leaves[k] for k in names[:5]), offsets(lengths).cuda())
        g, = torch.autograd.grad((y ** 2).sum(), leaves["x"], create_graph=True)
        (g ** 2).sum().backward()


def test_states_are_saved_where_a_gradient_is_asked_for():
    """called for its results alone (without gradients, or with inputs that want none) the object takes the memory of its results"""
    from paper_2305_01515_amd.dense import SelectiveScan
    rows, dim, states = 4096, 64, 64
    t = {k: v.cuda() for k, v in inputs(rows, 2, dim, states, 1, "bf16", 12).items()}
    off, plan = offsets([rows - 9, 9]).cuda(), SelectiveScan(dim, states, torch.bfloat16, 2, rows)
    results = (rows * dim * 2 + 2 * dim * states * 4) + 4096
    saved = rows // 8 * dim * states * 4

    def call():
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = plan(*(t[k] for k in ("x", "delta", "a", "b", "c")), off, **{k: t[k] for k in ("skip", "delta_bias", "z", "h0")})
        return torch.cuda.max_memory_allocated() - before, out
    took, want = call()
    assert took <= results
    t["h0"].requires_grad_()
    with torch.no_grad():
        took, got = call()
    assert took <= results and not got[0].requires_grad
    took, got_grad = call()
    assert took >= saved and got_grad[0].requires_grad
    for v, w, u in zip(want, got, got_grad):
        assert torch.equal(v, w) and torch.equal(v, u)


def test_a_failed_allocation_is_not_the_next_calls():
    """a handle for 2^26 rows of 4096 with 64 states would take more than 4 TB; other operators go on"""
    from paper_2305_01515_amd.dense import RMSNorm, SelectiveScan, ShortConv
    from paper_2305_01515_amd.tbe import TbeError
    conv, norm = ShortConv(8, 2, torch.float32, 1, 4), RMSNorm(8, torch.float32, 4)
    x, w, off = torch.ones(4, 8, device="cuda"), torch.ones(8, 2, device="cuda"), offsets([4]).cuda()
    for call in (lambda: conv.forward(x, off, w), lambda: norm.forward(x, w[:, 0].contiguous()), lambda: ShortConv(8, 2, torch.float32, 1, 4)):
        with pytest.raises(TbeError, match="TBE_ENOMEM"):
            SelectiveScan(4096, 64, torch.bfloat16, 1, 1 << 26)
        call()


def test_what_is_refused():
    from paper_2305_01515_amd.dense import SelectiveScan
    from paper_2305_01515_amd.tbe import TbeError
    for bad in (dict(dim=0), dict(states=65), dict(groups=2), dict(dim=130, groups=2)):
        with pytest.raises(TbeError):
            SelectiveScan(**{**dict(dim=64, states=16, dtype=torch.float32, max_bags=2, max_rows=9), **bad})
    with pytest.raises(ValueError):
        SelectiveScan(8, 4, torch.float64, 2, 9)
    plan = SelectiveScan(8, 4, torch.float32, 2, 9)
    t = {k: v.cuda() for k, v in inputs(9, 2, 8, 4, 1, "f32", 1).items()}
    args, off = [t[k] for k in ("x", "delta", "a", "b", "c")], offsets([4, 5]).cuda()
    for i in range(5):
        with pytest.raises(ValueError):
            plan.forward(*(v.bfloat16() if j == i else v for j, v in enumerate(args)), off)
        with pytest.raises(ValueError):
            plan.forward(*(v.t() if j == i else v for j, v in enumerate(args)), off)
    with pytest.raises(ValueError):
        plan.forward(*args, off.int())
    with pytest.raises(ValueError):
        plan.forward(*args, off, h0=t["h0"].transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(TbeError):
        plan.forward(*args, off, y=t["x"])
    with pytest.raises(TbeError):
        plan.forward(*args, offsets([3, 3, 3]).cuda())  # three bags
    with pytest.raises(ValueError):
        plan.backward(*args, off, torch.zeros(1, device="cuda"), t["dy"])
    saved = plan.forward(*args, off, save=True)[2]
    with pytest.raises(TbeError):  # not from a multiple of 16 bytes on
        plan.backward(*args, off, torch.empty(saved.numel() + 1, device="cuda")[1:], t["dy"])
    plan.forward(*args, torch.tensor([0, 6, 4]).cuda())
    with pytest.raises(TbeError):
        plan.check()
    plan.forward(*args, torch.tensor([1, 4, 9]).cuda())
    with pytest.raises(TbeError):
        plan.check()
    y, _, _ = plan.forward(*args, off)
    plan.check()
    state = torch.zeros(3, 8, 4, device="cuda")
    got = plan.step(state, *(v[:2] if i != 2 else v for i, v in enumerate(args)), slots=torch.tensor([1, 3]).cuda())
    with pytest.raises(TbeError):
        plan.check()
    assert (got[1] == 0).all() and (state[[0, 2]] == 0).all() and (state[1] != 0).any()
    with pytest.raises(TbeError):
        plan.step(state[:1], *(v[:2] if i != 2 else v for i, v in enumerate(args)))


def test_what_is_not_wanted_is_not_found():
    from paper_2305_01515_amd.dense import SelectiveScan
    t = {k: v.cuda() for k, v in inputs(300, 3, 40, 16, 1, "bf16", 6).items()}
    plan, off = SelectiveScan(40, 16, torch.bfloat16, 3, 300), offsets([200, 0, 100]).cuda()
    args = [t[k] for k in ("x", "delta", "a", "b", "c")] + [off]
    y, last, saved = plan.forward(*args, z=t["z"], save=True)
    given = torch.full((300, 50), 5.0, dtype=torch.bfloat16, device="cuda")
    y2, none, nothing = plan.forward(*args, z=t["z"], y=given[:, 3:43], want_last=False)
    assert none is None and nothing is None and torch.equal(y, y2) and (given[:, :3] == 5).all() and (given[:, 43:] == 5).all()
    with_zero = plan.backward(*args, saved, t["dy"], torch.zeros_like(last), z=t["z"])
    for k, v in plan.backward(*args, saved, t["dy"], z=t["z"]).items():
        assert torch.equal(v, with_zero[k])
