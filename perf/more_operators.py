"""What is timed of the operators that models on histories are built of beside the gated recurrence: a short causal convolution over
the rows of a bag, a selective state space scan over them, and a root-mean-square norm with the residual's addition -- and what
they compute, in plain torch operations.

Fields of a case (`op` says which of them it has):
  conv   mode       step (one new row for each of `bags` states among `slots`), forward, train (forward and backward)
         bags, mean, longest   bags, mean of their Poisson lengths, longest one
         dim, dtype, width, silu   elements of a row, type of the rows, rows that a result sees, whether silu follows
         weights, bias, before     type of the weights, whether there is a bias, whether bags go on from earlier rows
  ssm    mode, bags, mean, longest, dim, dtype   as above
         states, groups            states of an element of a row, groups of elements that share their b and c
         gate, skip, shift, h0     whether y is multiplied by silu(z), has skip * x added, deltas have a bias, bags start from given states
  norm   mode       forward, train, bits8 (results in 8 bits with scales)
         rows, dim, dtype          the input
         residual                  type of the residual that is added first, or "none"
         weights, group            type of the weights, elements that share a scale (0: a row)
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def _conv_case(name, **kw):
    return dict({"op": "conv", "silu": True, "bias": True, "before": False, "longest": 200, "slots": 0, "weights": "f32"}, name=name, **kw)


def _ssm_case(name, **kw):
    return dict({"op": "ssm", "states": 16, "groups": 1, "gate": True, "skip": True, "shift": True, "h0": False, "longest": 200, "slots": 0},
                name=name, **kw)


def _norm_case(name, **kw):
    return dict({"op": "norm", "residual": "none", "weights": "f32", "group": 0}, name=name, **kw)


def listed():
    return [
        # Serving: one new row for a handful of users; what counts is the latency of a call.
        _conv_case("conv_step", mode="step", bags=7, mean=1, dim=64, dtype="f32", width=4, slots=64),
        # Training on a batch of histories: the benchmark's batch and bag lengths (8192, Poisson 30, rows of 128), empty bags among them.
        _conv_case("conv_train", mode="train", bags=8192, mean=30, dim=128, dtype="bf16", width=4),
        # Scoring a few event streams of a hundred thousand rows, each continued from its last rows.
        _conv_case("conv_stream", mode="forward", bags=3, mean=100_003, longest=1 << 20, dim=64, dtype="f32", width=3, before=True, silu=False),
        # Serving: one new event for each of a batch of users out of a larger store of states.
        _ssm_case("ssm_step", mode="step", bags=509, mean=1, dim=256, dtype="bf16", slots=2048),
        # Scoring a batch of histories.
        _ssm_case("ssm_histories", mode="forward", bags=8192, mean=30, dim=128, dtype="f16"),
        # Training on the same histories, each continued from a stored state.
        _ssm_case("ssm_train", mode="train", bags=8192, mean=30, dim=128, dtype="bf16", h0=True),
        # Training on a few event streams of a hundred thousand rows: as good as no bags to spread the work over.
        _ssm_case("ssm_long", mode="train", bags=3, mean=100_003, longest=1 << 20, dim=64, dtype="f32", gate=False),
        # A wide model reads a few long histories before it serves them row by row.
        _ssm_case("ssm_prompt", mode="forward", bags=4, mean=1021, longest=1 << 20, dim=2048, dtype="bf16", groups=2),
        # Serving: the norm in front of a layer for the new rows of a handful of users.
        _norm_case("norm_newest", mode="forward", rows=7, dim=128, dtype="bf16", residual="f32"),
        # The norm of the histories of a batch in training, the residual in fp32.
        _norm_case("norm_train", mode="train", rows=8192 * 30, dim=128, dtype="bf16", residual="f32"),
        # Rows of a wide model for a product in 8 bits.
        _norm_case("norm_8bit", mode="bits8", rows=16384, dim=4096, dtype="bf16", residual="bf16", weights="bf16"),
        # Rows of an odd width, a scale for each 128 elements.
        _norm_case("norm_8bit_odd", mode="bits8", rows=4099, dim=1001, dtype="f16", residual="f32", group=128),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """Any shape of the listed ranges: single rows to event streams, odd widths, every type and mode."""
    op, dtype = rng.choice(["conv", "conv", "ssm", "ssm", "ssm", "norm", "norm"]), rng.choice(["f32", "f16", "bf16"])
    if op == "norm":
        c = _norm_case("", mode=rng.choice(["forward", "train", "bits8"]), dtype=dtype, residual=rng.choice(["none", dtype, "f32"]),
                       weights=rng.choice([dtype, "f32"]))
        c["dim"] = int(_log(rng, 1, 20000)) if rng.random() < 0.4 else 8 * int(_log(rng, 1, 2048))
        c["rows"] = max(1, int(_log(rng, 1, 3e7 / c["dim"])))
        c["group"] = rng.choice([0, 0, 32, 128]) if c["mode"] == "bits8" else 0
        del c["name"]
        return c
    mode = rng.choice(["step", "forward", "train", "train"])
    dim = int(_log(rng, 1, 500)) if rng.random() < 0.4 else 8 * int(_log(rng, 1, 256))
    if op == "conv":
        c = _conv_case("", mode=mode, dim=dim, dtype=dtype, width=rng.choice([1, 2, 3, 4, 4, 5, 8]), silu=rng.random() < 0.7,
                       bias=rng.random() < 0.7, before=rng.random() < 0.4, weights=rng.choice(["f32", dtype]))
        most = 2.5e7 / dim
    else:
        c = _ssm_case("", mode=mode, dim=dim, dtype=dtype, states=rng.choice([1, 4, 8, 16, 16, 16, 24, 64]), gate=rng.random() < 0.6,
                      skip=rng.random() < 0.7, shift=rng.random() < 0.7, h0=mode != "step" and rng.random() < 0.5)
        if dim % 128 == 0 and rng.random() < 0.5:
            c["groups"] = 2
        most = 4e8 / (dim * max(8, c["states"]))
    if mode == "step":
        c["bags"], c["mean"] = int(_log(rng, 1, min(4096, max(2, most)))), 1
        c["slots"] = c["bags"] + int(_log(rng, 1, 4096))
        if op == "ssm":
            c["slots"] = min(c["slots"], c["bags"] + int(2e8 / (dim * c["states"])))
    else:
        rows = _log(rng, 20, max(40, min(3e5, most)))
        c["mean"] = max(1, int(_log(rng, 1, max(2, rows))))
        c["bags"], c["longest"] = max(1, int(rows / c["mean"])), 4 * c["mean"] + 20
    del c["name"]
    return c


# ---- the inputs a case describes ----

def _lengths(case):
    """Rows of each bag: a function of the case alone."""
    rs = np.random.RandomState((case["bags"] * 31 + case["mean"] * 7 + case["dim"]) % (1 << 31))
    return np.clip(rs.poisson(case["mean"], case["bags"]), 0, case["longest"]).astype(np.int64)


def _randn(g, *shape, dtype="f32", mean=0.0, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(TYPES[dtype])


def _some(g, n, of):
    return torch.randperm(of, generator=g, device="cuda")[:n].contiguous()


def _prepare_conv(case, g):
    D, B, W, dt = case["dim"], case["bags"], case["width"], case["dtype"]
    s = {"weight": _randn(g, D, W, dtype=case["weights"], std=W ** -0.5), "bias": _randn(g, D, dtype=case["weights"], std=0.1) if case["bias"] else None,
         "before": None}
    if case["mode"] == "step":
        N = B
        s |= {"x": _randn(g, B, D, dtype=dt), "state": _randn(g, case["slots"], W - 1, D, dtype=dt), "slots": _some(g, B, case["slots"])}
    else:
        off = np.concatenate([[0], np.cumsum(_lengths(case))])
        N = int(off[-1])
        s |= {"offsets": torch.from_numpy(off).cuda(), "x": _randn(g, N, D, dtype=dt)}
        if case["before"]:
            s["before"] = _randn(g, B, W - 1, D, dtype=dt)
        if case["mode"] == "train":
            s["dy"] = _randn(g, N, D, dtype=dt, std=0.1)
    if own:
        from paper_2305_01515_amd import dense
        s["plan"] = dense.ShortConv(D, W, TYPES[dt], max_bags=B, max_rows=N, silu=case["silu"])
    return s


def _prepare_ssm(case, g):
    D, B, N, G, dt = case["dim"], case["bags"], case["states"], case["groups"], case["dtype"]
    # decays 1, 2, ... a unit of time and around them; steps of 0.001 to 0.1 at the start of a training, most of them
    a = -torch.arange(1, N + 1, device="cuda").float() * torch.exp(_randn(g, D, N, std=0.3))
    step = torch.exp(torch.rand(D, generator=g, device="cuda") * math.log(100) + math.log(0.001))
    s = {"a": a, "skip": _randn(g, D, mean=1.0, std=0.2) if case["skip"] else None,
         "delta_bias": torch.log(torch.expm1(step)) if case["shift"] else None, "h0": None, "z": None}
    if case["mode"] == "step":
        rows = B
        s |= {"state": _randn(g, case["slots"], D, N), "slots": _some(g, B, case["slots"])}
    else:
        off = np.concatenate([[0], np.cumsum(_lengths(case))])
        rows = int(off[-1])
        s |= {"offsets": torch.from_numpy(off).cuda(), "longest": int(max(1, _lengths(case).max(initial=1)))}
        if case["h0"]:
            s["h0"] = _randn(g, B, D, N)
    s["x"] = _randn(g, rows, D, dtype=dt)
    s["delta"] = _randn(g, rows, D, dtype=dt, mean=0.0 if case["shift"] else -3.0)
    s["b"], s["c"] = _randn(g, rows, G * N, dtype=dt), _randn(g, rows, G * N, dtype=dt)
    if case["gate"]:
        s["z"] = _randn(g, rows, D, dtype=dt)
    if case["mode"] == "train":
        s["dy"] = _randn(g, rows, D, dtype=dt, std=0.1)
        s["dlast"] = _randn(g, B, D, N, std=0.01)
    if own:
        from paper_2305_01515_amd import dense
        s["plan"] = dense.SelectiveScan(D, N, TYPES[dt], max_bags=B, max_rows=rows, groups=G)
    return s


def _prepare_norm(case, g):
    R, D, dt = case["rows"], case["dim"], case["dtype"]
    s = {"x": _randn(g, R, D, dtype=dt), "weight": _randn(g, D, dtype=case["weights"], mean=1.0, std=0.2), "residual": None}
    if case["residual"] != "none":
        s["residual"] = _randn(g, R, D, dtype=case["residual"], std=2.0)
    if case["mode"] == "train":
        s["dout"] = _randn(g, R, D, dtype=dt, std=0.1)
        s["dsummed"] = _randn(g, R, D, dtype=case["residual"], std=0.1) if s["residual"] is not None else None
    if own:
        from paper_2305_01515_amd import dense
        s["plan"] = dense.RMSNorm(D, TYPES[dt], max_rows=R, eps=EPS, residual_dtype=TYPES.get(case["residual"]))
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFF)
    s = {"conv": _prepare_conv, "ssm": _prepare_ssm, "norm": _prepare_norm}[case["op"]](case, g)
    s["case"] = case
    return s


# ---- the plain forms ----

def _sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def _softplus(u):
    return u.clamp(min=0) + torch.log1p(torch.exp(-u.abs()))


def _bag_of_rows(off, n):
    """bag of every row, and how many rows of it are before"""
    row = torch.arange(n, device="cuda")
    bag = torch.searchsorted(off, row, right=True) - 1
    return bag, row - off[bag]


def _taps(x, before, bag, age, width):
    """[rows, width, dim]: what every row's result sees, oldest first; zero in front of a bag that goes on from nothing"""
    back = torch.arange(width - 1, -1, -1, device="cuda")
    at = torch.arange(x.shape[0], device="cuda")[:, None] - back
    inside = age[:, None] >= back
    e = x[at.clamp(min=0)].float() * inside[..., None]
    if before is not None and width > 1:
        e = torch.where(inside[..., None], e, before[bag[:, None], (width - 1 + age[:, None] - back).clamp(0, width - 2)].float())
    return e


def _seen_by(g, w, off, place, bag):
    """gradient of the rows at `place` (which may lie in front of their bag) from those of the results that see them"""
    ahead = torch.arange(w.shape[1], device="cuda")
    to = place[:, None] + ahead
    inside = (to >= off[bag][:, None]) & (to < off[bag + 1][:, None])
    return (g[to.clamp(0, max(0, g.shape[0] - 1))] * inside[..., None] * w.t().flip(0)).sum(1)


def _plain_conv(s):
    case, dt, W = s["case"], s["x"].dtype, s["case"]["width"]
    w, x = s["weight"].float(), s["x"]
    if case["mode"] == "step":
        e = torch.cat([s["state"][s["slots"]], x[:, None]], 1)
        v = (e.float() * w.t()).sum(1)
        s["state"][s["slots"]] = e[:, 1:]
    else:
        off = s["offsets"]
        bag, age = _bag_of_rows(off, x.shape[0])
        e = _taps(x, s["before"], bag, age, W)
        v = (e * w.t()).sum(1)
    if s["bias"] is not None:
        v = v + s["bias"].float()
    y = (v * _sigmoid(v) if case["silu"] else v).to(dt)
    if case["mode"] == "step":
        return {"y": y, "state": s["state"]}
    # the rows that the next ones of a bag will see: its last width - 1, the ones before it among them
    place = off[1:, None] - torch.arange(W - 1, 0, -1, device="cuda")
    old = place - off[:-1, None]
    last = x[place.clamp(min=0)] if x.shape[0] else torch.zeros(case["bags"], W - 1, case["dim"], dtype=dt, device="cuda")
    earlier = s["before"] if s["before"] is not None else torch.zeros_like(last)
    filler = torch.gather(earlier, 1, (W - 1 + old).clamp(0, max(0, W - 2))[..., None].expand_as(last))
    last = torch.where(old[..., None] >= 0, last, filler)
    out = {"y": y, "last": last}
    if case["mode"] == "forward":
        return out
    g = s["dy"].float()
    if case["silu"]:
        f = _sigmoid(v)
        g = g * (f * (1 + v * (1 - f)))
    out["dx"] = _seen_by(g, w, off, torch.arange(x.shape[0], device="cuda"), bag).to(dt)
    out["dweight"] = (g[:, None] * e).sum(0).t().contiguous()
    if s["bias"] is not None:
        out["dbias"] = g.sum(0)
    if s["before"] is not None:
        old = off[:-1, None] + torch.arange(1 - W, 0, device="cuda")
        owner = torch.arange(case["bags"], device="cuda")[:, None].expand_as(old)
        out["dbefore"] = _seen_by(g, w, off, old.reshape(-1), owner.reshape(-1)).view(case["bags"], W - 1, case["dim"]).to(dt)
    return out


def _linear_scan(a, b, longest):
    """h_t = a_t h_{t-1} + b_t along the first axis, a_t = 0 where a bag starts: partial results of twice the rows each time."""
    k = 1
    while k < longest:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _of_groups(t, case):
    """[rows, dim, states] of b or c, shared by the elements of a group"""
    G, D = case["groups"], case["dim"]
    return t.float().view(-1, G, 1, case["states"]).expand(-1, G, D // G, -1).reshape(-1, D, case["states"])


def _plain_ssm(s):
    case, dt, a = s["case"], s["x"].dtype, s["a"]
    D, N, G = case["dim"], case["states"], case["groups"]
    x, u = s["x"].float(), s["delta"].float()
    if s["delta_bias"] is not None:
        u = u + s["delta_bias"]
    step = _softplus(u)
    b, c = _of_groups(s["b"], case), _of_groups(s["c"], case)
    decay = torch.exp(step[..., None] * a)
    into = (step * x)[..., None] * b
    if case["mode"] == "step":
        h = decay * s["state"][s["slots"]] + into
        s["state"][s["slots"]] = h
    else:
        off = s["offsets"]
        full = off[1:] > off[:-1]
        first, end = off[:-1][full], off[1:][full] - 1
        h0 = s["h0"] if s["h0"] is not None else torch.zeros(case["bags"], D, N, device="cuda")
        f = decay.clone()
        into[first] += decay[first] * h0[full]
        f[first] = 0
        h = _linear_scan(f, into, s["longest"])
    v = (h * c).sum(2)
    if s["skip"] is not None:
        v = v + s["skip"] * x
    gate = s["z"].float() * _sigmoid(s["z"].float()) if case["gate"] else None
    y = (v * gate if case["gate"] else v).to(dt)
    if case["mode"] == "step":
        return {"y": y, "state": s["state"]}
    last = h0.clone()
    last[full] = h[end]
    out = {"y": y, "last": last}
    if case["mode"] == "forward":
        return out
    dv = s["dy"].float()
    if case["gate"]:
        z, f = s["z"].float(), _sigmoid(s["z"].float())
        out["dz"] = (dv * v * (f * (1 + z * (1 - f)))).to(dt)
        dv = dv * gate
    f = torch.cat([decay[1:], torch.zeros_like(decay[:1])])  # the decay between a row and the next one
    f[end] = 0
    g = dv[..., None] * c
    g[end] += s["dlast"][full]
    g = _linear_scan(f.flip(0), g.flip(0), s["longest"]).flip(0)
    del f
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first] = h0[full]
    kept = g * before * decay
    into = (g * b).sum(2)
    dstep = (kept * a).sum(2) + x * into
    du = dstep * _sigmoid(u)
    dx = step * into
    if s["skip"] is not None:
        dx, out["dskip"] = dx + s["skip"] * dv, (dv * x).sum(0)
    out["dx"], out["ddelta"] = dx.to(dt), du.to(dt)
    out["da"] = (kept * step[..., None]).sum(0)
    out["db"] = (g * (step * x)[..., None]).view(-1, G, D // G, N).sum(2).view(-1, G * N).to(dt)
    out["dc"] = (h * dv[..., None]).view(-1, G, D // G, N).sum(2).view(-1, G * N).to(dt)
    if s["delta_bias"] is not None:
        out["ddelta_bias"] = du.sum(0)
    if s["h0"] is not None:
        out["dh0"] = s["dlast"].clone()
        out["dh0"][full] = g[first] * decay[first]
    return out


def _plain_norm(s):
    case, dt, w = s["case"], s["x"].dtype, s["weight"].float()
    # What the next layer adds to is stored in the residual's type; the norm is that of the stored rows.
    summed = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype) if s["residual"] is not None else s["x"]
    r = summed.float()
    rstd = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)
    v = r * rstd * w
    out = {"summed": summed} if s["residual"] is not None else {}
    if case["mode"] == "bits8":
        D, n = case["dim"], case["group"] or case["dim"]
        q = torch.nn.functional.pad(v, (0, -D % n)).view(v.shape[0], -1, n)
        scale = q.abs().amax(2) / 448
        code = torch.where(scale[..., None] > 0, q / scale[..., None], 0.0).clamp(-448, 448).to(torch.float8_e4m3fn)
        return dict(out, codes=code.view(v.shape[0], -1)[:, :D].contiguous(), scales=scale)
    out["out"] = v.to(dt)
    if case["mode"] == "train":
        d = s["dout"].float()
        out["dweight"] = (d * (r * rstd)).sum(0)
        d = d * w
        dr = rstd * (d - r * rstd * ((d * r).mean(1, keepdim=True) * rstd))
        if s["residual"] is not None:
            dr = dr + s["dsummed"].float()
            out["dresidual"] = dr.to(s["residual"].dtype)
        out["dx"] = dr.to(dt)
    return out


# ---- one pass ----

def _own_conv(s):
    case, plan = s["case"], s["plan"]
    if case["mode"] == "step":
        return {"y": plan.step(s["state"], s["x"], s["weight"], s["bias"], slots=s["slots"]), "state": s["state"]}
    y, last = plan.forward(s["x"], s["offsets"], s["weight"], s["bias"], s["before"])
    out = {"y": y, "last": last}
    if case["mode"] == "train":
        got = plan.backward(s["x"], s["offsets"], s["weight"], s["dy"], s["bias"], s["before"])
        out |= {k: v for k, v in zip(("dx", "dweight", "dbias", "dbefore"), got) if v is not None}
    return out


def _own_ssm(s):
    case, plan = s["case"], s["plan"]
    more = {k: s[k] for k in ("skip", "delta_bias", "z")}
    if case["mode"] == "step":
        return {"y": plan.step(s["state"], s["x"], s["delta"], s["a"], s["b"], s["c"], slots=s["slots"], **more), "state": s["state"]}
    rows = (s["x"], s["delta"], s["a"], s["b"], s["c"], s["offsets"])
    y, last, saved = plan.forward(*rows, h0=s["h0"], save=case["mode"] == "train", **more)
    out = {"y": y, "last": last}
    if case["mode"] == "train":
        got = plan.backward(*rows, saved, s["dy"], dlast=s["dlast"], h0=s["h0"], **more)
        out |= {"d" + k: v for k, v in got.items()}
    return out


def _own_norm(s):
    case, plan = s["case"], s["plan"]
    if case["mode"] == "bits8":
        codes, scales, summed = plan.quantise(s["x"], s["weight"], s["residual"], group=case["group"])
        out = {"codes": codes, "scales": scales}
    else:
        y, summed, rstd = plan.forward(s["x"], s["weight"], s["residual"])
        out = {"out": y}
    if s["residual"] is not None:
        out["summed"] = summed
    if case["mode"] == "train":
        out["dx"], dresidual, out["dweight"] = plan.backward(s["dout"], summed, rstd, s["weight"], s["dsummed"])
        if s["residual"] is not None:
            out["dresidual"] = dresidual
    return out


def run(state):
    op = state["case"]["op"]
    if op == "conv":
        return _own_conv(state) if own else _plain_conv(state)
    if op == "ssm":
        return _own_ssm(state) if own else _plain_ssm(state)
    return _own_norm(state) if own else _plain_norm(state)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        R, D = case["rows"], case["dim"]
        ws = 4 if case["weights"] == "f32" else 2
        rs = 0 if case["residual"] == "none" else 4 if case["residual"] == "f32" else 2
        n, w = R * D, D * ws
        if case["mode"] == "bits8":
            return {"bytes": n * (es + 2 * rs + 1) + 4 * R * -(-D // (case["group"] or D)) + w, "flops": 8 * n}
        forward = n * (2 * es + 2 * rs) + w
        if case["mode"] == "forward":
            return {"bytes": forward, "flops": 5 * n}
        # the stored sum is read by the backward as an input of its own
        return {"bytes": forward + n * (2 * es + ((3 * rs) or es)) + 4 * D, "flops": 15 * n}
    B, D = case["bags"], case["dim"]
    rows = B if case["mode"] == "step" else int(_lengths(case).sum())
    n = rows * D
    if case["op"] == "conv":
        W, ws = case["width"], 4 if case["weights"] == "f32" else 2
        w = D * (W + case["bias"]) * ws
        if case["mode"] == "step":
            return {"bytes": es * n * (2 + 2 * (W - 1)) + w + 8 * B, "flops": n * (2 * W + 5)}
        forward = es * (2 * n + B * D * (W - 1) * (1 + case["before"])) + w + 8 * (B + 1)
        if case["mode"] == "forward":
            return {"bytes": forward, "flops": n * (2 * W + 5)}
        return {"bytes": forward + es * (2 * n + B * D * (W - 1) * case["before"]) + 4 * D * (W + case["bias"]), "flops": n * (8 * W + 20)}
    N, G = case["states"], case["groups"]
    weights = 4 * D * (N + case["skip"] + case["shift"])
    shared = 2 * es * rows * G * N
    forward = es * n * (3 + case["gate"]) + shared + weights
    if case["mode"] == "step":
        return {"bytes": forward + 8 * n * N + 8 * B, "flops": n * (7 * N + 15)}
    forward += 4 * B * D * N * (1 + case["h0"]) + 8 * (B + 1)
    if case["mode"] == "forward":
        return {"bytes": forward, "flops": n * (7 * N + 15)}
    return {"bytes": forward + es * n * (3 + case["gate"]) + shared + weights + 4 * B * D * N * (1 + case["h0"]), "flops": n * (25 * N + 50)}


# ---- the operators' definitions in 64 bits ----

def _exact_conv(case, s):
    W, D, B = case["width"], case["dim"], case["bags"]
    x, w = s["x"].double(), s["weight"].double()
    bias = s["bias"].double() if case["bias"] else torch.zeros(D, dtype=torch.float64, device="cuda")
    if case["mode"] == "step":
        state = s["state"].double()
        seen = torch.cat([state[s["slots"]], x[:, None]], 1)
        v = torch.einsum("bwd,dw->bd", seen, w) + bias
        state[s["slots"]] = seen[:, 1:]
        return {"y": torch.nn.functional.silu(v) if case["silu"] else v, "state": state}
    # every bag with its earlier rows in front of it, one behind another
    size = _lengths(case)
    n, at, K = int(size.sum()), np.concatenate([[0], np.cumsum(size + W - 1)]), W - 1
    place = torch.from_numpy(np.arange(n) + np.repeat(np.arange(1, B + 1) * K, size)).cuda()
    head = torch.from_numpy((at[:-1, None] + np.arange(K)).reshape(-1)).cuda()
    tail = torch.from_numpy((at[1:, None] - K + np.arange(K)).reshape(-1)).cuda()
    e = torch.zeros(int(at[-1]), D, dtype=torch.float64, device="cuda")
    e[place] = x
    if case["before"]:
        e[head] = s["before"].double().view(-1, D)
    v = bias.expand(n, D).clone()
    for j in range(W):
        v += e[place - K + j] * w[:, j]
    out = {"y": torch.nn.functional.silu(v) if case["silu"] else v, "last": e[tail].view(B, K, D)}
    if case["mode"] == "train":
        g = s["dy"].double()
        if case["silu"]:
            p = torch.sigmoid(v)
            g = g * (p + v * p * torch.sigmoid(-v))
        de, dw = torch.zeros_like(e), torch.zeros_like(w)
        for j in range(W):
            de[place - K + j] += g * w[:, j]
            dw[:, j] = (g * e[place - K + j]).sum(0)
        out |= {"dx": de[place], "dweight": dw}
        if case["bias"]:
            out["dbias"] = g.sum(0)
        if case["before"]:
            out["dbefore"] = de[head].view(B, K, D)
    return out


def _exact_scan(a, b):
    """h_t = a_t h_{t-1} + b_t by blocks of rows: every block from a zero state, then the states before the blocks in turn"""
    n, shape = b.shape[0], b.shape[1:]
    size = 128 if n > 4000 else 16
    blocks = -(-n // size)
    pad = torch.zeros(blocks * size - n, *shape, dtype=b.dtype, device=b.device)
    a, b = torch.cat([a, pad]).view(blocks, size, *shape), torch.cat([b, pad]).view(blocks, size, *shape)
    h, p = torch.empty_like(b), torch.empty_like(a)
    state, prod = torch.zeros_like(b[:, 0]), torch.ones_like(a[:, 0])
    for j in range(size):
        state, prod = torch.addcmul(b[:, j], a[:, j], state), prod * a[:, j]
        h[:, j], p[:, j] = state, prod
    carry, before = torch.zeros_like(state[0]), torch.empty_like(state)
    for k in range(blocks):
        before[k] = carry
        carry = torch.addcmul(state[k], prod[k], carry)
    return h.addcmul_(p, before[:, None]).view(blocks * size, *shape)[:n]


def _exact_ssm(case, s):
    D, N, G, B = case["dim"], case["states"], case["groups"], case["bags"]
    R = s["x"].shape[0]
    train, step = case["mode"] == "train", case["mode"] == "step"
    b, c = s["b"].double().view(R, G, N), s["c"].double().view(R, G, N)
    if not step:
        off = np.concatenate([[0], np.cumsum(_lengths(case))])
        full = np.flatnonzero(off[1:] > off[:-1])
        first, end, bags = (torch.from_numpy(i).cuda() for i in (off[full], off[full + 1] - 1, full))
    parts, db, dc = [], torch.zeros_like(b), torch.zeros_like(c)
    width = D // G
    most = max(1, int(4e7 / (R * N)))  # elements of a row at a time
    for d0, d1, k in [(k * width + i, min(k * width + i + most, (k + 1) * width), k) for k in range(G) for i in range(0, width, most)]:
        x, u = s["x"][:, d0:d1].double(), s["delta"][:, d0:d1].double()
        a, bk, ck = s["a"][d0:d1].double(), b[:, k, None], c[:, k, None]
        if case["shift"]:
            u = u + s["delta_bias"][d0:d1].double()
        t = torch.nn.functional.softplus(u, threshold=1000.0)
        skip = s["skip"][d0:d1].double() if case["skip"] else torch.zeros(d1 - d0, dtype=torch.float64, device="cuda")
        decay = torch.exp(t[..., None] * a)
        drive = (t * x)[..., None] * bk
        out = {}
        if step:
            state = s["state"][:, d0:d1].double()
            h = torch.addcmul(drive, decay, state[s["slots"]])
            state[s["slots"]] = h
            out["state"] = state
        else:
            h0 = s["h0"][:, d0:d1].double() if case["h0"] else torch.zeros(B, d1 - d0, N, dtype=torch.float64, device="cuda")
            keep = decay.clone()
            keep[first] = 0
            drive[first] += decay[first] * h0[bags]
            h = _exact_scan(keep, drive)
            out["last"] = h0.clone()
            out["last"][bags] = h[end]
        v = torch.matmul(h, ck.transpose(1, 2).contiguous())[..., 0] + skip * x
        z = s["z"][:, d0:d1].double() if case["gate"] else None
        out["y"] = v * torch.nn.functional.silu(z) if case["gate"] else v
        if train:
            dv = s["dy"][:, d0:d1].double()
            if case["gate"]:
                p = torch.sigmoid(z)
                out["dz"] = dv * v * (p + z * p * torch.sigmoid(-z))
                dv = dv * (z * p)
            keep = torch.roll(decay, -1, 0)
            keep[end] = 0
            g = dv[..., None] * ck
            g[end] += s["dlast"][:, d0:d1].double()[bags]
            g = _exact_scan(keep.flip(0), g.flip(0)).flip(0)
            old = torch.roll(h, 1, 0)
            old[first] = h0[bags]
            old *= decay * g
            gb = (g * bk).sum(2)
            du = ((old * a).sum(2) + x * gb) * torch.sigmoid(u)
            out |= {"dx": skip * dv + t * gb, "ddelta": du, "da": torch.einsum("rdn,rd->dn", old, t)}
            db[:, k] += torch.einsum("rdn,rd->rn", g, t * x)
            dc[:, k] += torch.einsum("rdn,rd->rn", h, dv)
            if case["skip"]:
                out["dskip"] = (dv * x).sum(0)
            if case["shift"]:
                out["ddelta_bias"] = du.sum(0)
            if case["h0"]:
                out["dh0"] = s["dlast"][:, d0:d1].double()
                out["dh0"][bags] = (g * decay)[first]
        parts.append(out)
    per_element = ("da", "dskip", "ddelta_bias")
    out = {k: torch.cat([p[k] for p in parts], 0 if k in per_element else 1) for k in parts[0]}
    return dict(out, db=db.view(R, G * N), dc=dc.view(R, G * N)) if train else out


def _to_8_bits(q):
    """nearest number of 4 exponent and 3 mantissa bits, the even one of two"""
    gap = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / gap) * gap


def _exact_norm(case, s):
    D, w = case["dim"], s["weight"].double()
    added = s["residual"] is not None
    r = (s["x"].double() + s["residual"].double()).to(s["residual"].dtype).double() if added else s["x"].double()
    rstd = torch.rsqrt(r.square().sum(1, keepdim=True) / D + EPS)
    unit = r * rstd
    out = {"summed": r} if added else {}
    if case["mode"] == "bits8":
        v, n = unit * w, case["group"] or D
        scales = torch.stack([v[:, i:i + n].abs().max(1).values / 448 for i in range(0, D, n)], 1)
        spread = scales.repeat_interleave(n, 1)[:, :D]
        return dict(out, codes=_to_8_bits(torch.where(spread > 0, v / spread, 0.0)), scales=scales)
    out["out"] = unit * w
    if case["mode"] == "train":
        d = s["dout"].double()
        out["dweight"] = (d * unit).sum(0)
        out["dx"] = (d * w - unit * (d * w * unit).mean(1, keepdim=True)) * rstd
        if added:
            out["dx"] = out["dx"] + s["dsummed"].double()
            out["dresidual"] = out["dx"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "ssm": _exact_ssm, "norm": _exact_norm}[case["op"]](case, s)
