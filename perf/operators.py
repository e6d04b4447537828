"""What is timed of the operators beside the embedding path -- a gated recurrence over the rows of a bag, a learned bias
by buckets of a distance, and AdamW over many tensors -- and what they compute, in plain torch operations.

Fields of a case (`op` says which of them it has):
  scan   mode       step (one new row for each of `bags` states among `slots`), forward, train (forward and backward)
         bags, mean, longest   bags, mean of their Poisson lengths, longest one; with `equal` all have `mean` rows
         dim, dtype, coupled, h0   elements of a row, type of the rows, (1 - f) on the input, whether bags start from given states
  bias   mode       bias (the table's values), add (scores * scale + bias), grad (gradient of the table)
         batch, heads, lq, lk      shape of the scores; buckets, far: buckets of one side, distance from which the last one holds
         times      distances of time stamps, per sample, instead of positions
         both, causal, lengths     a side each for earlier and later keys, later keys masked, keys beyond a sample's length masked
  adamw  layers     widths of fully connected layers, each with a weight matrix and a bias
         dtype, grads, master, bits   types of parameters and gradients, fp32 copies beside 16-bit parameters, bits of a state
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LR, BETA1, BETA2, EPS, DECAY, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1234567
BLOCK = 256  # elements of a state in 8 bits that share a scale


def _scan_case(name, **kw):
    return dict({"op": "scan", "coupled": True, "h0": False, "equal": False, "longest": 200, "slots": 0}, name=name, **kw)


def _bias_case(name, **kw):
    return dict({"op": "bias", "times": False, "both": False, "causal": False, "lengths": False}, name=name, **kw)


def _adamw_case(name, **kw):
    return dict({"op": "adamw", "dtype": "f32", "grads": "f32", "master": False, "bits": 32}, name=name, **kw)


def listed():
    return [
        # Serving: one new row for a handful of users; what counts is the latency of a call.
        _scan_case("step_smallest", mode="step", bags=7, mean=1, dim=64, dtype="f32", slots=64),
        # Scoring a batch of histories: the benchmark's batch and bag lengths (8192, Poisson 30, rows of 128 in binary16),
        # empty bags among them.
        _scan_case("pool_histories", mode="forward", bags=8192, mean=30, dim=128, dtype="f16"),
        # Training on the same histories, each continued from a stored state.
        _scan_case("train_histories", mode="train", bags=8192, mean=30, dim=128, dtype="bf16", h0=True),
        # Training on a few event streams of a hundred thousand rows: as good as no bags to spread the work over.
        _scan_case("train_long", mode="train", bags=3, mean=100_003, longest=1 << 20, dim=64, dtype="f32", coupled=False),
        # The weights of a small dense model (13 dense features, the widths of a click model's bottom part).
        _adamw_case("adamw_mlp", layers="13-512-256-128-64"),
        # A large dense part in fp32.
        _adamw_case("adamw_large", layers="8191-8192-8192-4096-1000"),
        # The same with 16-bit parameters and gradients, fp32 copies and states in 8 bits.
        _adamw_case("adamw_8bit", layers="8191-8192-8192-4096-1000", dtype="bf16", grads="bf16", master=True, bits=8),
        # The bias of a layer that attends over positions, shared by all samples.
        _bias_case("bias_positions", mode="bias", batch=1, heads=16, lq=2048, lk=2048, dtype="bf16", buckets=16, far=128,
                   both=True),
        # Scores of one new event of each user against the stored history, by age; ragged histories.
        _bias_case("add_newest", mode="add", batch=512, heads=8, lq=1, lk=1001, dtype="f32", buckets=32, far=10_000_000,
                   times=True, lengths=True),
        # Scores inside the histories of a batch, by time differences, causal, ragged.
        _bias_case("add_times", mode="add", batch=256, heads=4, lq=199, lk=199, dtype="f16", buckets=32, far=10_000_000,
                   times=True, causal=True, lengths=True),
        # Their gradient.
        _bias_case("grad_times", mode="grad", batch=256, heads=4, lq=199, lk=199, dtype="f16", buckets=32, far=10_000_000,
                   times=True, causal=True, lengths=True),
        # Gradient of the positions' bias: a table of a few hundred numbers from all scores of a batch.
        _bias_case("grad_positions", mode="grad", batch=16, heads=8, lq=1024, lk=1024, dtype="bf16", buckets=16, far=128,
                   both=True),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """Any shape of the listed ranges: single rows to event streams, odd widths, every type, mode and mask."""
    op, dtype = rng.choice(["scan", "scan", "bias", "bias", "adamw"]), rng.choice(["f32", "f16", "bf16"])
    if op == "scan":
        mode = rng.choice(["step", "forward", "train", "train"])
        dim = rng.choice([1, 3, 5]) * int(_log(rng, 1, 80)) if rng.random() < 0.3 else 8 * int(_log(rng, 1, 64))
        c = _scan_case("", mode=mode, dim=dim, dtype=dtype, coupled=rng.random() < 0.6, h0=mode != "step" and rng.random() < 0.5)
        if mode == "step":
            c["bags"], c["mean"] = int(_log(rng, 1, 8192)), 1
            c["slots"] = c["bags"] + int(_log(rng, 1, 8192))
        else:
            rows = _log(rng, 20, 3e7 / dim if mode == "forward" else 1.8e7 / dim)
            c["mean"] = max(1, int(_log(rng, 1, max(2, rows))))
            c["bags"], c["longest"] = max(1, int(rows / c["mean"])), 4 * c["mean"] + 20
            c["equal"] = rng.random() < 0.2
    elif op == "bias":
        mode = rng.choice(["bias", "add", "grad", "grad"])
        times = rng.random() < 0.5
        c = _bias_case("", mode=mode, heads=rng.choice([1, 2, 3, 4, 6, 8, 12, 16]), dtype=dtype, times=times,
                       both=rng.random() < 0.5, causal=rng.random() < 0.4, lengths=rng.random() < 0.4)
        c["lq"] = 1 if rng.random() < 0.25 else int(_log(rng, 2, 1500))
        c["lk"] = int(_log(rng, 1, 4000)) if c["lq"] == 1 or rng.random() < 0.3 else c["lq"]
        c["batch"] = int(_log(rng, 1, max(1.5, min(1024, 3e7 / (c["heads"] * c["lq"] * c["lk"])))))
        c["batch"] = max(1, min(c["batch"], 12_000_000 // (c["lq"] * c["lk"])))
        if mode == "bias" and not times:
            c["batch"], c["lengths"] = 1, False
        c["buckets"], c["far"] = rng.choice([4, 8, 16, 24, 32, 64]), int(_log(rng, 1e4, 1e8) if times else _log(rng, 70, 2000))
    else:
        c = _adamw_case("", dtype=dtype, bits=rng.choice([8, 8, 32]))
        c["grads"] = rng.choice([dtype, dtype, "f32"])
        c["master"] = dtype != "f32" and rng.random() < 0.6
        widths = [int(_log(rng, 1, 4000)) for _ in range(rng.randint(2, 9))]
        c["layers"] = "-".join(map(str, widths))
    del c["name"]
    return c


# ---- the inputs a case describes ----

def _lengths(case):
    """Rows of each bag: a function of the case alone."""
    if case["equal"]:
        return np.full(case["bags"], case["mean"], np.int64)
    rs = np.random.RandomState((case["bags"] * 31 + case["mean"] * 7 + case["dim"]) % (1 << 31))
    return np.clip(rs.poisson(case["mean"], case["bags"]), 0, case["longest"]).astype(np.int64)


def _shapes(case):
    w = [int(x) for x in case["layers"].split("-")]
    return [s for i, o in zip(w[:-1], w[1:]) for s in ((o, i), (o,))]


def _thresholds(buckets, far):
    """The distances at which the buckets 1, 2, ... of a side begin: one for each distance up to half of them, the rest
    spread over the logarithm up to `far`."""
    exact = max(1, buckets // 2)
    t = list(range(1, exact + 1))
    for k in range(exact + 1, buckets):
        t.append(max(t[-1] + 1, math.ceil(exact * (far / exact) ** ((k - exact) / (buckets - exact)))))
    return t[:buckets - 1]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFF)


def _randn(g, *shape, dtype="f32", mean=0.0, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(TYPES[dtype])


def _prepare_scan(case, g):
    D, B, dt = case["dim"], case["bags"], case["dtype"]
    if case["mode"] == "step":
        s = {"state": _randn(g, case["slots"], D), "slots": torch.randperm(case["slots"], generator=g, device="cuda")[:B].contiguous(),
             "x": _randn(g, B, D, dtype=dt), "u": _randn(g, B, D, dtype=dt, mean=2.0, std=1.5)}
        N = B
    else:
        off = np.concatenate([[0], np.cumsum(_lengths(case))])
        N = int(off[-1])
        s = {"offsets": torch.from_numpy(off).cuda(), "x": _randn(g, N, D, dtype=dt), "longest": int(max(1, _lengths(case).max(initial=1))),
             "u": _randn(g, N, D, dtype=dt, mean=4.0 if case["mean"] > 1000 else 2.0, std=1.5),
             "h0": _randn(g, B, D) if case["h0"] else None}
        if case["mode"] == "train":
            s["dy"], s["dlast"] = _randn(g, N, D, dtype=dt, std=0.1), _randn(g, B, D, std=0.1)
    if own:
        from paper_2305_01515_amd import dense
        s["plan"] = dense.Scan(D, TYPES[dt], max_bags=B, max_rows=N, coupled=case["coupled"])
    return s


def _prepare_bias(case, g):
    B, H, lq, lk, dt = case["batch"], case["heads"], case["lq"], case["lk"], case["dtype"]
    thr = _thresholds(case["buckets"], case["far"])
    s = {"table": _randn(g, case["buckets"] * (2 if case["both"] else 1), H, std=0.5), "thresholds": thr,
         "thr": torch.tensor(thr, dtype=torch.int64, device="cuda"), "q_pos": None, "k_pos": None, "key_lengths": None,
         "q_offset": lk - lq if lq == 1 else 0}
    if case["times"]:
        gaps = (torch.empty(B, max(lq, lk), device="cuda").exponential_(generator=g) * 40_000 * torch.rand(B, max(lq, lk), generator=g, device="cuda") ** 6)
        stamps = 1_700_000_000 + gaps.to(torch.int64).cumsum(1)
        s["k_pos"] = stamps[:, :lk].contiguous()
        s["q_pos"] = stamps[:, lk - 1:lk].contiguous() if lq == 1 else stamps[:, :lq].contiguous()
    if case["lengths"]:
        s["key_lengths"] = torch.randint(0, lk + 1, (B,), generator=g, device="cuda")
    if case["mode"] == "add":
        s["scores"], s["scale"] = _randn(g, B, H, lq, lk, dtype=dt), 0.125
    if case["mode"] == "grad":
        s["dout"] = _randn(g, B, H, lq, lk, dtype=dt, std=0.1)
    if own:
        from paper_2305_01515_amd import dense
        s["plan"] = dense.RelativeBias(H, thr, bidirectional=case["both"])
    return s


def _prepare_adamw(case, g):
    shapes = _shapes(case)
    master = [_randn(g, *s, std=0.05) for s in shapes]
    s = {"params": [w.to(TYPES[case["dtype"]]) for w in master], "grads": [_randn(g, *s, dtype=case["grads"], std=0.01) for s in shapes],
         "decay": [DECAY if len(x) > 1 else 0.0 for x in shapes], "step": 100, "master": master if case["master"] else None}
    padded = [-(-math.prod(x) // BLOCK) * BLOCK for x in shapes]
    total = sum(padded)
    s["at"] = [sum(padded[:i]) for i in range(len(padded))]
    if case["bits"] == 32:
        s["m"] = _randn(g, total, std=0.003)
        s["v"] = _randn(g, total, std=0.01).square_()
    else:
        sign = torch.randint(0, 2, (total,), generator=g, device="cuda", dtype=torch.uint8) * 128
        s["m"] = torch.randint(0, 127, (total,), generator=g, device="cuda", dtype=torch.uint8) + sign
        s["v"] = torch.randint(1, 127, (total,), generator=g, device="cuda", dtype=torch.uint8)
        s["m_scale"] = torch.rand(total // BLOCK, generator=g, device="cuda") * 2e-5 + 1e-6
        s["v_scale"] = torch.rand(total // BLOCK, generator=g, device="cuda") * 2e-5 + 1e-5
    for a, n in zip(s["at"], (math.prod(x) for x in shapes)):  # what pads a tensor's last block is zero
        pad = -(-n // BLOCK) * BLOCK
        s["m"][a + n:a + pad] = 0
        s["v"][a + n:a + pad] = 0
    if own:
        from paper_2305_01515_amd import dense
        states = {k: s[k] for k in ("m", "v", "m_scale", "v_scale") if k in s}
        s["plan"] = dense.AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=s["decay"], state_bits=case["bits"],
                                master=s["master"], seed=SEED, step=s["step"], states=states)
    return s


def prepare(case, seed):
    g = _gen(seed)
    s = {"scan": _prepare_scan, "bias": _prepare_bias, "adamw": _prepare_adamw}[case["op"]](case, g)
    s["case"] = case
    return s


# ---- the plain forms ----

def _linear_scan(a, b, longest):
    """h_t = a_t h_{t-1} + b_t along the first axis, a_t = 0 where a bag starts: partial results of twice the rows each time."""
    k = 1
    while k < longest:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _plain_scan(s):
    case = s["case"]
    x, u, dt = s["x"].float(), s["u"].float(), s["x"].dtype
    f = 1 / (1 + torch.exp(-u))
    i = 1 / (1 + torch.exp(u)) if case["coupled"] else torch.ones_like(f)
    if case["mode"] == "step":
        h = f * s["state"][s["slots"]] + i * x
        s["state"][s["slots"]] = h
        return {"y": h.to(dt), "state": s["state"]}
    off = s["offsets"]
    full = off[1:] > off[:-1]
    first, end = off[:-1][full], off[1:][full] - 1
    h0 = s["h0"] if s["h0"] is not None else torch.zeros(case["bags"], case["dim"], device="cuda")
    a, b = f.clone(), i * x
    b[first] += f[first] * h0[full]
    a[first] = 0
    h = _linear_scan(a, b, s["longest"])
    last = h0.clone()
    last[full] = h[end]
    out = {"y": h.to(dt), "last": last}
    if case["mode"] == "forward":
        return out
    g = s["dy"].float().clone()
    g[end] += s["dlast"][full]
    a = torch.cat([f[1:], torch.zeros_like(f[:1])])  # the gate between a row and the next one
    a[end] = 0
    g = _linear_scan(a.flip(0), g.flip(0), s["longest"]).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first] = h0[full]
    out["dx"] = (g * i).to(dt)
    out["du"] = (g * (before - x if case["coupled"] else before) * f * (1 / (1 + torch.exp(u)))).to(dt)
    if s["h0"] is not None:
        out["dh0"] = s["dlast"].clone()
        out["dh0"][full] = g[first] * f[first]
    return out


def _buckets(s, case):
    """bucket and mask of every (sample, query, key); one sample where all are alike"""
    q = s["q_pos"] if s["q_pos"] is not None else torch.arange(case["lq"], device="cuda")[None] + s["q_offset"]
    k = s["k_pos"] if s["k_pos"] is not None else torch.arange(case["lk"], device="cuda")[None]
    d = k[:, None, :] - q[:, :, None]
    a = d.abs() if case["both"] else (-d).clamp(min=0)
    n = torch.bucketize(a, s["thr"], right=True)
    if case["both"]:
        n = n + (d > 0) * case["buckets"]
    off = torch.zeros_like(d, dtype=torch.bool)
    if case["causal"]:
        off = off | (d > 0)
    if s["key_lengths"] is not None:
        off = off | (torch.arange(case["lk"], device="cuda") >= s["key_lengths"][:, None, None])
    return n, off


def _plain_bias(s):
    case = s["case"]
    n, off = _buckets(s, case)
    if case["mode"] == "grad":
        d = s["dout"].float()
        if case["causal"] or case["lengths"]:
            d = d.masked_fill(off[:, None], 0.0)
        if n.shape[0] == 1:
            d = d.sum(0, keepdim=True)
        d = d.transpose(0, 1).reshape(case["heads"], -1)
        hot = (n.reshape(-1, 1) == torch.arange(s["table"].shape[0], device="cuda")).float()
        return {"dtable": torch.mm(d, hot).t().contiguous()}
    out = s["table"][n].permute(0, 3, 1, 2)
    if case["mode"] == "add":
        out = s["scores"].float() * s["scale"] + out
    if case["causal"] or case["lengths"]:
        out = out.masked_fill(off[:, None], -math.inf)
    return {"out": out.to(TYPES[case["dtype"]]).contiguous()}


def _mix(x):
    """32 pseudorandom bits of a 32-bit word (in an int64 tensor or a Python integer)"""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _to_8_bits(q, random):
    """code of 0 <= q <= 448 in the 8-bit type of 4 exponent and 3 mantissa bits; `random` (16 bits) is what decides how often
    a value between two codes becomes the upper one"""
    normal = ((q.view(torch.int32) + (random << 4)) >> 20) - 960
    small = torch.floor(q * 512 + random * (1 / 65536)).to(torch.int32)
    return torch.where(q < 2 ** -6, small, normal)


def _quantise(x, random, floor):
    """codes [blocks, BLOCK] and scales of x: the largest of a block is 448 scales"""
    top = x.abs().amax(1, keepdim=True)
    usable = (top < math.inf) & (top > 0)
    q = (x.abs() * (448 / top)).clamp(max=448)
    code = torch.where(usable, _to_8_bits(torch.where(usable, q, 0.0), random).clamp(max=126), 0)
    if floor:
        code = torch.where(usable & (x > 0), code.clamp(min=1), code)
    return (code + (x < 0) * usable * 128).to(torch.uint8), (top / 448)[:, 0]


def _plain_adamw(s):
    case, step = s["case"], s["step"] + 1
    s["step"] = step
    eight = case["bits"] == 8
    rate, root = LR / (1 - BETA1 ** step), 1 / math.sqrt(1 - BETA2 ** step)
    for t, (p, g, a, decay) in enumerate(zip(s["params"], s["grads"], s["at"], s["decay"])):
        n = p.numel()
        pad = -(-n // BLOCK) * BLOCK
        w = (s["master"][t] if case["master"] else p).reshape(-1).float()
        g = torch.nn.functional.pad(g.reshape(-1).float(), (0, pad - n))
        m, v = s["m"][a:a + pad], s["v"][a:a + pad]
        if eight:
            blocks = slice(a // BLOCK, (a + pad) // BLOCK)
            m = (m.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["m_scale"][blocks, None]).reshape(-1)
            r = (v.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["v_scale"][blocks, None]).reshape(-1)
            v = r * r
        m = m * BETA1 + g * (1 - BETA1)
        v = v * BETA2 + (g * g) * (1 - BETA2)
        r = torch.sqrt(v)
        w = w * (1 - LR * decay) - ((m * rate) / (r * root + EPS))[:n]
        p.reshape(-1).copy_(w)
        if case["master"]:
            s["master"][t].reshape(-1).copy_(w)
        if eight:
            key = _mix(_mix(_mix(SEED) ^ step) ^ t)
            word = _mix((torch.arange(pad, device="cuda") * 0x9E3779B9 + key) & 0xFFFFFFFF).to(torch.int64)
            word = word.view(-1, BLOCK)
            code, s["m_scale"][blocks] = _quantise(m.view(-1, BLOCK), (word >> 16).to(torch.int32), False)
            s["m"][a:a + pad] = code.reshape(-1)
            code, s["v_scale"][blocks] = _quantise(r.view(-1, BLOCK), (word & 0xFFFF).to(torch.int32), True)
            s["v"][a:a + pad] = code.reshape(-1)
        else:
            s["m"][a:a + pad], s["v"][a:a + pad] = m, v


# ---- one pass ----

def _own_scan(s):
    case, plan = s["case"], s["plan"]
    if case["mode"] == "step":
        return {"y": plan.step(s["state"], s["x"], s["u"], s["slots"]), "state": s["state"]}
    y, last, saved = plan.forward(s["x"], s["u"], s["offsets"], s["h0"], save=case["mode"] == "train")
    out = {"y": y, "last": last}
    if case["mode"] == "train":
        out["dx"], out["du"], dh0 = plan.backward(s["x"], s["u"], s["offsets"], saved, s["dy"], s["dlast"], s["h0"])
        if dh0 is not None:
            out["dh0"] = dh0
    return out


def _own_bias(s):
    case, plan = s["case"], s["plan"]
    where = {k: s[k] for k in ("q_pos", "k_pos", "q_offset", "key_lengths")}
    if case["mode"] == "grad":
        return {"dtable": plan.backward(s["dout"], causal=case["causal"], **where)}
    if case["mode"] == "add":
        return {"out": plan.forward(s["table"], scores=s["scores"], scale=s["scale"], causal=case["causal"], **where)}
    return {"out": plan.forward(s["table"], shape=(case["batch"], case["lq"], case["lk"]), dtype=TYPES[case["dtype"]],
                                causal=case["causal"], **where)}


def run(state):
    op = state["case"]["op"]
    if op == "adamw":
        state["plan"].step(state["grads"]) if own else _plain_adamw(state)
        out = {"params": state["params"], "master": state["master"] or [], "m": state["m"], "v": state["v"]}
        if state["case"]["bits"] == 8:  # the codes are numbers of this type, times the scale of their block
            out = dict(out, m=state["m"].view(torch.float8_e4m3fn), v=state["v"].view(torch.float8_e4m3fn),
                       m_scale=state["m_scale"], v_scale=state["v_scale"])
        return out
    if op == "scan":
        return _own_scan(state) if own else _plain_scan(state)
    return _own_bias(state) if own else _plain_bias(state)


def work(case):
    if case["op"] == "scan":
        es = 4 if case["dtype"] == "f32" else 2
        B, D = case["bags"], case["dim"]
        if case["mode"] == "step":
            return {"bytes": B * (D * (3 * es + 8) + 8), "flops": 8 * B * D}
        N = int(_lengths(case).sum())
        if case["mode"] == "forward":
            return {"bytes": 3 * es * N * D + 4 * B * D * (1 + case["h0"]) + 8 * (B + 1), "flops": 8 * N * D}
        return {"bytes": 6 * es * N * D + 4 * B * D * (2 + 2 * case["h0"]) + 8 * (B + 1), "flops": 24 * N * D}
    if case["op"] == "bias":
        es = 4 if case["dtype"] == "f32" else 2
        B, H, lq, lk = case["batch"], case["heads"], case["lq"], case["lk"]
        table = 4 * H * case["buckets"] * (2 if case["both"] else 1)
        other = table + (8 * B * (lq + lk) if case["times"] else 0) + (8 * B if case["lengths"] else 0)
        return {"bytes": B * H * lq * lk * es * (2 if case["mode"] == "add" else 1) + other, "flops": 2 * B * H * lq * lk}
    n = sum(math.prod(s) for s in _shapes(case))
    p, g = (4 if case[k] == "f32" else 2 for k in ("dtype", "grads"))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    weight = p + 8 if case["master"] else 2 * p
    return {"bytes": n * (weight + g + state), "flops": 15 * n}


# ---- the operators' definitions in 64 bits ----

def _exact_scan(a, b):
    """h_t = a_t h_{t-1} + b_t by blocks of rows: every block from a zero state, then the states before the blocks in turn"""
    n, d = b.shape
    blocks = -(-n // 128)
    a, b = (torch.nn.functional.pad(t, (0, 0, 0, blocks * 128 - n)).view(blocks, 128, d) for t in (a, b))
    h, p = torch.empty_like(b), torch.empty_like(a)
    state, prod = torch.zeros_like(b[:, 0]), torch.ones_like(a[:, 0])
    for j in range(128):
        state, prod = a[:, j] * state + b[:, j], prod * a[:, j]
        h[:, j], p[:, j] = state, prod
    carry, before = torch.zeros_like(state[0]), torch.empty_like(state)
    for k in range(blocks):
        before[k] = carry
        carry = prod[k] * carry + state[k]
    return (h + p * before[:, None]).view(-1, d)[:n]


def _exact_of_scan(case, s):
    x, u = s["x"].double(), s["u"].double()
    f = torch.sigmoid(u)
    i = torch.sigmoid(-u) if case["coupled"] else torch.ones_like(f)
    if case["mode"] == "step":
        state = s["state"].double()
        h = torch.lerp(x, state[s["slots"]], f) if case["coupled"] else torch.addcmul(x, f, state[s["slots"]])
        state[s["slots"]] = h
        return {"y": h, "state": state}
    off = s["offsets"].tolist()
    bags = [b for b in range(case["bags"]) if off[b + 1] > off[b]]
    first, end = [off[b] for b in bags], [off[b + 1] - 1 for b in bags]
    h0 = s["h0"].double() if case["h0"] else torch.zeros(case["bags"], case["dim"], dtype=torch.float64, device="cuda")
    before = torch.zeros_like(x)
    before[first] = h0[bags]
    a = f.clone()
    a[first] = 0
    h = _exact_scan(a, i * x + f * before)
    last = h0.clone()
    last[bags] = h[end]
    out = {"y": h, "last": last}
    if case["mode"] == "train":
        g, carry = s["dy"].double(), torch.roll(f, -1, 0)
        g[end] += s["dlast"].double()[bags]
        carry[end] = 0
        g = _exact_scan(carry.flip(0), g.flip(0)).flip(0)
        keep = torch.roll(h, 1, 0)
        keep[first] = h0[bags]
        out["dx"] = g * i
        out["du"] = g * (keep - x if case["coupled"] else keep) * f * torch.sigmoid(-u)
        if case["h0"]:
            out["dh0"] = s["dlast"].double()
            out["dh0"][bags] = (g * f)[first]
    return out


def _exact_of_bias(case, s):
    """sample by sample where the distances are a sample's own"""
    B, H, lq, lk = case["batch"], case["heads"], case["lq"], case["lk"]
    table, n = s["table"].double(), case["buckets"]
    edges = [-1] + s["thresholds"] + [1 << 62]
    total, outs = torch.zeros_like(table), []
    for b0 in range(0, B, 32):
        rows = range(b0, min(B, b0 + 32))
        q = s["q_pos"][b0:b0 + 32] if case["times"] else (torch.arange(lq, device="cuda") + s["q_offset"]).expand(len(rows), lq)
        k = s["k_pos"][b0:b0 + 32] if case["times"] else torch.arange(lk, device="cuda").expand(len(rows), lk)
        ahead = k[:, None] - q[..., None]
        seen = torch.ones_like(ahead, dtype=torch.bool)
        if case["causal"]:
            seen &= ahead <= 0
        if case["lengths"]:
            seen &= torch.arange(lk, device="cuda") < s["key_lengths"][b0:b0 + 32, None, None]
        out = torch.zeros(len(rows), H, lq, lk, dtype=torch.float64, device="cuda")
        for c in range(table.shape[0]):
            lo, hi = edges[c % n], edges[c % n + 1]
            dist = ahead if c >= n else -ahead
            inside = (dist >= lo) & (dist < hi) & (dist > 0) if c >= n else (dist >= (lo if c else 0)) & (dist < hi)
            if not case["both"] and c == 0:
                inside = dist < hi
            if case["mode"] == "grad":
                d = torch.where((inside & seen)[:, None], s["dout"][b0:b0 + 32].double(), 0.0)
                total[c] += d.sum((0, 2, 3))
            else:
                out += inside[:, None] * table[c][:, None, None]
        if case["mode"] == "add":
            out += s["scores"][b0:b0 + 32].double() * s["scale"]
        outs.append(torch.where(seen[:, None], out, -math.inf) if case["mode"] != "grad" else None)
    return {"dtable": total} if case["mode"] == "grad" else {"out": torch.cat(outs)}


def _exact_codes(x, random, floor):
    """values (in scales) and scales of a block's codes: between two neighbouring codes the upper one where the distance from
    the lower, as a share of theirs, and the random share make one"""
    top = x.abs().max(1, keepdim=True).values
    q = torch.where(top > 0, x.abs() / top * 448, 0.0)
    gap = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -6))) - 3)
    lower = torch.floor(q / gap)
    code = (lower + (q / gap - lower + random / 65536 >= 1)) * gap
    if floor:
        code = torch.where((x > 0) & (code == 0), 2.0 ** -9, code)
    return (code.clamp(max=448) * torch.sign(x)).reshape(-1), top[:, 0] / 448


def _exact_of_adamw(case, s):
    step, eight = s["step"] + 1, case["bits"] == 8
    out = {"params": [], "master": [], "m": s["m"].double() if not eight else s["m"].view(torch.float8_e4m3fn).double(),
           "v": s["v"].double() if not eight else s["v"].view(torch.float8_e4m3fn).double()}
    if eight:
        out["m_scale"], out["v_scale"] = s["m_scale"].double(), s["v_scale"].double()
    for t, p in enumerate(s["params"]):
        n, at = p.numel(), s["at"][t]
        blocks = -(-n // BLOCK)
        part, scales = slice(at, at + blocks * BLOCK), slice(at // BLOCK, at // BLOCK + blocks)
        g = torch.zeros(blocks * BLOCK, dtype=torch.float64, device="cuda")
        g[:n] = s["grads"][t].reshape(-1)
        m, v = out["m"][part].clone(), out["v"][part].clone()
        if eight:
            m = m * out["m_scale"][scales].repeat_interleave(BLOCK)
            v = (v * out["v_scale"][scales].repeat_interleave(BLOCK)) ** 2
        m += (g - m) * (1 - BETA1)
        v += (g ** 2 - v) * (1 - BETA2)
        w = (s["master"][t] if case["master"] else p).double().reshape(-1)
        mean, spread = m[:n] / (1 - BETA1 ** step), (v[:n] / (1 - BETA2 ** step)).sqrt()
        w = (w - LR * s["decay"][t] * w - LR * mean / (spread + EPS)).view(p.shape)
        out["params"].append(w)
        if case["master"]:
            out["master"].append(w)
        if eight:
            key = _mix(_mix(_mix(SEED) ^ step) ^ t)
            word = _mix((torch.arange(blocks * BLOCK, device="cuda") * 0x9E3779B9 + key) % (1 << 32)).view(-1, BLOCK)
            out["m"][part], out["m_scale"][scales] = _exact_codes(m.view(-1, BLOCK), word // 65536, False)
            out["v"][part], out["v_scale"][scales] = _exact_codes(v.sqrt().view(-1, BLOCK), word % 65536, True)
        else:
            out["m"][part], out["v"][part] = m, v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"scan": _exact_of_scan, "bias": _exact_of_bias, "adamw": _exact_of_adamw}[case["op"]](case, s)
