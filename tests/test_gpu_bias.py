"""The learned bias by buckets of a distance against its definition, element by element, and the table's gradient in 64 bits.

Bars.  A biased score is two roundings in fp32 (product, sum) and one to its type: 2 eps of |score scale| + |bias| and half an ulp of
the result.  A bias alone is exact up to that last rounding.  A sum of n gradients in fp32 is off by (log2(n) + 2048) eps of the sum of
their magnitudes if nothing longer than 2048 numbers is added one after another; the bar takes n instead where n is smaller."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
TYPES = {"f32": (torch.float32, EPS), "f16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}


def buckets_of(q, k, thresholds, both):
    """numpy int64 [batch, queries, keys]: by counting, no search"""
    d = k[:, None, :] - q[:, :, None]
    a = np.abs(d) if both else np.maximum(-d, 0)
    n = np.zeros_like(a)
    for t in thresholds:
        n += a >= t
    return n + (len(thresholds) + 1) * ((d > 0) & both), d


class Case:
    def __init__(self, batch, heads, lq, lk, thresholds, both=False, causal=False, lengths=None, positions="index", offset=0, dtype="f32", seed=0):
        g = torch.Generator().manual_seed(seed)
        rs = np.random.RandomState(seed)
        self.batch, self.heads, self.lq, self.lk, self.dtype = batch, heads, lq, lk, dtype
        self.thresholds, self.both, self.causal, self.offset = thresholds, both, causal, offset
        self.table = torch.randn((len(thresholds) + 1) * (1 + both), heads, generator=g)
        self.q_pos = self.k_pos = None
        q, k = np.arange(lq)[None].repeat(batch, 0) + offset, np.arange(lk)[None].repeat(batch, 0)
        if positions == "times":  # far beyond 32 bits, with equal neighbours
            k = 1_700_000_000_000 + np.cumsum(rs.randint(0, 4, (batch, lk)) * 10 ** rs.randint(0, 7, (batch, lk)), 1)
            q = k[:, -lq:].copy() if lq <= lk else 1_700_000_000_000 + np.sort(rs.randint(0, 10 ** 9, (batch, lq)), 1)
        if positions == "any":  # no order at all, negative ones too
            k, q = rs.randint(-500, 500, (batch, lk)), rs.randint(-500, 500, (batch, lq))
        if positions != "index":
            self.q_pos, self.k_pos = torch.from_numpy(q.astype(np.int64)), torch.from_numpy(k.astype(np.int64))
        self.n, self.d = buckets_of(q.astype(np.int64), k.astype(np.int64), thresholds, both)
        self.masked = np.zeros((batch, lq, lk), bool)
        self.lengths = None
        if causal:
            self.masked |= self.d > 0
        if lengths is not None:
            self.lengths = torch.tensor((lengths * batch)[:batch], dtype=torch.int64)
            self.masked |= np.arange(lk)[None, None] >= self.lengths.numpy()[:, None, None]
        self.bias = self.table.double().numpy()[self.n].transpose(0, 3, 1, 2)
        self.g = g

    def scores(self):
        return torch.randn(self.batch, self.heads, self.lq, self.lk, generator=self.g).to(TYPES[self.dtype][0])

    def where(self):
        cu = lambda t: None if t is None else t.cuda()  # noqa: E731
        return dict(q_pos=cu(self.q_pos), k_pos=cu(self.k_pos), q_offset=self.offset, key_lengths=cu(self.lengths), causal=self.causal)

    def plan(self):
        from paper_2305_01515_amd.dense import RelativeBias
        return RelativeBias(self.heads, self.thresholds, bidirectional=self.both)

    def check_values(self, got, scores, scale, mask_value):
        half = TYPES[self.dtype][1]
        mask = np.broadcast_to(self.masked[:, None], got.shape)
        got = got.double().cpu().numpy()
        want = self.bias + (0 if scores is None else scores.double().numpy() * scale)
        sizes = np.abs(self.bias) + (0 if scores is None else np.abs(scores.double().numpy() * scale))
        limit = (0 if scores is None else 2 * EPS) * sizes + half * np.abs(want) * (1 + 4 * EPS) + (2.0 ** -25 if self.dtype == "f16" else 0)
        assert (np.abs(got - want)[~mask] <= limit[~mask]).all()
        assert (got[mask] == float(torch.tensor(mask_value).to(TYPES[self.dtype][0]))).all()

    def check_gradient(self, got, dout):
        d = np.where(self.masked[:, None], 0.0, dout.double().cpu().numpy())
        for c in range(self.table.shape[0]):
            inside = (self.n == c)[:, None] & ~self.masked[:, None]
            count = int(inside.sum())
            part = np.where(inside, d, 0.0)
            want, sizes = part.sum((0, 2, 3)), np.abs(part).sum((0, 2, 3))
            bar = min(count, math.log2(count + 2) + 2048) * EPS * sizes
            assert (np.abs(got[c].double().cpu().numpy() - want) <= bar).all(), (c, count)


LOG = [1, 2, 3, 4, 6, 9, 16, 27, 40, 64]
CASES = {
    "square": dict(batch=2, heads=3, lq=70, lk=70, thresholds=LOG, both=True),
    "causal": dict(batch=2, heads=4, lq=129, lk=129, thresholds=LOG, causal=True),
    "wide": dict(batch=1, heads=2, lq=33, lk=517, thresholds=LOG, both=True, offset=200),
    "tall": dict(batch=1, heads=2, lq=300, lk=5, thresholds=LOG, both=True),
    "one_token": dict(batch=5, heads=8, lq=1, lk=1001, thresholds=LOG, offset=1000, lengths=[0, 1, 500, 1001, 1000]),
    "one_key": dict(batch=3, heads=2, lq=9, lk=1, thresholds=LOG, both=True),
    "one": dict(batch=1, heads=1, lq=1, lk=1, thresholds=[], both=False),
    "one_bucket": dict(batch=2, heads=2, lq=20, lk=31, thresholds=[], both=True),
    "rows_left_empty": dict(batch=4, heads=2, lq=40, lk=64, thresholds=LOG, both=True, causal=True, lengths=[0, 3, 64, 10], offset=-10),
    "far_offset": dict(batch=1, heads=2, lq=17, lk=40, thresholds=[1, 5, 1 << 33], both=True, offset=1 << 33),
    "times": dict(batch=3, heads=4, lq=199, lk=199, thresholds=[1, 2, 4, 30, 500, 10 ** 5, 10 ** 7], positions="times", causal=True, lengths=[199, 7, 0]),
    "times_both": dict(batch=2, heads=2, lq=65, lk=130, thresholds=list(range(1, 120)) + [10 ** 4, 10 ** 8], positions="times", both=True),
    "times_newest": dict(batch=6, heads=8, lq=1, lk=333, thresholds=[1, 100, 10 ** 6], positions="times", lengths=[333, 0, 1, 300, 20, 5]),
    "any_order": dict(batch=2, heads=2, lq=50, lk=77, thresholds=LOG, positions="any", both=True, causal=True),
    "many_buckets": dict(batch=1, heads=2, lq=150, lk=150, thresholds=list(range(1, 128)), both=True),
    "long": dict(batch=1, heads=1, lq=700, lk=1500, thresholds=LOG, both=True, offset=400),
}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("name", list(CASES))
def test_values_and_gradients(name, dtype):
    c = Case(dtype=dtype, seed=len(name), **CASES[name])
    plan, dt = c.plan(), TYPES[dtype][0]
    got = plan.forward(c.table.cuda(), shape=(c.batch, c.lq, c.lk), dtype=dt, **c.where())
    c.check_values(got, None, 1.0, -math.inf)
    scores = c.scores()
    got = plan.forward(c.table.cuda(), scores=scores.cuda(), scale=0.3, mask_value=-1e4, **c.where())
    c.check_values(got, scores, float(np.float32(0.3)), -1e4)
    dout = c.scores().cuda()
    dtable, dscores = plan.backward(dout, want_dscores=True, scale=0.5, **c.where())
    c.check_gradient(dtable, dout)
    masked = torch.from_numpy(np.broadcast_to(c.masked[:, None], dout.shape).copy()).cuda()
    assert torch.equal(dscores, torch.where(masked, 0.0, dout.float() * 0.5).to(dt))
    assert torch.equal(dtable, plan.backward(dout, **c.where()))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("name", ["square", "rows_left_empty", "times", "one_token"])
def test_strides_and_unaligned_starts(name, dtype):
    """scores and gradients cut out of wider ones, with heads before samples, and starting at odd elements"""
    c = Case(dtype=dtype, seed=5, **CASES[name])
    plan, dt = c.plan(), TYPES[dtype][0]
    scores = c.scores()
    for shift in (0, 1, 3):
        wide = torch.zeros(c.heads, c.batch, c.lq, c.lk + 5, dtype=dt, device="cuda")
        view = wide.transpose(0, 1)[..., shift:shift + c.lk]
        view.copy_(scores)
        room = torch.full_like(wide, 3.0)
        out = room.transpose(0, 1)[..., shift:shift + c.lk]
        plan.forward(c.table.cuda(), scores=view, scale=2.0, out=out, **c.where())
        c.check_values(out, scores, 2.0, -math.inf)
        assert bool((room[..., :shift] == 3).all()) and bool((room[..., shift + c.lk:] == 3).all())
        plan.forward(c.table.cuda(), scores=view, scale=2.0, out=view, **c.where())  # in place
        assert torch.equal(view, out)
        view.copy_(scores)
        c.check_gradient(plan.backward(view, **c.where()), scores)
    one = scores[:1].cuda().expand(scores.shape)  # a gradient that is the same for all samples
    c.check_gradient(plan.backward(one, **c.where()), scores[:1].expand(scores.shape))


@pytest.mark.parametrize("name", ["rows_left_empty", "times", "causal"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_what_masked_places_hold(name, dtype):
    """infinities, NaN and the type's lowest value where the mask is"""
    c = Case(dtype=dtype, seed=8, **CASES[name])
    plan, dt = c.plan(), TYPES[dtype][0]
    clean, dout = c.scores(), c.scores()
    masked = torch.from_numpy(np.broadcast_to(c.masked[:, None], clean.shape).copy())
    for value in (math.nan, math.inf, -math.inf, torch.finfo(dt).min):
        dirty, ddirty = clean.clone(), dout.clone()
        dirty[masked] = value
        ddirty[masked] = value
        for mask_value in (-math.inf, torch.finfo(dt).min):
            a = plan.forward(c.table.cuda(), scores=dirty.cuda(), mask_value=mask_value, **c.where())
            assert torch.equal(a, plan.forward(c.table.cuda(), scores=clean.cuda(), mask_value=mask_value, **c.where()))
        a, da = plan.backward(ddirty.cuda(), want_dscores=True, **c.where())
        b, db = plan.backward(dout.cuda(), want_dscores=True, **c.where())
        assert torch.equal(a, b) and torch.equal(da, db)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_tables_of_each_type(dtype):
    c = Case(2, 3, 20, 30, LOG, both=True, dtype="f32", seed=1)
    table = c.table.to(TYPES[dtype][0])
    c.bias = table.double().numpy()[c.n].transpose(0, 3, 1, 2)
    c.check_values(c.plan().forward(table.cuda(), shape=(2, 20, 30), dtype=torch.float32), None, 1.0, -math.inf)


def test_one_bias_for_all_samples_and_positions_shared():
    c = Case(1, 4, 60, 60, LOG, both=True, positions="any", seed=2)
    plan = c.plan()
    one = plan.forward(c.table.cuda(), shape=(1, 60, 60), dtype=torch.float32, **c.where())
    w = c.where()
    three = plan.forward(c.table.cuda(), shape=(3, 60, 60), dtype=torch.float32, q_pos=w["q_pos"].expand(3, 60), k_pos=w["k_pos"].expand(3, 60))
    assert torch.equal(three, one.expand(3, -1, -1, -1))


def test_gradient_against_differences_and_autograd():
    """the biased scores are linear in table and scores: a difference along a direction is the derivative up to rounding"""
    c = Case(2, 2, 30, 41, LOG, both=True, causal=True, seed=3)
    plan = c.plan()
    table, scores = c.table.cuda().requires_grad_(), c.scores().cuda().requires_grad_()
    weight = torch.randn(2, 2, 30, 41, generator=c.g).cuda()
    loss = lambda t, s: (plan(t, s, scale=0.7, mask_value=0.0, causal=True).double() * weight.double()).sum()  # noqa: E731
    loss(table, scores).backward()
    for p in (table, scores):
        way = torch.randn(p.shape, generator=c.g).cuda()
        with torch.no_grad():
            up, down = [(q + way if q is p else q, q - way if q is p else q) for q in (table, scores)], None
            diff = (loss(up[0][0], up[1][0]) - loss(up[0][1], up[1][1])) / 2
        want = (p.grad.double() * way.double()).sum()
        assert abs(float(diff - want)) < 1e-5 * float((p.grad.double() * way.double()).abs().sum())


def test_graph_replays():
    c = Case(4, 4, 50, 50, LOG, both=True, dtype="bf16", seed=6)
    plan, table, x = c.plan(), c.table.cuda(), c.scores().cuda()
    both = lambda: (plan.forward(table, scores=x), *plan.backward(x, want_dscores=True))  # noqa: E731
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both()
    for _ in range(4):
        x.copy_(c.scores())
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in outs]
        for a, b in zip(kept, both()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("heads", [1, 8, 20])
@pytest.mark.parametrize("count", [31, 32, 47, 48, 63, 64, 65, 95, 100, 126, 127])
@pytest.mark.parametrize("both", [False, True])
def test_numbers_of_buckets_and_heads(count, heads, both):
    """what a workgroup keeps of sums and of the table grows with both, and has to fit"""
    c = Case(2, heads, 21, 45, list(range(1, 2 * count, 2)), both=both, positions="any", causal=heads == 8, dtype="bf16" if count % 2 else "f32", seed=count)
    plan = c.plan()
    dt = TYPES[c.dtype][0]
    c.check_values(plan.forward(c.table.cuda(), shape=(2, 21, 45), dtype=dt, **c.where()), None, 1.0, -math.inf)
    dout = c.scores().cuda()
    c.check_gradient(plan.backward(dout, **c.where()), dout)
    i = Case(2, heads, 21, 45, list(range(1, 2 * count, 2)), both=both, causal=heads == 8, dtype=c.dtype, seed=count)
    i.check_gradient(i.plan().backward(dout, **i.where()), dout)


def test_empty_sizes():
    c = Case(1, 2, 5, 5, LOG, both=True)
    plan = c.plan()
    for shape in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        assert plan.forward(c.table.cuda(), shape=shape, dtype=torch.float32).numel() == 0
        assert torch.equal(plan.backward(torch.zeros(shape[0], 2, *shape[1:], device="cuda")), torch.zeros(22, 2, device="cuda"))


def test_log_thresholds():
    from paper_2305_01515_amd.dense import log_thresholds
    for n in (1, 2, 3, 8, 16, 32, 64, 128):
        t = log_thresholds(n, 128)
        assert len(t) == n - 1 and all(b > a for a, b in zip(t, t[1:])) and t[:1] in ([], [1])


def test_refusals():
    from paper_2305_01515_amd.dense import RelativeBias
    from paper_2305_01515_amd.tbe import TbeError
    for heads, thr in ((0, [1]), (5000, [1]), (2, [0]), (2, [3, 3]), (2, [2, 1]), (2, list(range(1, 200)))):
        with pytest.raises(TbeError) as e:
            RelativeBias(heads, thr)
        assert e.value.code == -1
    plan = RelativeBias(2, [1, 2])
    table, s = torch.zeros(3, 2).cuda(), torch.zeros(2, 2, 4, 5).cuda()
    for bad in (dict(table=torch.zeros(4, 2).cuda()), dict(table=table.double()), dict(scores=s.double()), dict(scores=s.transpose(2, 3)),
                dict(scores=s[:, :1]), dict(q_pos=torch.zeros(2, 5, dtype=torch.int64).cuda()), dict(k_pos=torch.zeros(2, 5).cuda()),
                dict(key_lengths=torch.zeros(3, dtype=torch.int64).cuda()), dict(out=torch.zeros(2, 2, 4, 6).cuda())):
        with pytest.raises(ValueError):
            plan.forward(**dict(dict(table=table, scores=s), **bad))
    with pytest.raises(ValueError):
        plan.backward(torch.zeros(2, 3, 4, 5).cuda())
