"""The first chunk of a call (the last one for the gradient) says its state and no map, whatever its gates hold and wherever the bags begin:
chunks behind it look no further.  Offsets that do not begin at 0 or end at the rows are reported and the next call is as if nothing had been;
a NaN gate behind the start of a bag stays in its bag.  Many chunks of short bags, so that chunks hear from each other, on the
ordinary build and on those that do not wait (there, which chunks were waited for decides the last bits: values on the bars of
test_gpu_scan)."""
import pytest
import torch

from test_gpu_scan import TYPES, f64, inputs, near, reference
from test_gpu_scan_waits import impatient  # noqa: F401

pytestmark = pytest.mark.gpu

BAGS = [7, 30, 1, 64, 3] * 120  # 12600 rows


NAMES = ("y", "last", "dx", "du", "dh0")


def bars(lengths, x, u, dy, dlast, h0):
    f = lambda t: f64(t.cpu())  # noqa: E731
    return reference(f(x), f(u), lengths, f(h0), f(dy), f(dlast), True)


def within(name, dtype, got, want, keep):
    value, bar = want[name]
    keep = keep.cpu().numpy()
    half = TYPES[dtype][1] if dtype != "f32" and name in ("y", "dx", "du") else 0.0
    near(name, got[torch.from_numpy(keep).cuda()], (value[keep], bar[keep]), half, 2.0 ** -25 if half and dtype == "f16" else 1e-37)


def refused(dim, dtype):
    from paper_2305_01515_amd.dense import Scan
    from paper_2305_01515_amd.tbe import TbeError
    x, u, dy, dlast, h0, off = [t.cuda() for t in inputs(BAGS, dim, dtype, "own", seed=dim)]
    n, bags = x.shape[0], len(BAGS)
    plan = Scan(dim, x.dtype, bags, n)
    y, last, saved = plan.forward(x, u, off, h0, save=True)
    want = plan.backward(x, u, off, saved, dy, dlast, h0)
    plan.check()
    for skip in (1, 700, 5000):  # rows in front of the first bag or behind the last one that belong to none
        front, back = off.clone(), off.clone()
        front[front < skip] = skip
        back[back > n - skip] = n - skip
        both = torch.maximum(front, torch.tensor(skip).cuda()).clamp(max=n - skip)
        for bad in (front, back, both, torch.full_like(off, n // 2)):
            room = torch.full((n + 200, dim), 7.0, dtype=x.dtype, device="cuda")
            plan.forward(x, u, bad, h0, y=room[100:100 + n], save=True)
            with pytest.raises(TbeError) as e:
                plan.check()
            assert e.value.code == -1
            plan.backward(x, u, bad, saved, dy, dlast, h0)
            with pytest.raises(TbeError):
                plan.check()
            assert bool((room[:100] == 7).all()) and bool((room[100 + n:] == 7).all())
    again, last2, saved2 = plan.forward(x, u, off, h0, save=True)
    plan.check()
    return (x, u, dy, dlast, h0), (y, last, *want), (again, last2, *plan.backward(x, u, off, saved2, dy, dlast, h0))


CASES = [(64, "f32"), (128, "bf16"), (33, "f16"), (8, "f32")]


@pytest.mark.parametrize("dim,dtype", CASES)
def test_refused_offsets_over_many_chunks(dim, dtype):
    _, before, after = refused(dim, dtype)
    for a, b in zip(before, after):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dim,dtype", CASES)
def test_refused_offsets_where_chunks_do_not_wait(impatient, dim, dtype):  # noqa: F811
    args, _, after = refused(dim, dtype)
    want = bars(BAGS, *args)
    for name, got in zip(NAMES, after):
        within(name, dtype, got, want, torch.ones(got.shape[0], dtype=torch.bool))


def poisoned(dim, dtype, value, exact):
    """a bag from the middle of the first chunk on over several chunks, one that ends in the last chunk, gates of both are `value` in the
    first and the last chunk"""
    from paper_2305_01515_amd.dense import Scan
    chunk = 8192 // dim
    lengths = [5, chunk // 2, 3 * chunk, 2] + [20] * (60 * chunk // 20) + [3, 3 * chunk, 4]
    x, u, dy, dlast, h0, off = [t.cuda() for t in inputs(lengths, dim, dtype, "own", seed=dim + 1)]
    plan = Scan(dim, x.dtype, len(lengths), x.shape[0])

    def everything(u):
        y, last, saved = plan.forward(x, u, off, h0, save=True)
        out = (y, last, *plan.backward(x, u, off, saved, dy, dlast, h0))
        plan.check()
        return out
    clean = everything(u)
    want = None if exact else bars(lengths, x, u, dy, dlast, h0)
    for bag, at in ((2, 3), (len(lengths) - 2, 3 * chunk - 1)):
        row = int(off[bag]) + at
        dirty = u.clone()
        dirty[row, ::3] = value
        got = everything(dirty)
        rows = slice(int(off[bag]), int(off[bag + 1]))
        assert bool(got[0][row:rows.stop, ::3].isnan().all())
        for name, a, b in zip(NAMES, got, clean):
            keep = torch.ones(a.shape[0], dtype=torch.bool, device="cuda")
            keep[rows if name in ("y", "dx", "du") else bag] = False
            if exact:
                assert torch.equal(a[keep], b[keep]), (bag, name)
            else:
                within(name, dtype, a, want, keep)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dim,dtype", [(64, "f32"), (128, "bf16"), (32, "f16")])
def test_nan_gates_in_the_first_and_the_last_chunk(dim, dtype, sign):
    poisoned(dim, dtype, torch.tensor(float("nan")).copysign(torch.tensor(float(sign))).item(), exact=True)


@pytest.mark.parametrize("dim,dtype", [(64, "f32"), (128, "bf16")])
def test_nan_gates_where_chunks_do_not_wait(impatient, dim, dtype):  # noqa: F811
    poisoned(dim, dtype, float("nan"), exact=False)
