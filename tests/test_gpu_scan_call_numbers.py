"""Marks and words carry the number of the call they are of, 32 and 30 bits of it, and memory that no call has written holds zeros: numbers whose bits are all zero
are passed over.  The builds that do not wait begin with the numbers 2^30 - 3 and 2^32 - 3."""
import pytest
import torch

from test_gpu_scan import f64, inputs, near, reference
from test_gpu_scan_waits import impatient  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths", [[3] * 20 + [2000, 1, 0, 900], [3000], [40] * 60])
def test_calls_around_the_ends_of_the_numbers(impatient, lengths):  # noqa: F811
    """a call of few rows first, so that later ones find marks and words that no call has written"""
    from paper_2305_01515_amd.dense import Scan
    dim = 64
    small = [t.cuda() for t in inputs([5], dim, "f32", "own", seed=1)]
    many = inputs(lengths, dim, "f32", "own", seed=2)
    x, u, dy, dlast, h0, off = [t.cuda() for t in many]
    args = [f64(many[k]) for k in (0, 1)] + [lengths] + [f64(many[k]) for k in (4, 2, 3)]
    want = reference(*args, True)
    for before in range(8):  # the large call has each number around the end once
        plan = Scan(dim, torch.float32, len(lengths), x.shape[0])
        for _ in range(before):
            plan.forward(small[0], small[1], small[5], small[4])
        y, last, saved = plan.forward(x, u, off, h0, save=True)
        dx, du, dh0 = plan.backward(x, u, off, saved, dy, dlast, h0)
        plan.check()
        for name, got in (("y", y), ("last", last), ("dx", dx), ("du", du), ("dh0", dh0)):
            near(name, got, want[name], 0.0, 1e-37)
