"""Lengths beyond the keys (and below zero) mask what a length of all keys (of none) masks, in every form: alone, added, both gradients, positions
as indices and given, rows shorter than a pack of 16 bytes among them.  Gradients are small whole numbers, so sums are exact."""
import math

import numpy as np
import pytest
import torch

from test_gpu_bias import Case, LOG, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("positions", ["index", "any"])
@pytest.mark.parametrize("keys", [1, 2, 3, 4, 5, 7, 8, 9, 45])
def test_lengths_outside_the_keys(keys, positions, dtype):
    lengths = [keys + 1, keys + 7, (1 << 63) - 1, -1, -(1 << 63), keys, 0]
    clamped = [min(max(n, 0), keys) for n in lengths]
    make = lambda n: Case(7, 3, 21, keys, LOG, both=True, lengths=n, positions=positions, offset=3, dtype=dtype, seed=keys)  # noqa: E731
    c, same = make(lengths), make(clamped)
    assert np.array_equal(c.masked, same.masked)
    plan, dt = c.plan(), TYPES[dtype][0]
    got = plan.forward(c.table.cuda(), shape=(7, 21, keys), dtype=dt, **c.where())
    c.check_values(got, None, 1.0, -math.inf)
    scores = c.scores()
    c.check_values(plan.forward(c.table.cuda(), scores=scores.cuda(), scale=0.5, **c.where()), scores, 0.5, -math.inf)
    dout = torch.randint(-3, 4, scores.shape, generator=c.g).to(dt).cuda()
    kept = np.where(c.masked[:, None], 0.0, dout.double().cpu().numpy())
    want = torch.tensor(np.stack([np.where((c.n == k)[:, None], kept, 0.0).sum((0, 2, 3)) for k in range(c.table.shape[0])]))
    assert torch.equal(plan.backward(dout, **c.where()).double().cpu(), want)
    dtable, dscores = plan.backward(dout, want_dscores=True, **c.where())
    assert torch.equal(dtable.double().cpu(), want) and np.array_equal(dscores.double().cpu().numpy(), kept)
