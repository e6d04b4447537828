"""Chunks that hear from each other: bags short on average, so that this form runs, with a long one among them, and what makes the waits
safe.  A chunk that has looked for long at what another has yet to say goes through its bag's rows itself.  libtbe.so looks 1024 times
first, which no size provokes; here are builds of it that look 0 and 16 times.  Values on the bars of test_gpu_scan."""
import os

import pytest
import torch

from test_gpu_scan import run_and_compare

pytestmark = pytest.mark.gpu

BAGS = {"short": [7, 0, 30, 1, 64, 0, 3] * 60, "long_first": [5000] + [3] * 400, "long_last": [3] * 400 + [5000], "long_amid": [1, 2, 0] * 150 + [4000] + [9] * 150,
        "two_long": [40] * 20 + [2500] + [1] * 300 + [2500] + [5] * 20, "ends_at_chunks": [128] * 40, "ends_before_chunks": [127] + [128] * 39 + [1]}


@pytest.fixture(params=[0, 1], ids=["looks_0", "looks_16"])
def impatient(request, monkeypatch):
    from paper_2305_01515_amd import build, dense, tbe
    path = build.IMPATIENT[request.param]
    if not os.path.exists(path):
        build.build()
    monkeypatch.setattr(tbe, "LIB_PATH", path)
    monkeypatch.setattr(tbe, "_lib", None)
    monkeypatch.setattr(dense, "_ready", False)
    assert dense._lib()._name == path
    return request.param


@pytest.mark.parametrize("dim,dtype,h0", [(64, "f32", "own"), (128, "bf16", "none"), (72, "f16", "one")])
@pytest.mark.parametrize("name", list(BAGS))
def test_long_bags_among_short_ones(name, dim, dtype, h0):
    plan, (x, u, off, s0, dy, dlast), outs = run_and_compare(BAGS[name], dim, dtype, True, h0, seed=dim)
    for _ in range(3):  # states are the same bits wherever a chunk finds them
        y, last, saved = plan.forward(x, u, off, s0, save=True)
        for a, b in zip(outs, (y, last, saved, *plan.backward(x, u, off, saved, dy, dlast, s0))):
            assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dim,dtype,coupled", [(64, "f32", True), (64, "f32", False), (128, "bf16", True), (33, "f16", True)])
@pytest.mark.parametrize("name", list(BAGS))
def test_chunks_that_do_not_wait(impatient, name, dim, dtype, coupled):
    run_and_compare(BAGS[name], dim, dtype, coupled, "own", seed=dim + 1)
