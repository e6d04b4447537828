"""Shared by the tests of the norm, the short convolution and the selective scan: types, inputs, layouts, the comparison with a result in 64 bits
and its bar."""
import numpy as np
import torch

EPS = 2.0 ** -24
TYPES = {"f32": (torch.float32, 0.0), "f16": (torch.float16, 2.0 ** -11), "bf16": (torch.bfloat16, 2.0 ** -8)}  # half a step of what is stored
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}  # half a step of the smallest numbers
RAGGED = [0, 1, 3, 0, 0, 17, 64, 63, 65, 2, 127, 128, 129, 0, 31, 255, 257, 1, 1, 0]


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int64)


def near(name, got, value, bar, dtype="f32"):
    """|got - value| within the bar of the computation and the rounding to the type it is stored in"""
    off, half = np.abs(f64(got) - value), TYPES[dtype][1]
    assert np.isfinite(f64(got)).all(), f"{name}: not finite"
    limit = bar + half * (np.abs(value) + bar) + TINY[dtype]
    assert (off <= limit).all(), f"{name}: {np.max(off / limit):.3g} of its bar at {np.unravel_index(np.argmax(off / limit), off.shape)}"


def placed(t, layout):
    """the same rows elsewhere: `wide` with other columns between them, `shifted` from one element after an aligned address"""
    if t is None or layout == "plain":
        return None if t is None else t.cuda()
    n, d = t.shape
    more = 5 if layout == "wide" else 1
    room = torch.full((n * (d + more) + 1,), 7.0, dtype=t.dtype, device="cuda")
    v = room[1:].view(n, d + more)[:, :d]
    v.copy_(t)
    return v


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-v))
