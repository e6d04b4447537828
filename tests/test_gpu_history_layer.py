"""The operators together, as a layer on histories uses them: norm with the residual, short convolution, selective scan, its result the next residual's summand."""
import numpy as np
import pytest
import torch

from rows_util import offsets

pytestmark = pytest.mark.gpu
DIM, STATES, WIDTH = 24, 16, 4


def weights(seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std=1.0: torch.randn(*s, generator=g) * std  # noqa: E731
    return {"norm": r(DIM, std=0.2) + 1, "conv": r(DIM, WIDTH, std=0.5), "conv_bias": r(DIM, std=0.1), "delta": r(DIM, DIM, std=0.2), "b": r(DIM, STATES, std=0.2),
            "c": r(DIM, STATES, std=0.2), "z": r(DIM, DIM, std=0.2), "a": -torch.rand(DIM, STATES, generator=g) * 4 - 0.1, "skip": r(DIM), "delta_bias": r(DIM, std=0.3) - 2}


def plain(w, x, r, lengths):
    """the layer in the tensors' own type, row by row, with torch's autograd"""
    s = x + r
    n = s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-6) * w["norm"]
    out, at = [], 0
    for size in lengths:
        e = torch.cat([torch.zeros(WIDTH - 1, DIM, dtype=x.dtype), n[at:at + size]])
        h = torch.zeros(DIM, STATES, dtype=x.dtype)
        for t in range(size):
            v = w["conv_bias"] + (e[t:t + WIDTH] * w["conv"].t()).sum(0)
            u = v * torch.sigmoid(v)
            step = torch.nn.functional.softplus(u @ w["delta"] + w["delta_bias"])
            h = torch.exp(step[:, None] * w["a"]) * h + (step * u)[:, None] * (u @ w["b"])[None]
            z = n[at + t] @ w["z"]
            out.append(((h * (u @ w["c"])[None]).sum(1) + w["skip"] * u) * z * torch.sigmoid(z))
        at += size
    return torch.stack(out), s


class Layer:
    def __init__(self, bags, rows):
        from paper_2305_01515_amd.dense import RMSNorm, SelectiveScan, ShortConv
        self.norm = RMSNorm(DIM, torch.float32, rows, residual_dtype=torch.float32)
        self.conv = ShortConv(DIM, WIDTH, torch.float32, bags, rows)
        self.scan = SelectiveScan(DIM, STATES, torch.float32, bags, rows)

    def __call__(self, w, x, r, off):
        n, s = self.norm(x, w["norm"], r)
        u, seen = self.conv(n, off, w["conv"], w["conv_bias"])
        y, h = self.scan(u, u @ w["delta"], w["a"], u @ w["b"], u @ w["c"], off, w["skip"], w["delta_bias"], n @ w["z"])
        return y, s, seen, h

    def step(self, w, x, r, seen, h):
        n, s, _ = self.norm.forward(x, w["norm"], r)
        u = self.conv.step(seen, n, w["conv"], w["conv_bias"])
        return self.scan.step(h, u, u @ w["delta"], w["a"], u @ w["b"], u @ w["c"], w["skip"], w["delta_bias"], n @ w["z"]), s


def test_training_pass():
    """results and gradients of a layer against the same in 64 bits.  Each operator is within some hundred 2^-24 of its magnitudes (their own tests); products and
    sums of up to 24 terms between them add as much, and gates pass errors on by their slopes, at most some tens: 2e-4 of the largest number."""
    lengths = [7, 0, 70, 1, 140, 3]
    g = torch.Generator().manual_seed(1)
    x, r, wy, ws = (torch.randn(sum(lengths), DIM, generator=g) for _ in range(4))
    w64 = {k: v.double().requires_grad_() for k, v in weights(2).items()}
    x64, r64 = x.double().requires_grad_(), r.double().requires_grad_()
    y, s = plain(w64, x64, r64, lengths)
    ((y * wy.double()).sum() + (s * ws.double()).sum()).backward()
    w = {k: v.cuda().requires_grad_() for k, v in weights(2).items()}
    xs, rs = x.cuda().requires_grad_(), r.cuda().requires_grad_()
    layer = Layer(len(lengths), sum(lengths))
    got, summed, _, _ = layer(w, xs, rs, offsets(lengths).cuda())
    ((got * wy.cuda()).sum() + (summed * ws.cuda()).sum()).backward()
    layer.conv.check()
    layer.scan.check()
    for name, a, b in [("y", got, y), ("x", xs.grad, x64.grad), ("r", rs.grad, r64.grad)] + [(k, w[k].grad, w64[k].grad) for k in w]:
        a, b = a.detach().double().cpu(), b.detach()
        assert (a - b).abs().max() <= 2e-4 * b.abs().max(), name


def test_prompt_then_single_rows():
    """a prompt of each length, then rows one by one: what one pass over the whole gives.  The same operations on the same numbers but for orders of sums: some
    hundred 2^-24 of the largest number, through gates as above"""
    lengths, more = [0, 1, 5, 70], 6
    g = torch.Generator().manual_seed(3)
    whole = [torch.randn(n + more, DIM, generator=g) for n in lengths]
    res = [torch.randn(n + more, DIM, generator=g) for n in lengths]
    w = {k: v.cuda() for k, v in weights(4).items()}
    layer = Layer(4, sum(lengths) + 4 * more)
    y, _, _, _ = layer(w, torch.cat(whole).cuda(), torch.cat(res).cuda(), offsets([n + more for n in lengths]).cuda())
    want = list(y.split([n + more for n in lengths]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # the same objects on another stream
        _, _, seen, h = layer(w, torch.cat([v[:n] for v, n in zip(whole, lengths)]).cuda(), torch.cat([v[:n] for v, n in zip(res, lengths)]).cuda(), offsets(lengths).cuda())
        for t in range(more):
            got, _ = layer.step(w, torch.stack([v[n + t] for v, n in zip(whole, lengths)]).cuda(), torch.stack([v[n + t] for v, n in zip(res, lengths)]).cuda(), seen, h)
            for k, n in enumerate(lengths):
                assert (got[k] - want[k][n + t]).abs().max() <= 2e-4 * y.abs().max()
    torch.cuda.current_stream().wait_stream(side)


def test_rows_far_apart():
    """rows of a store: places beyond 2^32 elements"""
    from paper_2305_01515_amd.dense import RMSNorm, SelectiveScan, ShortConv
    rows, apart, D, N = 20, 1 << 28, 40, 16
    if torch.cuda.mem_get_info()[0] < 3 * rows * apart * 2:
        pytest.skip("takes 11 GB")
    store = torch.empty(rows * apart, dtype=torch.bfloat16, device="cuda").view(rows, apart)
    g = torch.Generator().manual_seed(5)
    near = {k: torch.randn(rows, n, generator=g).bfloat16().cuda() for k, n in (("x", D), ("delta", D), ("z", D), ("dy", D), ("b", N), ("c", N), ("r", D))}
    far, at = {}, 0
    for k, v in near.items():
        far[k] = store[:, at:at + v.shape[1]]
        far[k].copy_(v)
        at += v.shape[1]
    y = store[:, at:at + D]
    off, w, a = offsets([12, 8]).cuda(), torch.randn(D, 4, generator=g).cuda(), -torch.rand(D, N, generator=g).cuda()
    conv, scan, norm = ShortConv(D, 4, torch.bfloat16, 2, rows), SelectiveScan(D, N, torch.bfloat16, 2, rows), RMSNorm(D, torch.bfloat16, rows, residual_dtype=torch.bfloat16)

    def all_of(t, y):
        out = [conv.forward(t["x"], off, w, y=y)[0].clone(), *conv.backward(t["x"], off, w, t["dy"])[:2]]
        args = [t["x"], t["delta"], a, t["b"], t["c"], off]
        _, last, saved = scan.forward(*args, z=t["z"], y=y, save=True)
        out += [y.clone(), last, *scan.backward(*args, saved, t["dy"], z=t["z"]).values()]
        o, s, rstd = norm.forward(t["x"], w[:, 0].contiguous(), t["r"], out=y)
        return out + [o.clone(), s, *norm.backward(t["dy"], s, rstd, w[:, 0].contiguous(), t["r"])]
    for v, u in zip(all_of(near, torch.empty_like(near["x"])), all_of(far, y)):
        assert torch.equal(v, u)
    conv.check()
    scan.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,states", [(70, 64), (130, 64), (65, 32), (129, 33)])
def test_rows_that_end_within_a_wavefront(dim, states, dtype):
    """the same elements as the first ones of a wider row (whose wavefronts are whole): the same bits"""
    from paper_2305_01515_amd.dense import SelectiveScan
    wide, lengths = 192, [1, 2, 3, 4, 5, 0, 77, 11]
    rows, bags = sum(lengths), len(lengths)
    g = torch.Generator().manual_seed(dim)
    t = {k: torch.randn(rows, wide, generator=g).to(dtype).cuda() for k in ("x", "delta", "z")}
    b, c = (torch.randn(rows, states, generator=g).to(dtype).cuda() for _ in range(2))
    a, h0, off = -torch.rand(wide, states, generator=g).cuda(), torch.randn(bags, wide, states, generator=g).cuda(), offsets(lengths).cuda()
    got = []
    for n in (wide, dim):
        p = SelectiveScan(n, states, dtype, bags, rows)
        y, last, _ = p.forward(t["x"][:, :n], t["delta"][:, :n], a[:n], b, c, off, z=t["z"][:, :n], h0=h0[:, :n].contiguous())
        got.append((y[:, :dim], last[:, :dim]))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
