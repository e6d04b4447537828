"""The norm with the residual's addition against its formula in 64 bits.

Bars.  eps = 2^-24.  The sum of x and the residual is rounded to fp32 and then to its type, the stored number: two roundings of it differ from one only between two
neighbours, so the formula goes from the stored sum, which is itself compared with an error of half a step and eps.  A lane adds 32 squares at most, the lanes
of a row 10 times two: 50 eps of the mean, 25 of its root, 5 for the quotient and the products: 32 eps of a result.  mean(d s rstd) adds 50 eps of
its magnitudes, the backward 40 eps of each of its terms.  Sums over n rows add (n + 100) eps of their magnitudes.  Codes are nearest numbers of 3 mantissa bits: half a step, 2^-4
of the number, or 2^-10 scales below 2^-6."""
import numpy as np
import pytest
import torch

from rows_util import EPS, TYPES, f64, near, placed

pytestmark = pytest.mark.gpu


def inputs(rows, dim, dtype, residual, weights, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype][0]
    t = {"x": (torch.randn(rows, dim, generator=g) * scale).to(dt), "dout": torch.randn(rows, dim, generator=g).to(dt),
         "weight": (torch.randn(dim, generator=g) + 0.5).to(TYPES[weights][0]), "residual": None, "dsummed": None}
    if residual:
        t |= {k: (torch.randn(rows, dim, generator=g) * scale).to(TYPES[residual][0]) for k in ("residual", "dsummed")}
    return t


def stored_sum(t, summed, residual):
    """the stored sum as the formula's input, after a look at it"""
    if not residual:
        assert summed is not None
        return f64(summed)
    near("summed", summed, f64(t["x"]) + f64(t["residual"]), EPS * (np.abs(f64(t["x"])) + np.abs(f64(t["residual"]))), residual)
    return f64(summed)


def run_and_compare(rows, dim, dtype, residual, weights, layout="plain", seed=0, eps=1e-6, scale=1.0):
    from paper_2305_01515_amd.dense import RMSNorm
    t = inputs(rows, dim, dtype, residual, weights, seed, scale)
    gpu = {k: placed(v, layout) if k != "weight" else v.cuda() for k, v in t.items()}
    plan = RMSNorm(dim, TYPES[dtype][0], rows, eps, TYPES[residual][0] if residual else None)
    out, summed, rstd = plan.forward(gpu["x"], gpu["weight"], gpu["residual"])
    s, w, d = stored_sum(t, summed, residual), f64(t["weight"]), f64(t["dout"])
    r = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    near("out", out, s * r * w, 32 * EPS * np.abs(s * r * w), dtype)
    near("rstd", rstd, r[:, 0], 28 * EPS * r[:, 0])
    dx, dresidual, dweight = plan.backward(gpu["dout"], summed, rstd, gpu["weight"], gpu["dsummed"])
    u, extra = s * r, 0 if not residual else f64(t["dsummed"])
    dot, size = (d * w * u).mean(1, keepdims=True), np.abs(d * w * u).mean(1, keepdims=True)
    value = r * (d * w - u * dot) + extra
    bar = r * (40 * EPS * np.abs(d * w) + np.abs(u) * (100 * EPS * size + 40 * EPS * np.abs(dot))) + 4 * EPS * np.abs(value) + EPS * np.abs(extra)
    near("dx", dx, value, bar, dtype)
    if residual:
        near("dresidual", dresidual, value, bar, residual)
        assert dresidual is dx or residual != dtype
    else:
        assert dresidual is None
    near("dweight", dweight, (d * u).sum(0), (rows + 100 + 40) * EPS * np.abs(d * u).sum(0))
    return plan, gpu, (out, summed, rstd, dx, dresidual, dweight)


KINDS = [("f32", None, "f32"), ("f32", "f32", "bf16"), ("f16", None, "f16"), ("f16", "f16", "f32"), ("f16", "f32", "f32"), ("bf16", None, "f32"), ("bf16", "bf16", "bf16"),
         ("bf16", "f32", "f32")]


@pytest.mark.parametrize("dtype,residual,weights", KINDS)
@pytest.mark.parametrize("rows,dim,layout", [(70, 64, "plain"), (1, 128, "plain"), (33, 1, "plain"), (19, 7, "wide"), (300, 100, "shifted"), (9, 513, "plain"), (40, 1001, "shifted"),
                                             (5, 4096, "wide"), (3, 8193, "plain"), (2, 20001, "shifted"), (2, 32768, "plain"), (2000, 24, "plain")])
def test_sizes(rows, dim, layout, dtype, residual, weights):
    run_and_compare(rows, dim, dtype, residual, weights, layout, seed=dim)


@pytest.mark.parametrize("dtype,residual,weights", [KINDS[1], KINDS[2], KINDS[7]])
@pytest.mark.parametrize("rows,dim", [(12000, 130), (9000, 200), (2500, 1001), (2500, 3000), (2300, 8000), (2100, 8200)])
def test_more_rows_than_workgroups_of_the_backward(rows, dim, dtype, residual, weights):
    """each has a second group of rows, whose part of the weights' gradient is added to the first one's, in registers or (8200 elements) in memory; without it the
    gradient of a weight would be off by the root of the rows left out, several times the bar"""
    run_and_compare(rows, dim, dtype, residual, weights, seed=rows)


def test_no_rows():
    from paper_2305_01515_amd.dense import RMSNorm
    plan, w = RMSNorm(64, torch.bfloat16, 8, residual_dtype=torch.float32), torch.ones(64, device="cuda")
    x, r = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 64, device="cuda")
    out, summed, rstd = plan.forward(x, w, r)
    dx, dr, dw = plan.backward(x, summed, rstd, w, r)
    assert out.shape == summed.shape == dx.shape == dr.shape == (0, 64) and rstd.shape == (0,) and (dw == 0).all()
    codes, scales, _ = plan.quantise(x, w, r)
    assert codes.shape == (0, 64) and scales.shape == (0, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_and_small_rows(dtype):
    run_and_compare(20, 200, dtype, None, "f32", scale=1e12, seed=1)
    run_and_compare(20, 200, dtype, None, "f32", scale=1e-12, eps=1e-26, seed=2)
    run_and_compare(20, 200, dtype, None, "f32", scale=1e-12, seed=3)


def test_rows_of_zeros_infinities_and_nan_stay_their_own():
    from paper_2305_01515_amd.dense import RMSNorm
    t = {k: v.cuda() for k, v in inputs(64, 100, "f32", None, "f32", 5).items() if v is not None}
    plan = RMSNorm(100, torch.float32, 64)
    clean, *_ = plan.forward(t["x"], t["weight"])
    t["x"][3], t["x"][10, 5], t["x"][11, 7] = 0, float("inf"), float("nan")
    out, _, _ = plan.forward(t["x"], t["weight"])
    rest = [i for i in range(64) if i not in (3, 10, 11)]
    assert torch.equal(out[rest], clean[rest]) and (out[3] == 0).all() and torch.isnan(out[10, 5]) and torch.isnan(out[11]).all()
    codes, scales, _ = plan.quantise(t["x"], t["weight"], group=16)
    back = codes.float() * scales.repeat_interleave(16, 1)[:, :100]
    assert (back[3] == 0).all() and (scales[3] == 0).all() and torch.isnan(back[11]).all() and torch.isnan(back[10, :16]).all() and torch.isfinite(back[rest]).all()
    codes, scales, _ = plan.quantise(t["x"], t["weight"])
    assert torch.isnan(codes[10].float() * scales[10]).all() and torch.isnan(codes[11].float() * scales[11]).all()


@pytest.mark.parametrize("dtype,residual,weights", KINDS)
@pytest.mark.parametrize("rows,dim,group,layout", [(70, 64, 0, "plain"), (9, 128, 32, "wide"), (19, 7, 16, "shifted"), (33, 1, 0, "plain"), (40, 1001, 128, "shifted"), (40, 1001, 0, "plain"),
                                                   (5, 4100, 256, "plain"), (3, 20001, 16, "plain"), (3, 20001, 0, "wide"), (6, 300, 64, "plain")])
def test_results_in_8_bits(rows, dim, group, layout, dtype, residual, weights):
    from paper_2305_01515_amd.dense import RMSNorm
    t = inputs(rows, dim, dtype, residual, weights, dim)
    gpu = {k: placed(v, layout) if k != "weight" else v.cuda() for k, v in t.items()}
    plan = RMSNorm(dim, TYPES[dtype][0], rows, 1e-6, TYPES[residual][0] if residual else None)
    codes, scales, summed = plan.quantise(gpu["x"], gpu["weight"], gpu["residual"], group=group)
    s, n = stored_sum(t, summed, residual), group or dim
    v = s / np.sqrt((s * s).mean(1, keepdims=True) + 1e-6) * f64(t["weight"])
    parts = -(-dim // n)
    assert scales.shape == (rows, parts) and codes.dtype == torch.float8_e4m3fn
    top = np.stack([np.abs(v[:, i * n:(i + 1) * n]).max(1) for i in range(parts)], 1)
    near("scales", scales, top / 448, 34 * EPS * top / 448)
    scale = np.repeat(f64(scales), n, 1)[:, :dim]
    off = np.abs(f64(codes.float()) * scale - v)
    # half a step of the code, and 40 eps of what was rounded
    assert (off <= (2.0 ** -4 + 40 * EPS) * np.abs(v) + 2.0 ** -10 * scale).all()
    at = np.abs(v) >= 2.0 ** -6 * scale * 1.01  # nearest: a code's neighbours are no nearer, but for 40 eps
    q = np.abs(v) / np.where(scale > 0, scale, 1)
    step = np.exp2(np.floor(np.log2(np.maximum(q, 2.0 ** -6))) - 3)
    assert (off <= (step / 2 * scale + 80 * EPS * np.abs(v)))[at].all()


def test_small_results_in_8_bits():
    """a weight that makes everything tiny: scales down to the smallest number, codes as of any other row"""
    from paper_2305_01515_amd.dense import RMSNorm
    x, plan = torch.randn(4, 64, generator=torch.Generator().manual_seed(1)).cuda(), RMSNorm(64, torch.float32, 4)
    plain, _, _ = plan.quantise(x, torch.ones(64, device="cuda"))
    for p in (-60, -110):  # powers of two: everything scales exactly while it is a normal number
        codes, scales, _ = plan.quantise(x, torch.full((64,), 2.0 ** p, device="cuda"))
        assert torch.equal(codes.view(torch.uint8), plain.view(torch.uint8)) and (scales > 0).all()
    codes, scales, _ = plan.quantise(x, torch.zeros(64, device="cuda"))
    assert (codes.float() == 0).all() and (scales == 0).all()


@pytest.mark.parametrize("dtype,dim,group,power", [(*case, power) for case in (("bf16", 4096, 0), ("bf16", 1000, 32)) for power in (0, -110, 110)] +
                         [("f16", 4096, 0, 0), ("f16", 256, 64, 0)])
def test_codes_half_way_are_even(dtype, dim, group, power):
    """Rows and weights of 16 bits: their products s w, and 448 s w over the largest one, are exact in 64 bits or far enough from half way between two codes (22 bits by 22, so
    2^-27 of it) that rounding to 53 bits says which side: every code is the nearest, the even one of two.  Weights times 2^power: results near both ends of fp32 (bfloat16)."""
    from paper_2305_01515_amd.dense import RMSNorm
    t = inputs(500, dim, dtype, None, dtype, dim + group)
    t["weight"] = t["weight"] * 2.0 ** power
    plan = RMSNorm(dim, TYPES[dtype][0], 500)
    codes, scales, _ = plan.quantise(t["x"].cuda(), t["weight"].cuda(), group=group)
    v = np.zeros((500, -(-dim // (group or dim)) * (group or dim)))
    v[:, :dim] = f64(t["x"]) * f64(t["weight"])
    v = v.reshape(500, -1, group or dim)
    q = 448 * v / np.abs(v).max(2, keepdims=True)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(q), 1e-30))), -6) - 3)
    assert (np.rint(q / step) != np.floor(q / step + 0.5)).any() or dtype == "f16"  # some do lie half way, below an even code
    want = (np.rint(q / step) * step).reshape(500, -1)[:, :dim]
    assert np.array_equal(f64(codes.float()), want)


def test_squares_beyond_32_bits():
    """sums of squares up to 2^128 are found; a row beyond that is zeros, and so are its gradients, apart from what comes to the stored sum"""
    from paper_2305_01515_amd.dense import RMSNorm
    plan, w = RMSNorm(64, torch.float32, 3, residual_dtype=torch.float32), torch.full((64,), 2.0, device="cuda")
    x = torch.tensor([2.0 ** 60, 2.0 ** 61, 1.0]).view(3, 1).expand(3, 64).contiguous().cuda()  # 64 squares: 2^126, 2^128, 64
    zero = torch.zeros_like(x)
    out, summed, rstd = plan.forward(x, w, zero)
    assert torch.equal(summed, x) and (out[[0, 2]] - 2).abs().max() <= 1e-6 and not out[1].any() and rstd[1] == 0
    codes, scales, _ = plan.quantise(x, w, zero)
    assert not codes[1].float().any() and scales[1] == 0 and (codes[[0, 2]].float() * scales[[0, 2]] - 2).abs().max() <= 1e-6
    dx, _, dw = plan.backward(zero + 3, summed, rstd, w, zero + 5)
    assert (dx[1] == 5).all() and torch.isfinite(dx).all() and torch.isfinite(dw).all()


def test_sum_in_place_of_its_inputs():
    from paper_2305_01515_amd.dense import RMSNorm
    for dtype, residual in (("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")):
        t = {k: v.cuda() for k, v in inputs(50, 1001, dtype, residual, "f32", 1).items()}
        plan = RMSNorm(1001, TYPES[dtype][0], 50, residual_dtype=TYPES[residual][0])
        out, summed, rstd = plan.forward(t["x"], t["weight"], t["residual"])
        r, x = t["residual"].clone(), t["x"].clone()
        out2, s2, _ = plan.forward(t["x"], t["weight"], r, summed=r)
        assert s2 is r and torch.equal(r, summed) and torch.equal(out, out2)
        if dtype == residual:
            out3, _, _ = plan.forward(x, t["weight"], t["residual"], summed=x)
            assert torch.equal(x, summed) and torch.equal(out, out3)


def test_the_same_bits_again_and_in_graphs():
    plan, gpu, want = run_and_compare(700, 1000, "bf16", "f32", "f32", seed=3)

    def both():
        out, summed, rstd = plan.forward(gpu["x"], gpu["weight"], gpu["residual"])
        return [out, summed, rstd, *plan.backward(gpu["dout"], summed, rstd, gpu["weight"], gpu["dsummed"])]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(4):
        for v in got:
            v.zero_()
        graph.replay()
        for v, w in zip(got, want):
            assert torch.equal(v, w)
        plan.forward(gpu["x"][:7], gpu["weight"], gpu["residual"][:7])
        torch.cuda.synchronize()


@pytest.mark.parametrize("residual", [None, "f32"])
def test_gradients_through_autograd(residual):
    from paper_2305_01515_amd.dense import RMSNorm
    t = inputs(9, 12, "f32", residual, "f32", 2)
    names = ("x", "weight", "residual") if residual else ("x", "weight")

    def loss(v):
        s = v["x"] + v["residual"] if residual else v["x"]
        out = s / np.sqrt((s * s).mean(1, keepdims=True) + 1e-6) * v["weight"]
        return (out * f64(t["dout"])).sum() + ((s * f64(t["dsummed"])).sum() if residual else 0)
    leaves = {k: t[k].cuda().requires_grad_() for k in names}
    plan = RMSNorm(12, torch.float32, 9, residual_dtype=TYPES[residual][0] if residual else None)
    got = plan(*leaves.values())
    if residual:
        out, summed = got
        ((out * t["dout"].cuda()).sum() + (summed * t["dsummed"].cuda()).sum()).backward()
    else:
        (got * t["dout"].cuda()).sum().backward()
    rs = np.random.RandomState(0)
    for k in names:
        way, v, step = rs.standard_normal(t[k].shape), {n: f64(t[n]) for n in names}, 1e-6
        slope = (loss(dict(v, **{k: v[k] + step * way})) - loss(dict(v, **{k: v[k] - step * way}))) / (2 * step)
        # differences: step^2 of the third derivative, and 2^-53 of the loss over the step; gradients: some hundred eps of their magnitudes
        assert abs(slope - (f64(leaves[k].grad) * way).sum()) <= 1e-5 * (np.abs(f64(leaves[k].grad) * way).sum() + 1), k
    if residual:  # the sum alone, and the result alone
        for pick in (0, 1):
            g = torch.autograd.grad(plan(*leaves.values())[pick].sum(), [leaves["x"], leaves["residual"]])
            assert torch.equal(g[0], g[1]) and (pick == 0 or (g[0] == 1).all())
    with pytest.raises(RuntimeError, match="once_differentiable"):
        out = plan(leaves["x"], leaves["weight"])
        g, = torch.autograd.grad((out ** 2).sum(), leaves["x"], create_graph=True)
        (g ** 2).sum().backward()


def test_what_is_refused():
    from paper_2305_01515_amd.dense import RMSNorm
    from paper_2305_01515_amd.tbe import TbeError
    for bad in (dict(dim=0), dict(dim=32769), dict(max_rows=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(TbeError):
            RMSNorm(**{**dict(dim=64, dtype=torch.float32, max_rows=9), **bad})
    for kinds in ((torch.float64, None), (torch.float32, torch.bfloat16), (torch.float16, torch.bfloat16)):
        with pytest.raises(ValueError):
            RMSNorm(8, kinds[0], 9, residual_dtype=kinds[1])
    t = {k: v.cuda() for k, v in inputs(9, 16, "bf16", "f32", "f32", 1).items()}
    plan, bare = RMSNorm(16, torch.bfloat16, 9, residual_dtype=torch.float32), RMSNorm(16, torch.bfloat16, 9)
    for call in (lambda: bare.forward(t["x"], t["weight"], t["residual"]), lambda: plan.forward(t["x"].half(), t["weight"]), lambda: plan.forward(t["x"], t["weight"][:8]),
                 lambda: plan.forward(t["x"], t["weight"], t["residual"].bfloat16()), lambda: plan.forward(t["x"], t["weight"].double()),
                 lambda: plan.forward(t["x"], t["weight"], summed=t["residual"]), lambda: bare.backward(t["dout"], t["x"], t["residual"][:, 0].contiguous(), t["weight"], t["residual"])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: plan.forward(t["x"], t["weight"], out=t["x"]), lambda: plan.quantise(t["x"], t["weight"], group=24), lambda: plan.quantise(t["x"], t["weight"], group=8),
                 lambda: plan.quantise(t["x"], t["weight"], group=512), lambda: plan.quantise(t["x"], t["weight"], group=-16),
                 lambda: plan.forward(torch.cat([t["x"]] * 2), t["weight"])):
        with pytest.raises(TbeError):
            call()
