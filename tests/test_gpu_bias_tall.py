"""The gradients for many queries by few keys, positions as indices: the work grows with the scores, not with the square of the queries.
A sum of n gradients of one sign and size 1 (whole numbers below 2^24, or sums of even ones) is exact in fp32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def buckets_of(queries, keys, offset, thresholds, both):
    d = torch.arange(keys, device="cuda")[None, :] - (torch.arange(queries, device="cuda") + offset)[:, None]
    a = d.abs() if both else (-d).clamp(min=0)
    n = torch.zeros_like(a)
    for t in thresholds:
        n += a >= t
    return n + (len(thresholds) + 1) * ((d > 0) & both), d


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("queries,keys,heads,dtype", [(1 << 18, 1, 2, torch.float32), (100_003, 8, 3, torch.bfloat16), (50_001, 9, 2, torch.float16),
                                                      (33_333, 64, 1, torch.float32), (1_000_001, 3, 1, torch.bfloat16), (5_000, 500, 2, torch.float16)])
def test_many_queries_by_few_keys(queries, keys, heads, dtype, causal):
    from paper_2305_01515_amd.dense import RelativeBias
    thresholds, offset = [1, 2, 3, 10, 100, 1000, 30_000, 200_000], -queries // 2
    plan = RelativeBias(heads, thresholds, bidirectional=True)
    g = torch.Generator(device="cuda").manual_seed(queries)
    dout = torch.randint(-3, 4, (1, heads, queries, keys), generator=g, device="cuda").to(dtype)
    n, d = buckets_of(queries, keys, offset, thresholds, True)
    seen = d <= 0 if causal else torch.ones_like(d, dtype=torch.bool)
    want = torch.stack([(torch.where((n == c) & seen, dout[0].double(), 0.0)).sum((1, 2)) for c in range(plan.buckets)])
    assert torch.equal(plan.backward(dout, q_offset=offset, causal=causal).double(), want)
    dtable, dscores = plan.backward(dout, q_offset=offset, causal=causal, want_dscores=True, scale=0.5)
    assert torch.equal(dtable.double(), want)
    assert torch.equal(dscores, torch.where(seen, dout * 0.5, 0.0).to(dtype))


@pytest.mark.parametrize("queries,keys", [(1 << 26, 1), ((1 << 27) - 5, 3)])
def test_a_hundred_million_queries(queries, keys):
    from paper_2305_01515_amd.dense import RelativeBias
    thresholds = [1, 1 << 10, 1 << 20, 1 << 25]
    plan = RelativeBias(1, thresholds)
    dout = torch.zeros(1, 1, queries, keys, dtype=torch.bfloat16, device="cuda")
    dout[:, :, ::64] = 2.0
    want = torch.zeros(5, dtype=torch.float64)
    for key in range(keys):
        # queries at multiples of 64, key at `key`: distances max(query - key, 0)
        q = torch.arange(0, queries, 64, device="cuda") - key
        want += 2.0 * torch.bincount(torch.bucketize(q.clamp(min=0), torch.tensor(thresholds, device="cuda"), right=True), minlength=5).double().cpu()
    assert torch.equal(plan.backward(dout)[:, 0].double().cpu(), want)
