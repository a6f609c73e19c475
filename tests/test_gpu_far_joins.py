"""Attention whose keys are dealt to waves or workgroups, at scores so far from zero that the parts
take their exponents in different ways: by one product that is rounded below 2^24, from
differences beyond.  The parts have to meet as if all had been exact.

Two keys count, with scores a few units apart that float32 holds exactly; the others' weights are 0.
Differences of scores are exact and a weight is off by its rounding alone, 2^-8 for bf16 inputs; exponents,
the scale in the log2 domain and the sums are 2^-16 together."""
import math

import pytest

from gpu_common import say, torch
from serve_common import bounds, need_serve

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NEAR, FAR = 11629079, 11629081            # times log2 e: 1.6 below 2^24, 1.3 above it
BELOW = -136 * 2.0**25                    # its product with log2 e is off by 160 in float32


def plant(K, at, score):
    """Key rows K [.., D] at the places `at` whose product with ``queries`` is `score`."""
    if score >= 0:
        K[..., at, 0], K[..., at, 1], K[..., at, 2] = score // 65536 * 2.0**8, score // 256 % 256 * 2.0**4, float(score % 256)
        K[..., at, 3] = 0.0
    else:
        K[..., at, :3], K[..., at, 3] = 0.0, score * 2.0**-10


def queries(*shape, dtype):
    q = torch.zeros(*shape, dtype=dtype, device="cuda")
    q[..., 0], q[..., 1], q[..., 2], q[..., 3] = 2.0**8, 2.0**4, 1.0, 2.0**10
    return q


# places of the first key, of the second ones, their scores, that of all others
CASES = {
    "near and far": ([10], [70], NEAR, FAR, 0),
    "far and near": ([10], [70], FAR, NEAR, 0),
    "far apart": ([10], [330], NEAR, FAR, 0),
    "far, one behind the other": ([70], [330], FAR, FAR + 2, 0),
    "near, after scores far below": ([5 * 64 + 10], [70], NEAR, NEAR - 2, BELOW),
    "near, behind scores far below": ([6 * 64 + 10], [64 * i for i in range(9, 18)], NEAR, NEAR - 2, BELOW),
}


def expected(case, n):
    """Weights [n, n] of the keys for each row, float64; NaN: rows that see neither of them."""
    a, b, sa, sb, _ = case
    w = torch.zeros(n, n, dtype=torch.float64)
    for at, s in ((a, sa), (b, sb)):
        for j in at:
            if j < n:
                w[j:, j] = math.exp(s - max(sa, sb))
    return w / w.sum(1, keepdim=True)


def keys(case, heads, n, D, dtype):
    a, b, sa, sb, rest = case
    K = torch.zeros(heads, n, D, dtype=dtype, device="cuda")
    plant(K, list(range(n)), rest)
    plant(K, a, sa)
    plant(K, [j for j in b if j < n], sb)
    V = torch.rand(heads, n, D, generator=torch.Generator().manual_seed(n)).mul_(2).sub_(1).to(dtype).cuda()
    return K, V


def held(out, case, V, first, G, dtype, what):
    """out [Hq, rows, D], the first row at position `first`."""
    n = V.shape[1]
    w = expected(case, n).cuda()[first:first + out.shape[1]]
    see = ~w.isnan().any(1)
    want = torch.stack([w @ v.double() for v in V]).repeat_interleave(G, 0)
    bar = 2.0**-16 + (2.0**-8 if dtype == BF16 else 0.0)
    worst = float((out.double() - want)[:, see].abs().max()) / bar
    say(f"{what}: off by {worst:.3f} of the bar")
    assert see.any() and worst <= 1.0


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("Hq,Hkv,D,n,dtype", [(12, 2, 128, 500, BF16), (32, 4, 64, 500, BF16), (12, 2, 128, 4096, BF16),
                                              (32, 4, 64, 1536, BF16), (32, 32, 64, 2000, BF16), (24, 24, 128, 3000, BF16),
                                              (4, 2, 64, 500, F32), (4, 2, 128, 500, F32)])
def test_prompts(case, Hq, Hkv, D, n, dtype):
    serve = need_serve()
    K, V = keys(CASES[case], Hkv, n, D, dtype)
    q = queries(Hq, n, D, dtype=dtype)
    out = torch.empty(Hq, n, D, dtype=F32, device="cuda")
    cu = bounds([n])
    serve.prompt_attn(q, K, V, cu, out, serve.prompt_desc(q, K, V, out, cu, scale=1.0))
    held(out, CASES[case], V, 0, Hq // Hkv, dtype, f"prompt {case} {Hq}/{Hkv} D={D} n={n} {dtype}")


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("Hq,Hkv,D,page,new", [(12, 2, 128, 64, 70), (16, 1, 64, 16, 70), (12, 2, 128, 16, 1), (4, 4, 64, 64, 700),
                                               (16, 1, 64, 64, 5)])
def test_pages(case, Hq, Hkv, D, page, new):
    serve = need_serve()
    n = 1280
    K, V = keys(CASES[case], Hkv, n, D, BF16)
    Kp, Vp = (x.unflatten(1, (n // page, page)).transpose(0, 1).contiguous() for x in (K, V))
    table = torch.arange(n // page, dtype=torch.int32, device="cuda")[None].contiguous()
    q = queries(Hq, new, D, dtype=BF16)
    out = torch.empty(Hq, new, D, dtype=F32, device="cuda")
    cu, start = bounds([new]), torch.tensor([n - new], device="cuda")
    desc = serve.page_attn_desc(q, Kp, table, cu, out, scale=1.0)
    ws = torch.empty(serve.page_attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    serve.page_attn(q, Kp, Vp, table, cu, out, ws, desc, start=start)
    held(out, CASES[case], V, n - new, Hq // Hkv, BF16, f"pages {case} {Hq}/{Hkv} D={D} {new} tokens")
