"""The decode step over the 4-bit cache at scales up to the largest: scores far below
and above what exponents of float32 numbers hold."""
import numpy as np
import pytest

from gpu_common import say, torch
from serve_common import U, bounds, need_serve
from test_gpu_kv4 import filled, step

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("scale", [0.0, 1e10, 1e31, 2.0**126, 1e38])
@pytest.mark.parametrize("D", [64, 128])
def test_one_key_is_its_values(D, scale):
    """A softmax over one key has weight 1 whatever the score."""
    serve = need_serve()
    B, Hq, Hkv, L = 3, 6, 2, 50
    cache, K, V = filled(serve, B, Hkv, L, D, seed=9)
    Q = (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(1)) * 3).to(BF16).cuda()
    pos = torch.tensor([0, 31, 49], device="cuda")
    got = step(serve, Q, cache, pos, window=1, scale=scale).double().cpu().numpy()
    for b in range(B):
        assert np.array_equal(got[b], V[b][:, int(pos[b])].repeat(Hq // Hkv, 0))


@pytest.mark.parametrize("scale,power", [(1e10, 0), (1e31, 0), (2.0**126, 0), (1e38, 0), (1.0, 40), (0.0, 110)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,L", [(2, 100), (1, 5000), (70, 3000)])
def test_far_scores(B, L, D, scale, power):
    """Small integers in Q (times a power of two) and K: scores are exact, and those below a
    row's largest have no weight: the mean of the best keys' values, off by (n + 64) u
    max|V|.  Every second sequence has scores below 0 alone."""
    serve = need_serve()
    say(f"kv4 far scores B={B} L={L} D={D} scale={scale} 2^{power}")
    Hq, Hkv = 6, 2
    g = torch.Generator().manual_seed(D + L)
    k = torch.randint(-1, 2, (B, Hkv, L, D), generator=g).float()
    q = torch.randint(-1, 2, (B, Hq, D), generator=g).float()
    k[1::2, ..., 0], q[1::2, :, 0] = 1.0, -2.0 * D
    if B == 1:
        k[..., 0], q[..., 0] = 1.0, -2.0 * D
    v = torch.randn(B, Hkv, L, D, generator=g)
    rows = [x.transpose(0, 1).reshape(Hkv, B * L, D).to(BF16).cuda() for x in (k, v)]
    cache, back = serve.kv4_cache(B, Hkv, L, D), [torch.empty_like(x) for x in rows]
    serve.kv4_store(*rows, bounds([L] * B), *cache)
    serve.kv4_load(*cache, bounds([L] * B), *back)
    assert torch.equal(back[0], rows[0])                           # K is held exactly
    Q = (q * 2.0**power).to(BF16).cuda()
    pos = torch.full((B,), L - 1, device="cuda")
    got = step(serve, Q, cache, pos, window=L, scale=scale).double()
    kk, vv = (x.double().view(Hkv, B, L, D).transpose(0, 1).repeat_interleave(Hq // Hkv, 1) for x in back)
    s = (kk * Q.double()[:, :, None]).sum(-1)
    top = (s == s.amax(-1, keepdim=True)).double()
    want = ((top / top.sum(-1, keepdim=True))[..., None] * vv).sum(2)
    assert (got - want).abs().max().item() <= (L + 64) * U * vv.abs().max().item()
