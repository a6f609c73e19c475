"""4-bit weights on the GPU: the format exactly, products against float64 over the values the
codes stand for.

Bars: a product of a code, a power of two and a bf16 value (or one of the three bf16 parts of a
float32 value) is exact; a sum of K of them in float32 in any order is off by at most K u sum
|x w|, u = 2^-24 (3 K for the three parts, whose magnitudes add up to |x| (1 + 2^-7)), the bias
adds a rounding; the store rounds by half a step.  SwiGLU: its derivatives are at most 1.1 in
the gate and |silu(a)| <= |a| in the other half, exp and the division are a few u."""
import math

import numpy as np
import pytest

from gpu_common import say, torch
from oracle import serve as o_srv
from serve_common import need_serve, replay_checked

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0**-24


def randn(*shape, seed=0, dtype=BF16, by=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * by).to(dtype).cuda()


def padded(W):
    """Rows of whole blocks, zeros behind, float64 on the host."""
    W = W.double().cpu().numpy()
    return np.pad(W, ((0, 0), (0, -W.shape[1] % 32)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (40, 700), (5, 33), (32, 512), (3, 520)])
def test_pack_and_load(N, K, dtype):
    serve = need_serve()
    W = randn(N, K + 3, dtype=dtype, seed=N)[:, 1:K + 1].float() * 10.0 ** torch.randint(-3, 3, (N, 1), device="cuda")
    if K > 40:
        W[0, 3], W[N - 1, 35], W[0, 64:96] = math.nan, -math.inf, 0.0
    wide = torch.zeros(N, K + 5, dtype=dtype, device="cuda")
    wide[:, 1:K + 1] = W                                        # rows of odd stride
    C, S = serve.w4_weight(N, K)
    C.fill_(0xA5)
    serve.w4_pack(wide[:, 1:K + 1], C, S)
    codes, scales = o_srv.quantise(padded(wide[:, 1:K + 1]))
    wantC, wantS = o_srv.w4_tiles(codes[:, :K], scales)
    a, b = o_srv.unpack(C.cpu().numpy()), o_srv.unpack(wantC)
    assert bool(((a == b) | ((a & 7 == 0) & (b & 7 == 0))).all())
    tiles = -(-K // 128)
    got, want = (x.transpose(0, 1, 4, 2, 3).reshape(x.shape[0], -1, 4, 16)[:, :tiles] for x in (S.cpu().numpy(), wantS))
    assert np.array_equal(got, want)
    value = torch.tensor(o_srv.values(codes, scales))[:, :K]
    for back in (BF16, F32):
        out = torch.full((N, K + 11), 3.0, dtype=back, device="cuda")
        for view in (out[:, 1:K + 1], out[:, :K]):
            out.fill_(3.0)
            serve.w4_load(C, S, view)
            assert torch.equal(view.double().cpu().nan_to_num(nan=-1e9), value.nan_to_num(nan=-1e9))
            assert (out[:, K + 1:] == 3).all()


def weights(serve, N, K, seed=0):
    """Weights and the values they stand for."""
    C, S = serve.w4_weight(N, K)
    serve.w4_pack(randn(N, K, seed=seed, dtype=F32, by=0.05), C, S)
    return C, S, serve.w4_load(C, S, torch.empty(N, K, dtype=F32, device="cuda")).double().cpu()


def bar(x, W, bias, want, dtype):
    terms = x.abs() @ W.abs().t() + (0 if bias is None else bias.abs())
    return (3 * W.shape[1] * 1.01 if dtype == F32 else W.shape[1]) * U * terms + 4 * U * terms


def rounded(want, dtype):
    return want.abs() * (2.0**-8 if dtype == BF16 else U)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 130, 257])
@pytest.mark.parametrize("N,K", [(16, 128), (48, 1536), (50, 1000), (1, 1), (333, 97), (2048, 520)])
def test_linear(rows, N, K, dtype):
    serve = need_serve()
    C, S, W = weights(serve, N, K, seed=N)
    x = randn(rows, (K + 7) // 8 * 8 + 8, dtype=dtype, seed=rows)
    x[:, K:] = math.nan                                         # behind the row: not read as part of it
    x = x[:, :K]
    bias = randn(N, dtype=dtype, seed=3)
    for b in (None, bias):
        out = torch.full((rows, N + 3), 7.0, dtype=dtype, device="cuda")
        serve.w4_linear(x, C, S, out[:, :N], bias=b)
        xd, bd = x.double().cpu(), None if b is None else b.double().cpu()
        want = xd @ W.t() + (0 if b is None else bd)
        off = (out[:, :N].double().cpu() - want).abs() / (bar(xd, W, bd, want, dtype) + rounded(want, dtype))
        say(f"linear {rows} x {K} -> {N}: off by {float(off.max()):.3f} of the bar")
        assert off.max() <= 1.0 and (out[:, N:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 7, 32, 50, 100])
@pytest.mark.parametrize("N,K", [(32, 128), (1120, 1536), (96, 200)])
def test_gated(rows, N, K, dtype):
    serve = need_serve()
    C, S, W = weights(serve, N, K, seed=N + 1)
    x, bias = randn(rows, K, dtype=dtype, seed=rows, by=2.0), randn(N, dtype=dtype, seed=4)
    for b in (None, bias):
        out = torch.empty(rows, N // 2, dtype=dtype, device="cuda")
        serve.w4_linear(x, C, S, out, bias=b, gated=True)
        xd, bd = x.double().cpu(), None if b is None else b.double().cpu()
        y = xd @ W.t() + (0 if b is None else bd)
        off = bar(xd, W, bd, y, dtype)
        a, up = y.chunk(2, 1)
        da, du = off.chunk(2, 1)
        want = a * torch.sigmoid(a) * up
        # |silu'| <= 1.1; exp, 1 + exp and the quotient: (|a| + 6) u of the value
        lim = (1.1 * da) * (up.abs() + du) + a.abs() * du + want.abs() * (a.abs() + 8) * 2 * U + rounded(want, dtype)
        worst = float(((out.double().cpu() - want).abs() / lim).max())
        say(f"gated {rows} x {K} -> {N}: off by {worst:.3f} of the bar")
        assert worst <= 1.0


def test_gated_ends():
    """Gates far from 0 on both sides: silu is 0 and the gate itself."""
    serve = need_serve()
    W = torch.zeros(32, 32, device="cuda")
    W[:16, 0], W[16:, 1] = 1.0, 1.0
    C, S = serve.w4_weight(32, 32)
    serve.w4_pack(W, C, S)
    x = torch.zeros(3, 32, device="cuda")
    x[:, 0], x[:, 1] = torch.tensor([-1e4, 1e4, 0.0]), 2.0
    out = serve.w4_linear(x, C, S, torch.empty(3, 16, device="cuda"), gated=True)
    assert torch.equal(out, torch.tensor([[0.0], [2e4], [0.0]], device="cuda").expand(3, 16))


def test_float32_rows_are_taken_whole():
    """The product with an identity gives every float32 value back, bit for bit; infinities and
    NaN reach their row alone."""
    serve = need_serve()
    C, S = serve.w4_weight(64, 64)
    serve.w4_pack(torch.eye(64, device="cuda"), C, S)
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-2**31, 2**31 - 1, (40, 64), generator=g, dtype=torch.int32).view(F32)
    e = torch.frexp(x).exponent                                 # all three parts of it are normal numbers
    x = torch.where(x.isfinite() & (e > -90), x, torch.tensor(1.0 + 2.0**-23)).cuda()
    x[0, 0], x[0, 1] = 3.4028234e38, 1.17549435e-38 * 2**40
    got = serve.w4_linear(x, C, S, torch.empty(40, 64, device="cuda"))
    assert torch.equal(got, x)
    x = torch.ones(3, 64, device="cuda")
    x[1, 5], x[2, 6] = math.inf, math.nan
    C, S, W = weights(serve, 16, 64)
    for dtype in (F32, BF16):
        y = serve.w4_linear(x.to(dtype), C, S, torch.empty(3, 16, dtype=dtype, device="cuda")).cpu()
        want = torch.where(W[:, 5] == 0, math.nan, W[:, 5].sign() * math.inf)
        assert y[0].isfinite().all() and y[2].isnan().all()
        assert torch.equal(y[1].double().nan_to_num(nan=-1e9, posinf=1e30, neginf=-1e30),
                           want.nan_to_num(nan=-1e9, posinf=1e30, neginf=-1e30))


def test_nan_blocks():
    serve = need_serve()
    W = randn(20, 256, dtype=F32)
    W[3, 70] = math.inf
    C, S = serve.w4_weight(20, 256)
    serve.w4_pack(W, C, S)
    y = serve.w4_linear(randn(4, 256), C, S, torch.empty(4, 20, dtype=BF16, device="cuda"))
    assert y[:, 3].isnan().all() and y[:, :3].isfinite().all() and y[:, 4:].isfinite().all()


def test_rows_do_not_meet():
    """A row's result does not depend on the rows beside it, nor on the rows that are not there."""
    serve = need_serve()
    C, S, _ = weights(serve, 100, 300)
    x = randn(64, 304)[:, :300]
    for rows in (16, 64):
        whole = serve.w4_linear(x[:rows], C, S, torch.empty(rows, 100, dtype=BF16, device="cuda"))
        y = x[:rows].clone()
        wide = torch.empty(rows, 304, dtype=BF16, device="cuda")
        wide[:, :300] = y
        wide[1::2] = math.nan
        part = serve.w4_linear(wide[:, :300], C, S, torch.empty(rows, 100, dtype=BF16, device="cuda"))
        assert torch.equal(part[::2], whole[::2])


def test_captured_and_replayed():
    serve = need_serve()
    C, S, _ = weights(serve, 640, 1536)
    x, out = randn(5, 1536), torch.zeros(5, 320, dtype=BF16, device="cuda")
    replay_checked(lambda: serve.w4_linear(x, C, S, out, gated=True), [out], lambda i: x.copy_(randn(5, 1536, seed=i + 9)))


def test_many_outputs():
    """Codes whose offsets pass 32 bits: 2.2 million outputs of 4,096 inputs."""
    serve = need_serve()
    N, K = 2_200_000, 4096
    C, S = serve.w4_weight(N, K)
    part = randn(64, K, dtype=F32, by=0.05)
    c, s = serve.w4_weight(64, K)
    serve.w4_pack(part, c, s)
    C[-4:], S[-4:] = c, s
    x = randn(2, K)
    got = serve.w4_linear(x, C, S, torch.empty(2, N, dtype=BF16, device="cuda"))
    want = serve.w4_linear(x, c, s, torch.empty(2, 64, dtype=BF16, device="cuda"))
    assert torch.equal(got[:, -64:], want) and not got[:, :-64].any()


def test_many_rows():
    """Rows beyond what a form of few rows can launch."""
    serve = need_serve()
    C, S, W = weights(serve, 48, 64)
    x = randn(300_000, 64)
    out = serve.w4_linear(x, C, S, torch.empty(300_000, 48, dtype=BF16, device="cuda"))
    few = serve.w4_linear(x[-64:], C, S, torch.empty(64, 48, dtype=BF16, device="cuda"))
    want = x.double() @ W.t().cuda()
    assert bool(((out.double() - want).abs() <= bar(x.double(), W.cuda(), None, want, BF16) + rounded(want, BF16)).all())
    assert bool(((out[-64:].double() - few.double()).abs() <= 2 * rounded(want[-64:], BF16)).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,N,K", [(3, 1504, 5000), (70, 1504, 5000), (130, 1504, 5000), (300, 1504, 5000),
                                      (400, 1504, 1032), (600, 1504, 520), (1500, 1504, 520),
                                      (1, 16_416, 200), (20, 16_416, 200), (50, 16_416, 200), (2, 16_480, 1032)])
def test_every_form(rows, N, K, dtype):
    """40 tiles of inputs, the last one not whole, for every number of waves that deal them; outputs
    enough for the form that shares rows, their last tiles no whole workgroup's."""
    serve = need_serve()
    C, S, W = weights(serve, N, K, seed=9)
    x = randn(rows, K, dtype=dtype, seed=rows)
    want = x.double().cpu() @ W.t()
    lim = bar(x.double().cpu(), W, None, want, dtype)
    out = serve.w4_linear(x, C, S, torch.empty(rows, N, dtype=dtype, device="cuda"))
    assert bool(((out.double().cpu() - want).abs() <= lim + rounded(want, dtype)).all())
    out = serve.w4_linear(x, C, S, torch.empty(rows, N // 2, dtype=dtype, device="cuda"), gated=True)
    a, up = want.chunk(2, 1)
    da, du = lim.chunk(2, 1)
    want = a * torch.sigmoid(a) * up
    lim = (1.1 * da) * (up.abs() + du) + a.abs() * du + want.abs() * (a.abs() + 8) * 2 * U + rounded(want, dtype)
    assert bool(((out.double().cpu() - want).abs() <= lim).all())
