"""Products with 4-bit weights that have one input to an output: every output is one product, so
float32 rows come back bit for bit through every form."""
import pytest

from gpu_common import say, torch
from serve_common import need_serve

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def selection(serve, N, K, at, by=1.0):
    """Weights of N outputs with `by` at input at[n]."""
    W = torch.zeros(N, K, dtype=BF16, device="cuda")
    W[torch.arange(N, device="cuda"), at] = by
    C, S = serve.w4_weight(N, K)
    serve.w4_pack(W, C, S)
    return C, S


def any_bits(rows, K, least, seed):
    """float32 values of any sign and mantissa, exponents from 2^least on."""
    g = torch.Generator("cuda").manual_seed(seed)
    bits = torch.randint(0, 2**23, (rows, K), generator=g, device="cuda", dtype=torch.int32)
    e = torch.randint(127 + least, 255, (rows, K), generator=g, device="cuda", dtype=torch.int32)
    sign = torch.randint(-1, 1, (rows, K), generator=g, device="cuda", dtype=torch.int32) << 31
    return (bits | e << 23 | sign).view(F32)


# rows of up to 16, 32, 64 and more with few outputs and many; two ways of the inputs and one
@pytest.mark.parametrize("rows", [1, 5, 16, 17, 20, 32, 33, 70, 300, 1500])
@pytest.mark.parametrize("N,K", [(16_416, 520), (1504, 1032), (40, 4360)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_come_back(rows, N, K, dtype):
    serve = need_serve()
    at = torch.randint(0, K, (N,), generator=torch.Generator().manual_seed(N)).cuda()
    at[:4] = torch.tensor([0, K - 1, K // 2, 127], device="cuda")
    C, S = selection(serve, N, K, at)
    x = any_bits(rows, K, -90, rows).to(dtype)
    x = torch.where(x.isfinite(), x, 1.0)                     # float32 values that round beyond bf16
    out = torch.empty(rows, N, dtype=dtype, device="cuda")
    assert torch.equal(serve.w4_linear(x, C, S, out), x[:, at])
    # inputs of only a little more than bf16's bits: a part that is left out shows
    if dtype == F32:
        x = 1.0 + torch.randint(1, 2**23, (rows, K), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 2.0**-23
        assert torch.equal(serve.w4_linear(x, C, S, out), x[:, at])
    # the gated form: a gate of 0 gives 0, one far above 0 itself
    half = torch.zeros(N // 2, dtype=torch.int64, device="cuda")
    C, S = selection(serve, N // 32 * 32, K, torch.cat([half[:N // 32 * 16], at[:N // 32 * 16]]))
    x = torch.where(x.abs() < 1e30, x, 1.0)
    x[:, 0] = 2.0**10
    out = torch.empty(rows, N // 32 * 16, dtype=dtype, device="cuda")
    assert torch.equal(serve.w4_linear(x, C, S, out, gated=True), x[:, at[:N // 32 * 16]] * 2.0**10)


@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("N", [64, 16_416])
def test_the_smallest_values(rows, N):
    """float32 rows are three parts of eight bits, the last one a multiple of bf16's least number: whole
    from 2^-110 on, below it cut off by less than 2^-133."""
    serve = need_serve()
    K = 128
    at = torch.arange(N, device="cuda") % K
    x = any_bits(rows, K, -126, 3)
    x = torch.ldexp(torch.frexp(x).mantissa, torch.randint(-125, -90, x.shape, generator=torch.Generator("cuda").manual_seed(5),
                                                           device="cuda"))
    low = (x.abs() < 2.0**-110)[:, at]
    assert low.any() and not low.all()
    for by in (1.0, 2.0**-10, 2.0**20):                       # 2^-10: sums below float32's normal numbers
        C, S = selection(serve, N, K, at, by)
        got = serve.w4_linear(x, C, S, torch.empty(rows, N, device="cuda")).double()
        off = (got - (x.double() * by)[:, at]).abs()
        exact = ~low & (by * x.abs()[:, at] >= 2.0**-126)
        say(f"{rows} rows, {N} outputs, times {by}: {float(off[low].max() / by):.3e} below 2^-110")
        assert not off[exact].any() and bool((off < 2.0**-133 * max(by, 2.0**-16) + 2.0**-149).all())


@pytest.mark.parametrize("byte", [0, 1, 2, 3, 127, 252])
def test_scales_that_a_program_lays_out(byte):
    """Every code under scales that packing does not write, 2^-127 and up, reads as what it stands for."""
    serve = need_serve()
    C, S = serve.w4_weight(16, 128)
    C[0, 0, 0] = torch.arange(16, dtype=torch.uint8, device="cuda")[:, None]        # the even inputs of output r: code r
    S.fill_(byte)
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
    want = torch.cat([e2m1, -e2m1]) * 2.0**(byte - 127)
    assert torch.equal(serve.w4_load(C, S, torch.empty(16, 128, device="cuda"))[:, 6].double().cpu(), want)
    for dtype in (F32, BF16):
        x = torch.zeros(2, 128, dtype=dtype, device="cuda")
        x[:, 2] = 1.0
        assert torch.equal(serve.w4_linear(x, C, S, torch.empty(2, 16, dtype=dtype, device="cuda"))[1].double().cpu(), want)
