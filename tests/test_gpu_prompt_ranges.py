"""Packed prompt attention at the ends of what its arguments may hold: scores and
scales whose products leave float32, infinities and NaN of V under any weight, and
float32 weights below 2^-126.  Every form that the batch's shape chooses is reached.
"""
import numpy as np
import pytest

from gpu_common import say, torch
from serve_common import U, attn_bar, bounds, need_serve

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# form: dtype, Hq, Hkv, lengths of the prompts
FORMS = {
    "narrow": (BF16, 4, 2, [300]),
    "split": (BF16, 12, 2, [2048]),
    "wide": (BF16, 12, 2, [3000, 1200, 1500]),
    "short": (BF16, 12, 2, [5, 40, 64, 7, 1, 100] * 35),
    "f32": (F32, 4, 2, [300, 77]),
}


def run(serve, q, k, v, cu, scale=0.0, causal=1):
    out = torch.full(q.shape, 9.0, dtype=F32, device="cuda")
    return serve.prompt_attn(q, k, v, cu, out, serve.prompt_desc(q, k, v, out, cu, causal=causal, scale=scale))


def expect(q, k, v, lens, weigh, causal=1):
    """float64: ``weigh`` makes the weights [n, n] of the masked scores of a prompt and head."""
    G, at, out = q.shape[0] // k.shape[0], 0, []
    for n in lens:
        late = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        heads = []
        for h in range(q.shape[0]):
            s = q[h, at:at + n].double() @ k[h // G, at:at + n].double().t().contiguous()
            if causal:
                s.masked_fill_(late, -np.inf)
            heads.append(weigh(s) @ v[h // G, at:at + n].double())
        out.append(torch.stack(heads))
        at += n
    return torch.cat(out, 1)


def best(s):
    """Equal weights on the largest scores."""
    top = (s == s.amax(1, keepdim=True)).double()
    return top / top.sum(1, keepdim=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("scale,power", [(2.0**126, 0), (1e38, 0), (1e12, 0), (1.0, 40), (0.0, 60), (1.0, 118), (2.0**-20, 100)])
def test_far_scores(form, D, scale, power):
    """Q and K of small integers (times a power of two): scores are exact, and those below
    a row's largest have no weight.  Outputs are then sums of at most n values V with
    weights of 1, off by (n + 64) u max|V|."""
    serve = need_serve()
    dtype, Hq, Hkv, lens = FORMS[form]
    say(f"prompt {form} D={D} scale={scale} 2^{power}")
    g = torch.Generator().manual_seed(D + power)
    T = sum(lens)
    q = (torch.randint(-1, 2, (Hq, T, D), generator=g) * 2.0**power).to(dtype).cuda()
    k = torch.randint(-1, 2, (Hkv, T, D), generator=g).to(dtype).cuda()
    v = torch.randn(Hkv, T, D, generator=g).to(dtype).cuda()
    for causal in (1, 0) if form in ("narrow", "short", "f32") else (1,):
        got = run(serve, q, k, v, bounds(lens), scale, causal)
        want = expect(q, k, v, lens, best, causal)
        assert (got.double() - want).abs().max().item() <= (max(lens) + 64) * U * v.double().abs().max().item()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_far_rows_leave_the_others_as_they_are(form, D):
    """Queries of every fifth token far from 0: the other rows stay within their bars (the
    rows of a wave move their references together, so not to the bit).  Keys that are far
    until a nearer one has come: its weight is all there is, so the output is its value,
    off by 8 u: the product 3 log2 e is rounded in the reference (3 u in the weight, of which
    bf16 products see a rounded one), the exponential, the quotient."""
    serve = need_serve()
    dtype, Hq, Hkv, lens = FORMS[form]
    g = torch.Generator().manual_seed(D)
    T = sum(lens)
    q, k, v = (torch.randn(h, T, D, generator=g) for h in (Hq, Hkv, Hkv))
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    far = q.clone()
    far[:, ::5] *= 2.0**30
    got = run(serve, far, k, v, bounds(lens))
    assert got.isfinite().all()
    want = expect(q, k, v, lens, lambda s: (s * D**-0.5).softmax(1))
    bar = attn_bar(q, k, v, max(lens), D**-0.5, want, dtype, F32)
    near = torch.arange(T, device="cuda") % 5 > 0
    assert ((got.double() - want).abs() <= bar)[:, near].all()
    # all scores -2^40 but the last of each prompt's
    q = torch.zeros_like(q)
    q[..., 0] = 1.0
    k = torch.zeros_like(k)
    k[..., 0] = -(2.0**40)
    last = bounds(lens)[1:] - 1
    k[:, last, 0] = 3.0
    got = run(serve, q, k, v, bounds(lens), 1.0)
    want = v[:, last].double().repeat_interleave(Hq // Hkv, 0)
    assert ((got[:, last].double() - want).abs() <= 8 * U * want.abs()).all() and got.isfinite().all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_attended_infinities_whatever_their_weight(form, D):
    """An infinity of V reaches every token that attends to it, one whose weight is
    exp(-362) too, before and after a key of weight exp(362) has come; infinities of
    both signs, or a NaN, give NaN; every other output is that of finite values."""
    serve = need_serve()
    dtype, Hq, Hkv, lens = FORMS[form]
    say(f"prompt infinities {form} D={D}")
    g = torch.Generator().manual_seed(D)
    T = sum(lens)
    q = torch.zeros(Hq, T, D)
    q[:, :, 0] = 64.0
    k = torch.zeros(Hkv, T, D)
    v = torch.randn(Hkv, T, D, generator=g)
    at = 0
    for n in lens:
        for low, odd, high in ((3, 20, 35), (130, 160, 250), (1000, 1090, 1151)):
            if n <= high:
                break
            k[:, at + low, 0] = -64.0 * D**0.5 / 11.3
            v[:, at + low, low % 7] = np.inf
            v[:, at + low, 9] = -np.inf
            v[:, at + odd, 9] = np.inf
            v[:, at + odd, 11 + low % 7] = np.nan
            k[:, at + high, 0] = 64.0 * D**0.5 / 11.3
        at += n
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    got = run(serve, q, k, v, bounds(lens))
    fin = v.nan_to_num(0, 0, 0)
    want = expect(q, k, fin, lens, lambda s: (s * D**-0.5).softmax(1))
    odd = v - fin                                              # infinities and NaN among zeros
    odd = torch.where(v.isfinite(), torch.zeros_like(v), v).double()
    at = 0
    for n in lens:
        want[:, at:at + n] += odd[:, at:at + n].cumsum(1).repeat_interleave(Hq // Hkv, 0)
        at += n
    assert torch.equal(got.isnan(), want.isnan())
    inf = want.isinf()
    assert torch.equal(got[inf].double(), want[inf])
    ok = want.isfinite()
    bar = attn_bar(q, k, v, max(lens), D**-0.5, want.nan_to_num(0, 0, 0), dtype, F32)
    assert ((got.double() - want).abs() <= bar)[ok].all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_a_second_pass_leaves_the_bits_of_finite_outputs(form, D):
    """An infinity in one dimension of a value: the other dimensions, and the tokens before
    it, have the bits that they have without it."""
    serve = need_serve()
    dtype, Hq, Hkv, lens = FORMS[form]
    g = torch.Generator().manual_seed(D + 1)
    T = sum(lens)
    q, k, v = (torch.randn(h, T, D, generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
    clean = run(serve, q, k, v, bounds(lens))
    at = 0
    for n in lens:
        v[:, at + n // 2, 5] = np.inf
        clean[:, at + n // 2:at + n, 5] = np.inf
        at += n
    assert torch.equal(run(serve, q, k, v, bounds(lens)), clean)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,low,high", [(20, 0, None), (20, 0, 7), (200, 1, 70), (200, 40, 130), (200, 150, 10)])
def test_float32_weights_below_the_normal_range(D, n, low, high):
    """A weight of exp(-90) on a value of 1e38 counts.  It is a multiple of 2^-149, off by
    2^-20 of itself; beside that the score's error (as in attn_bar) and the sums'."""
    serve = need_serve()
    q = torch.zeros(2, n, D)
    q[:, :, 0] = 1.0
    k = torch.zeros(1, n, D)
    if high is None:
        k[0, low, 0] = -90.0
    else:
        k[0, high, 0] = 90.0                                   # the others fall to exp(-90)
    v = torch.zeros(1, n, D)
    v[0, low] = 1e38
    q, k, v = (x.cuda() for x in (q, k, v))
    got = run(serve, q, k, v, bounds([n]), 1.0)
    want = expect(q, k, v, [n], lambda s: s.softmax(1))
    rel = 2 * (D + 4) * U * 90 + (2 * n + 64) * U + 2.0**-19
    assert ((got.double() - want).abs() <= rel * want).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_infinite_scores(form, D):
    """Scores of -inf have no weight; tokens that attend to nothing else, or to a score of
    +inf, have no softmax: NaN, as the formula gives."""
    serve = need_serve()
    dtype, Hq, Hkv, lens = FORMS[form]
    g = torch.Generator().manual_seed(D + 2)
    T = sum(lens)
    q, k, v = (torch.randn(h, T, D, generator=g) for h in (Hq, Hkv, Hkv))
    q[..., 0] = 1.0
    at = 0
    for n in lens:
        k[:, at:at + min(3, n), 0] = -np.inf
        if n > 30:
            k[:, at + n - 2, 0] = np.inf
        at += n
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    got = run(serve, q, k, v, bounds(lens)).double()
    want = expect(q, k, v, lens, lambda s: (s * D**-0.5).softmax(1))
    assert want.isnan().any() and torch.equal(got.isnan(), want.isnan())
    bar = attn_bar(q, k, v, max(lens), D**-0.5, want.nan_to_num(0), dtype, F32)
    assert ((got - want).abs() <= bar)[~want.isnan()].all()
