"""Log probabilities, entropy and top alternatives on the GPU vs the oracle.

Bars: u = 2^-24.  A row's sum is built from the exponentials of differences d = x - m:
d is rounded once (u |d|), its product with log2 e once more and the exponential is
within an ulp (2 u), so a term w is off by (2 |d| + 2) u w, at most 3 u w more for |d|
w <= 1 / e; a thread adds at most n = vocab / 256 + 1 of them in turn, rescales at most
as often (3 u each), and 8 merges follow: the sum, and so its logarithm, is off by
at most (4 n + 64) u relatively; log2, its product with ln 2 and the two differences
add 4 u (|x - m| + log sum + |result|).  The entropy's second sum is off by the same factor
of its own size, which is at most log(vocab) times the first.
"""
import numpy as np
import pytest

from gpu_common import say, torch
from oracle import serve as o_srv
from serve_common import U, need_serve, replay_checked

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def score(serve, x, targets, k, entropy=True):
    rows, m = targets.shape
    out = [torch.full((rows, m), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda") if entropy else None,
           torch.full((rows, k), 9, dtype=torch.int64, device="cuda"), torch.full((rows, k), 9.0, device="cuda")]
    d = serve.logprob_desc(x, m, k)
    n = serve.logprobs_workspace_bytes(d)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    serve.logprobs(x, targets, *out, ws[:n], d)
    assert (ws[n:] == 0xFF).all()
    return out


def close(got, want, bar):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), (got[odd], want[odd])
    assert (np.abs(got - want)[~odd] <= np.broadcast_to(bar, want.shape)[~odd]).all(), np.abs(got - want)[~odd].max()


def check(x, targets, k, out):
    lp, ent, ids, top = (None if t is None else t.cpu().numpy() for t in out)
    V = x.shape[1]
    for r in range(len(x)):
        wlp, went, wids, wtop = o_srv.logprobs(x[r].double().cpu().numpy(), targets[r].tolist(), k)
        base = (4 * (V / 256 + 1) + 64) * U
        lv = np.log(V) + 1
        with np.errstate(invalid="ignore"):
            close(lp[r], wlp, base + 4 * U * (2 * np.abs(wlp) + lv))
            if ent is not None:
                close(ent[r], went, 2 * base * lv + 4 * U * lv)
            assert np.array_equal(ids[r], wids)
            close(top[r], wtop, base + 4 * U * (2 * np.abs(wtop) + lv))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,m,k", [(1, 1, 1, 1), (3, 2, 2, 4), (5, 63, 1, 64), (2, 64, 0, 5), (4, 65, 3, 0),
                                            (2, 257, 5, 20), (3, 4097, 1, 7), (1, 32000, 5, 5), (2, 50257, 1, 64),
                                            (300, 1001, 1, 3), (2000, 500, 1, 1), (1, 151936, 5, 20), (9, 151936, 300, 1)])
def test_rows_match_the_oracle(dtype, rows, vocab, m, k):
    serve = need_serve()
    say(f"logprobs {dtype} {rows} x {vocab}, {m} targets, top {k}")
    g = torch.Generator().manual_seed(vocab + rows)
    x = (torch.randn(rows, vocab, generator=g) * 3).to(dtype).cuda()
    targets = torch.randint(0, vocab, (rows, m), generator=g).cuda()
    check(x, targets, k, score(serve, x, targets, k))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ties_go_to_the_lowest_id(dtype):
    serve = need_serve()
    x = torch.zeros(4, 9001)
    x[1] = torch.arange(9001) % 3
    x[2, 8000:] = 1.0
    x[3, ::1000] = -0.0                          # equal to 0
    x[3, 17] = -1.0
    x = x.to(dtype).cuda()
    targets = torch.zeros(4, 1, dtype=torch.int64, device="cuda")
    check(x, targets, 64, score(serve, x, targets, 64))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [700, 40_001])
def test_masked_tokens(dtype, vocab):
    """-inf and the type's lowest value in single tokens, most tokens and whole rows; a
    padding target and one past the vocabulary."""
    serve = need_serve()
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(9, vocab, generator=g) * 4
    x[0, ::2] = -np.inf
    x[1, 3:] = -np.inf                           # fewer tokens than alternatives
    x[2] = -np.inf
    x[3, 1:] = low
    x[4] = low                                   # a uniform row
    x[5, :-1] = -np.inf
    x[6] = -np.inf
    x[6, 5] = low
    x[7, ::3] = low
    x[8] = torch.finfo(dtype).max                # uniform at the other end
    x = x.to(dtype).cuda()
    targets = torch.tensor([[0, 1, -1, vocab, -100, vocab - 1]], device="cuda").repeat(9, 1)
    check(x, targets, 6, score(serve, x, targets, 6))


@pytest.mark.parametrize("vocab", [700, 40_001])
def test_nan_and_infinity(vocab):
    serve = need_serve()
    x = torch.randn(5, vocab, generator=torch.Generator().manual_seed(1))
    x[0, 650] = np.nan
    x[1, 3] = np.inf
    x[2, 600], x[2, 400], x[2, 500] = np.inf, np.nan, np.nan
    x[3] = np.nan
    x[4], x[4, 9] = -np.inf, np.nan
    x = x.cuda()
    targets = torch.tensor([[3, -1]], device="cuda").repeat(5, 1)
    check(x, targets, 5, score(serve, x, targets, 5))


@pytest.mark.parametrize("order", ["ascending", "descending", "late"])
def test_orders_that_keep_the_list_busy(order):
    """Every logit a new best, none after the first, and the best ones last."""
    serve = need_serve()
    V = 60_000
    x = torch.linspace(-20, 20, V)[None].repeat(2, 1)
    if order == "descending":
        x = x.flip(1)
    if order == "late":
        x = torch.zeros(2, V)
        x[:, -30:] = torch.arange(30.0)
    x = x.contiguous().cuda()
    targets = torch.tensor([[0], [V - 1]], device="cuda")
    check(x, targets, 64, score(serve, x, targets, 64))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off,pad", [(0, 0), (1, 0), (3, 5), (0, 8)])
def test_alignment_and_row_strides(dtype, off, pad):
    """Rows at any element alignment; what lies between them is not read."""
    serve = need_serve()
    rows, V = 6, 5003
    buf = torch.full((rows * (V + pad) + off + 64,), float("nan"), dtype=dtype, device="cuda")
    x = buf[off:off + rows * (V + pad)].view(rows, V + pad)[:, :V]
    x.copy_(torch.randn(rows, V, generator=torch.Generator().manual_seed(off)) * 2)
    targets = torch.tensor([[0, V - 1]], device="cuda").repeat(rows, 1)
    check(x, targets, 9, score(serve, x, targets, 9))


def test_entropy_and_lists_may_be_missing():
    serve = need_serve()
    x = torch.randn(3, 70_000, generator=torch.Generator().manual_seed(2)).cuda()
    targets = torch.zeros(3, 1, dtype=torch.int64, device="cuda")
    out = score(serve, x, targets, 0, entropy=False)
    check(x, targets, 0, out)
    ent = torch.empty(3, device="cuda")
    d = serve.logprob_desc(x, 0, 0)
    ws = torch.empty(serve.logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    serve.logprobs(x, None, None, ent, None, None, ws, d)
    assert torch.equal(ent, score(serve, x, targets, 2)[1])


def test_offsets_beyond_32_bits():
    serve = need_serve()
    rows, V = 300, 16_000_000
    x = torch.empty(rows, V, dtype=BF16, device="cuda")                # 9.6 GB
    x[:-1].fill_(0)
    x[-1].normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    targets = torch.full((rows, 1), V - 1, dtype=torch.int64, device="cuda")
    lp, ent, ids, top = score(serve, x, targets, 3)
    want = torch.log_softmax(x[-1].double(), 0)
    tv, ti = want.topk(3)
    base = (4 * (V / 256 + 1) + 64) * U
    assert abs(lp[-1, 0].item() - want[-1].item()) <= base + 200 * U and (top[-1].double() - tv).abs().max() <= base + 200 * U
    assert torch.equal(x[-1][ids[-1]], x[-1][ti]) and (ids[0] == torch.arange(3, device="cuda")).all()
    assert abs(lp[0, 0].item() + np.log(V)) <= base + 200 * U


def test_rows_do_not_depend_on_each_other_and_graph():
    """A row's bits on another stream; one pass captured and replayed."""
    serve = need_serve()
    x = (torch.randn(40, 32000, generator=torch.Generator().manual_seed(4)) * 3).to(BF16).cuda()
    targets = torch.randint(0, 32000, (40, 2), generator=torch.Generator().manual_seed(5)).cuda()
    out = score(serve, x, targets, 5)
    again = score(serve, x, targets, 5)
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    d = serve.logprob_desc(x, 2, 5)
    ws = torch.empty(serve.logprobs_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = [torch.empty_like(t) for t in out]
    serve.logprobs(x, targets, *other, ws, d, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, other))
    replay_checked(lambda: serve.logprobs(x, targets, *out, ws, d), out, lambda i: (x.mul_(-0.9), targets.add_(1).remainder_(32000)))
