"""The paged cache on the GPU: rows into their pages bit for bit, attention of new tokens
over it against float64."""
import math

import numpy as np
import pytest

from gpu_common import say, torch
from oracle import serve as o_srv
from serve_common import attn_bar, bounds, head_view, need_serve, replay_checked

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
EVERY = 2**31 - 1


def randn(*shape, seed=0, dtype=BF16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def ids(v, dtype=torch.int64):
    return torch.tensor(v, dtype=dtype, device="cuda")


def a_table(need, max_pages, pages, seed=0, fill=-1):
    """Block table of sequences of need[b] pages, scattered over all `pages`."""
    order = np.random.default_rng(seed).permutation(pages)[:sum(need)]
    table, at = np.full((len(need), max_pages), fill, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


@pytest.mark.parametrize("kind", ["none", "plain", "yarn"])
@pytest.mark.parametrize("D,Hq,Hkv,page", [(64, 5, 5, 1), (128, 6, 2, 16), (64, 8, 1, 64), (128, 0, 3, 32)])
@pytest.mark.parametrize("long", [40, 2100])            # one pair a lane, four pairs a lane
def test_store(kind, D, Hq, Hkv, page, long):
    """Every row at its place with the bits of the plain rotation; tokens without a place,
    places without a token and rows outside the sequences as they were."""
    serve = need_serve()
    from paper_2607_21927_amd import ris
    lens, start = [long, 0, 1, 33, 20, 9], [5, 0, 99, 80, -3, 10**12]
    lead, T = 2, sum(lens) + 5
    cu = bounds(lens) + lead
    places = (long + 5 + page - 1) // page * page
    mp = places // page
    pages = 3 * mp + 7
    need = [mp, 0, mp, 0, mp, 0]
    table = a_table(need, mp, pages, seed=D + page)
    table[0, 0] = pages                       # one past the last page
    table[3] = -(2**31)
    if mp > 1:
        table[2, mp - 1] = 2**31 - 1
    buf = randn(T, (Hq + 2 * Hkv) * D + 8, seed=D)[:, :(Hq + 2 * Hkv) * D]
    q, k, v = head_view(buf, 0, Hq, D), head_view(buf, Hq, Hkv, D), head_view(buf, Hq + Hkv, Hkv, D)
    rd = None if kind == "none" else ris.rope_desc(dict(plain=ris.ROPE_PLAIN, yarn=ris.ROPE_YARN)[kind], 1e4,
                                                   orig_max_pos=2048, factor=4.0)
    both = torch.full((pages, 2, Hkv, page, D), 7.0, dtype=BF16, device="cuda")     # pages of K and V side by side
    Kp, Vp = both[:, 0], both[:, 1]
    q_out = head_view(torch.full((T, max(Hq, 1) * D), 3.0, dtype=BF16, device="cuda"), 0, Hq, D)
    kw = dict(q=q, q_out=q_out) if Hq else {}
    say(f"store: {kind} D={D} heads {Hq}/{Hkv} page {page} {long} tokens")
    serve.page_store(k, v, cu, ids(table, torch.int32), Kp, Vp, start=ids(start), rope=rd, **kw)
    torch.cuda.synchronize()
    want, want_q = torch.full_like(both, 7.0), torch.full_like(q_out, 3.0)
    at = lead
    for b, (n, p) in enumerate(zip(lens, start)):
        if n == 0:
            continue
        rows = []
        for x in (q, k):
            x = x[:, at:at + n]
            if rd is not None and x.shape[0]:
                x = serve.rope_packed(x, torch.empty(x.shape, dtype=BF16, device="cuda"), bounds([n]), rd, start=ids([p]))
            rows.append(x)
        want_q[:, at:at + n] = rows[0]
        where = o_srv.page_places(table[b], page, pages)
        for i in range(n):
            if 0 <= p + i < places and where[p + i, 0] >= 0:
                pg, slot = where[p + i]
                want[pg, 0, :, slot], want[pg, 1, :, slot] = rows[1][:, i], v[:, at + i]
        at += n
    assert torch.equal(both, want)
    if Hq:
        assert torch.equal(q_out, want_q)
        # in place
        serve.page_store(k, v, cu, ids(table, torch.int32), Kp, Vp, start=ids(start), rope=rd, q=q, q_out=q)
        assert torch.equal(q[:, lead:at], want_q[:, lead:at]) and torch.equal(both[:, 1], want[:, 1])


def test_store_keeps_infinities_and_nan():
    serve = need_serve()
    k, v = randn(2, 10, 64), randn(2, 10, 64, seed=1)
    v[0, 3, 7], v[1, 4, 63], k[0, 2, 5] = math.nan, math.inf, -math.inf
    Kp, Vp = serve.page_cache(2, 2, 16, 64)
    serve.page_store(k, v, bounds([10]), ids([[1]], torch.int32), Kp, Vp)
    for got, x in ((Kp, k), (Vp, v)):
        assert torch.equal(got[1, :, :10].view(torch.int16), x.view(torch.int16)) and not got[0].any()


@pytest.mark.parametrize("n", [10, 2100])
def test_store_copies_bits(n):
    """What is not rotated keeps its bits: every bf16 pattern, signalling NaN and denormals among
    them."""
    serve = need_serve()
    bits = torch.arange(n * 2 * 64, dtype=torch.int32, device="cuda").mul_(40503).to(torch.int16).view(BF16).view(2, n, 64)
    k, q = bits.flip(1).contiguous(), bits.flip(0).contiguous()
    page = 64
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    Kp, Vp = serve.page_cache(table.shape[1], 2, page, 64)
    q_out = torch.zeros_like(q)
    serve.page_store(k, bits, bounds([n]), table, Kp, Vp, q=q, q_out=q_out)
    for got, x in ((Kp, k), (Vp, bits)):
        rows = got[table[0].long()].transpose(1, 2).flatten(0, 1)[:n].transpose(0, 1)
        assert torch.equal(rows.contiguous().view(torch.int16), x.view(torch.int16))
    assert torch.equal(q_out.view(torch.int16), q.view(torch.int16))


def attend(serve, q, Kp, Vp, table, cu, start, window=None, sink=0, scale=0.0, out=None, dtype=F32):
    Hq, T, D = q.shape
    if out is None:
        out = torch.full((Hq, T, D), 3.0, dtype=dtype, device="cuda")
    desc = serve.page_attn_desc(q, Kp, table, cu, out, window=window, sink=sink, scale=scale)
    ws = torch.full((serve.page_attn_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")     # NaN
    return serve.page_attn(q, Kp, Vp, table, cu, out, ws, desc, start=start)


def held(lens, start, page, Hq, Hkv, D, seed=0, spare=3, cap=None):
    """A batch whose cache is filled up to its last token: q, pages (what no sequence owns, or
    lies behind its end, is NaN), table (numpy), cu, start."""
    places = max(max(p + n for p, n in zip(start, lens)), 1)
    mp = cap or (places + page - 1) // page
    need = [min(mp, (p + n + page - 1) // page) if n else 0 for p, n in zip(start, lens)]
    pages = sum(need) + spare
    table = a_table(need, mp, pages, seed=seed)
    Kp, Vp = randn(pages, Hkv, page, D, seed=seed + 1), randn(pages, Hkv, page, D, seed=seed + 2)
    dead = np.ones((pages, page), bool)
    for b, (p, n) in enumerate(zip(start, lens)):
        where = o_srv.page_places(table[b], page, pages)[:p + n if n else 0]
        where = where[where[:, 0] >= 0]
        dead[where[:, 0], where[:, 1]] = False
    dead = torch.tensor(dead, device="cuda")[:, None, :, None]
    Kp.masked_fill_(dead, math.nan)
    Vp.masked_fill_(dead, math.nan)
    return randn(Hq, sum(lens), D, seed=seed + 3), Kp, Vp, table, bounds(lens), start


def check(serve, q, Kp, Vp, table, cu, start, window=EVERY, sink=0, scale=0.0, dtype=F32, what=""):
    D = q.shape[-1]
    got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), window, sink, scale, dtype=dtype).double().cpu()
    c = scale or D**-0.5
    want = torch.tensor(o_srv.paged_attention(q.double().cpu().numpy(), Kp.double().cpu().numpy(), Vp.double().cpu().numpy(),
                                              table, cu.tolist(), start, window, sink, c))
    n = min(max(1, table.shape[1] * Kp.shape[2]), window + sink) + 1
    bar = attn_bar(q, Kp, Vp, n, c, want, BF16, dtype)
    assert torch.equal(got.isnan(), want.isnan()), what
    fin = want.isfinite()
    assert torch.equal(got[~fin].nan_to_num(nan=1e30), want[~fin].nan_to_num(nan=1e30))
    worst = float(((got - want).abs() / bar)[fin].max()) if fin.any() else 0.0
    say(f"{what} off by {worst:.3f} of the bar")
    assert worst <= 1.0
    return got


BATCHES = {
    "one": ([1], [0]),
    "step": ([1, 1, 1, 1, 1], [0, 63, 64, 300, 127]),
    "few": ([3, 1, 5, 0, 2], [10, 700, 61, 5, 0]),
    "chunk": ([70, 0, 129, 1], [0, 0, 333, 500]),
    "prompt": ([257], [0]),
    "shared": ([70, 0, 30, 1, 1], [1200, 0, 0, 700, 2]),      # places enough for row tiles to be shared by workgroups
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("Hq,Hkv,D,page", [(12, 2, 128, 64), (8, 1, 64, 16), (3, 3, 64, 128), (15, 5, 128, 1), (7, 1, 64, 2)])
def test_attention(batch, Hq, Hkv, D, page, dtype):
    serve = need_serve()
    lens, start = BATCHES[batch]
    for window, sink in ((EVERY, 0), (100, 3), (1, 0), (0, 70), (64, 64)):
        check(serve, *held(lens, start, page, Hq, Hkv, D, seed=7), window=window, sink=sink, dtype=dtype,
              what=f"{batch} {Hq}/{Hkv} D={D} page {page} window {window} sink {sink}")


@pytest.mark.parametrize("G", [1, 16, 33, 128])
def test_groups(G):
    serve = need_serve()
    check(serve, *held([5, 1, 40], [100, 3, 0], 16, 2 * G, 2, 64, seed=G), window=50, sink=2, what=f"G={G}")


@pytest.mark.parametrize("Hq,Hkv,D", [(12, 2, 128), (32, 4, 64)])
def test_long_caches(Hq, Hkv, D):
    """One and a few tokens over tens of thousands of keys, sequences of very unequal lengths."""
    serve = need_serve()
    for lens, start, window, sink in (([1], [33_333], EVERY, 0), ([1, 4, 1], [9_000, 12, 20_001], EVERY, 0),
                                      ([2, 1], [30_000, 77], 5000, 10)):
        check(serve, *held(lens, start, 64, Hq, Hkv, D, seed=len(lens)), window=window, sink=sink, what=f"{start} window {window}")


def test_empty_rows_and_positions_without_a_place():
    """Pages that are not there, positions before 0 and behind the last place, rows outside every
    sequence."""
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([6, 30, 4, 8], [200, 5, 140, 0], 16, 12, 2, 128, seed=3, cap=9)   # 144 places
    table[0] = -1                                        # nothing there: zeros
    table[1, 0] = Kp.shape[0] + 5                        # the first 16 keys are not there
    start = [30, 5, 142, -3]                             # two of four and five of eight have a place
    got = check(serve, q, Kp, Vp, table, cu, start, what="places")
    assert not got[:, :6].any() and not got[:, 38:40].any() and not got[:, 40:43].any() and got[:, 43:].any()
    check(serve, q, Kp, Vp, table, cu, start, window=3, sink=1, what="places under a window")
    out = torch.full((12, 50, 128), 3.0, dtype=BF16, device="cuda")
    q50 = randn(12, 50, 128)
    for c in (cu + 1, cu - 4):                           # rows before and behind; clipped offsets
        attend(serve, q50, Kp, Vp, ids(table, torch.int32), c, ids([0, 5, 142, -3]), out=out.fill_(3.0))
        lo, hi = max(int(c[0]), 0), int(c[-1])
        assert (out[:, :lo] == 3).all() and (out[:, hi:] == 3).all() and not (out[:, lo:hi] == 3).all(-1).any()


def test_far_starts_give_zeros():
    serve = need_serve()
    q, Kp, Vp, table, cu, _ = held([2, 2, 2, 2], [0, 0, 0, 0], 16, 4, 1, 64)
    out = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids([2**62, -2**62, 2**31 - 1, -2**31 - 1]))
    assert not out.any()
    serve.page_store(q[:1], q[:1], cu, ids(table, torch.int32), Kp[:, :1], Vp[:, :1], start=ids([2**62, -2**62, 2**31, -9]))


def test_what_is_not_attended_to_does_not_count():
    """NaN and infinities behind a window, behind a row's position, in another row's keys."""
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([40, 3], [100, 700], 16, 6, 2, 128, seed=5)
    where = [o_srv.page_places(t, 16, Kp.shape[0]) for t in table]

    def put(x, b, j, d, v):
        x[where[b][j, 0], :, where[b][j, 1], d] = v
    for b, j in ((0, 30), (0, 64), (1, 500), (1, 3)):         # outside every window of 20 and 2 first tokens
        put(Vp, b, j, 3, math.nan), put(Kp, b, j, 5, math.inf)
    check(serve, q, Kp, Vp, table, cu, start, window=20, sink=2, what="behind the window")
    # seen by some rows of a tile alone: NaN, infinities of one and of both signs
    put(Vp, 0, 110, 4, math.inf), put(Vp, 0, 125, 4, -math.inf), put(Vp, 0, 118, 9, math.nan), put(Vp, 1, 701, 0, -math.inf)
    check(serve, q, Kp, Vp, table, cu, start, window=20, sink=2, what="in some rows' windows")


@pytest.mark.parametrize("n,p", [(3, 400), (1, 3000), (100, 400), (40, 5000)])
def test_infinite_values_count_whatever_their_weight(n, p):
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([n], [p], 64, 2, 1, 64, seed=8)
    Kp *= 40.0
    where = o_srv.page_places(table[0], 64, Kp.shape[0])
    Vp[where[7, 0], :, where[7, 1], 11] = math.inf
    got = check(serve, q, Kp, Vp, table, cu, start, what="an infinite value")
    assert (got[..., 11] == math.inf).all()


def test_scores_far_from_zero():
    """Scores around +-30,000 with differences of a few units: weights are those differences'."""
    serve = need_serve()
    for sign in (1.0, -1.0):
        for lens, start in (([2, 70], [900, 0]), ([2, 1], [900, 3]), ([60, 1], [10, 100])):
            q, Kp, Vp, table, cu, start = held(lens, start, 32, 4, 1, 64, seed=9)
            Kp[..., 0], q[..., 0] = 512.0, sign * 512.0
            check(serve, q, Kp, Vp, table, cu, start, scale=0.125, what=f"far {sign} {lens}")
            check(serve, q, Kp, Vp, table, cu, start, scale=2.0**14, what=f"farther {sign} {lens}")


@pytest.mark.parametrize("n,p", [(1, 70), (1, 5000), (90, 70), (90, 3000)])
def test_scores_of_minus_infinity_alone(n, p):
    """NaN, though zeros where there is no score at all; a NaN query is its own row's alone."""
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([n, 1, n], [p, 30, 0], 16, 2, 1, 64, seed=2)
    where = o_srv.page_places(table[0], 16, Kp.shape[0])[:p + n]
    Kp[where[:, 0], 0, where[:, 1], 0] = -math.inf
    q[:, :n, 0], q[0, n] = 1.0, math.nan
    table[2] = -1
    out = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start))
    assert out[:, :n].isnan().all() and out[0, n].isnan().all() and out[1, n].isfinite().all() and not out[:, n + 1:].any()


def test_scales():
    serve = need_serve()
    for scale in (1e-38, 1e-3, 3.0, 2.0**100):
        case = held([1, 20], [300, 40], 64, 2, 2, 128, seed=4)
        if scale > 1e30:                                      # the largest score alone counts
            q, Kp, Vp, table, cu, start = case
            got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), scale=scale)
            assert got.isfinite().all()
            continue
        check(serve, *case, scale=scale, what=f"scale {scale}")


def test_far_page_numbers():
    """Rows whose offsets in the pages pass 32 bits."""
    serve = need_serve()
    pages, page, D = 70_000, 256, 128                          # 4.6 GB each
    Kp = torch.zeros(pages, 1, page, D, dtype=BF16, device="cuda")
    Vp = torch.zeros(pages, 1, page, D, dtype=BF16, device="cuda")
    table = np.array([[69_999, 3, 40_000], [65_536, 65_535, 69_998]], np.int32)
    lens, start, small = [4, 300], [600, 200], [69_999, 3, 40_000, 65_536, 65_535, 69_998]
    q, k, v = randn(2, 304, D), randn(1, 304, D, seed=1), randn(1, 304, D, seed=2)
    for i, p in enumerate(small):
        Kp[p], Vp[p] = randn(1, page, D, seed=10 + i), randn(1, page, D, seed=20 + i)
    cu = bounds(lens)
    serve.page_store(k, v, cu, ids(table, torch.int32), Kp, Vp, start=ids(start))
    got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start))
    K6, V6 = Kp[small].clone(), Vp[small].clone()
    near = np.array([[0, 1, 2], [3, 4, 5]], np.int32)
    assert torch.equal(K6[[0, 1, 2]][:, 0].flatten(0, 1)[600:604], k[0, :4])
    want = attend(serve, q, K6, V6, ids(near, torch.int32), cu, ids(start))
    assert torch.equal(got, want)
    check(serve, q, K6, V6, near, cu, start, what="far pages")


def test_shared_pages():
    """Sequences that share their first pages see the same keys."""
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([1, 1, 1], [255, 255, 200], 64, 4, 2, 64, seed=6)
    table[1, :3], table[2, :3] = table[0, :3], table[0, :3]
    check(serve, q, Kp, Vp, table, cu, start, what="shared")


def test_strided_views():
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([30, 1, 9], [5, 400, 64], 32, 12, 2, 128, seed=12)
    want = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), window=77, sink=3, dtype=BF16)
    buf = torch.zeros(40, 20 * 128, dtype=BF16, device="cuda")
    qv = head_view(buf, 4, 12, 128).copy_(q)
    both = torch.stack([Kp, Vp], 1)
    wide = torch.full((3, table.shape[1] + 5), 1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = ids(table, torch.int32)
    out = head_view(torch.zeros(40, 13 * 128, dtype=BF16, device="cuda"), 0, 12, 128)
    got = attend(serve, qv, both[:, 0], both[:, 1], wide[:, :table.shape[1]], cu, ids(start), window=77, sink=3, out=out)
    assert torch.equal(got, want)


def test_many_sequences():
    """More sequences than one search step, empty ones among them."""
    serve = need_serve()
    rng = np.random.default_rng(0)
    lens = [int(n) for n in rng.integers(0, 4, 300)]
    start = [int(p) for p in rng.integers(0, 90, 300)]
    check(serve, *held(lens, start, 16, 4, 2, 64, seed=13), what="300 sequences")
    check(serve, *held(lens, start, 16, 4, 2, 64, seed=13), window=30, sink=1, what="300 sequences, window")


def test_chunks_give_what_the_whole_prompt_gives():
    """A prompt stored and attended to in pieces against dense attention of the whole: both are
    within the bar of the same formula."""
    serve = need_serve()
    Hq, Hkv, D, n = 12, 2, 128, 700
    q, k, v = randn(Hq, n, D), randn(Hkv, n, D, seed=1), randn(Hkv, n, D, seed=2)
    whole = torch.empty(Hq, n, D, dtype=F32, device="cuda")
    cu = bounds([n])
    serve.prompt_attn(q, k, v, cu, whole, serve.prompt_desc(q, k, v, whole, cu))
    Kp, Vp = serve.page_cache(12, Hkv, 64, D)
    table = ids([[11, 3, 7, 0, 1, 9, 5, 2, 4, 8, 6]], torch.int32)
    at = 0
    for m in (1, 130, 64, 300, 2, 203):
        c = bounds([m])
        serve.page_store(k[:, at:at + m], v[:, at:at + m], c, table, Kp, Vp, start=ids([at]))
        got = attend(serve, q[:, at:at + m], Kp, Vp, table, c, ids([at]))
        want = whole[:, at:at + m].double()
        bar = 2 * attn_bar(q, k, v, n, D**-0.5, want, BF16, F32)
        assert bool(((got.double() - want).abs() <= bar).all()), at
        at += m


def test_captured_and_replayed():
    """Store and attention in a graph whose lengths, positions and pages change between replays."""
    serve = need_serve()
    Hq, Hkv, D, page, T = 12, 2, 128, 64, 60
    qkv = randn(T, (Hq + 2 * Hkv) * D)
    q, k, v = (head_view(qkv, a, n, D) for a, n in ((0, Hq), (Hq, Hkv), (Hq + Hkv, Hkv)))
    Kp, Vp = (randn(200, Hkv, page, D, seed=s) for s in (1, 2))
    table = ids(np.random.default_rng(3).permutation(200)[:192].reshape(4, 48), torch.int32)
    cu, start = bounds([1, 50, 1, 8]), ids([2000, 30, 900, 7])
    out = torch.zeros(T, Hq * D, dtype=BF16, device="cuda")
    view = head_view(out, 0, Hq, D)
    desc = serve.page_attn_desc(q, Kp, table, cu, view, window=1500, sink=4)
    ws = torch.empty(serve.page_attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def step():
        serve.page_store(k, v, cu, table, Kp, Vp, start=start)
        serve.page_attn(q, Kp, Vp, table, cu, view, ws, desc, start=start)

    def change(i):
        qkv.copy_(randn(T, (Hq + 2 * Hkv) * D, seed=20 + i))
        cu.copy_(bounds([[1, 50, 1, 8], [20, 20, 20, 0], [1, 1, 1, 1], [60, 0, 0, 0]][i]))
        start.copy_(ids([[2001, 80, 901, 15], [100, 2000, 0, 5], [3000, 3, 2500, 0], [2900, 0, 0, 0]][i]))
        table.copy_(table.roll(i, 0))
    replay_checked(step, [out], change, times=4)


def test_another_stream():
    serve = need_serve()
    q, Kp, Vp, table, cu, start = held([3, 1], [60, 2000], 64, 12, 2, 128, seed=14)
    t, s0 = ids(table, torch.int32), ids(start)
    want = attend(serve, q, Kp, Vp, t, cu, s0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = attend(serve, q, Kp, Vp, t, cu, s0)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def on_the_gpu(q, Kp, Vp, table, cu, start, window, sink):
    """The oracle's formula with torch in float64, for batches that are too large for it."""
    Hq, T, D = q.shape
    pages, Hkv, page, _ = Kp.shape
    out = torch.zeros(Hq, T, D, dtype=torch.float64, device="cuda")
    for b, (a, z) in enumerate(zip(cu.tolist()[:-1], cu.tolist()[1:])):
        at = torch.tensor(o_srv.page_places(table[b], page, pages), device="cuda")
        p = torch.arange(start[b], start[b] + z - a, device="cuda")[:, None]
        j = torch.arange(len(at), device="cuda")
        keep = (j <= p) & ((j > p - window) | (j < sink)) & (at[:, 0] >= 0) & (p >= 0) & (p < len(at))
        at = at.clamp(min=0)
        for h in range(Hq):
            k, v = (x[at[:, 0], h // (Hq // Hkv), at[:, 1]].double().nan_to_num(0, 0, 0) for x in (Kp, Vp))
            w = torch.where(keep, q[h, a:z].double() @ k.t().contiguous() * D**-0.5, -math.inf).softmax(1).nan_to_num(0)
            out[h, a:z] = w @ v
    return out


@pytest.mark.parametrize("Hq,Hkv,D,lens", [(16, 16, 128, [5000, 3300]), (16, 16, 64, [8300]), (24, 8, 128, [2700, 1, 2700, 0, 460]),
                                           (16, 16, 64, [9000, 3100])])
def test_many_row_tiles(Hq, Hkv, D, lens):
    """So many row tiles that they are not shared, with little and much left for the last round;
    positions without a place and infinities among what is."""
    serve = need_serve()
    start = [600] + [40] * (len(lens) - 1)
    q, Kp, Vp, table, cu, start = held(lens, start, 64, Hq, Hkv, D, seed=3)
    if len(lens) > 1:
        start[-1] = -10                                              # the first ten tokens have no place
    for window, sink in ((300, 5), (EVERY, 0)):
        want = on_the_gpu(q, Kp, Vp, table, cu, start, window, sink)
        got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), window, sink)
        bar = attn_bar(q, Kp, Vp, max(start) + max(lens), D**-0.5, want, BF16, F32)
        worst = float(((got.double() - want).abs() / bar).max())
        say(f"{lens} {Hq}/{Hkv} D={D} window {window}: off by {worst:.3f} of the bar")
        assert worst <= 1.0
        assert len(lens) == 1 or not got[:, -lens[-1]:][:, :10].any()
    # an infinite value that the first and last tokens of a sequence attend to, and one that few do
    w = o_srv.page_places(table[0], 64, Kp.shape[0])
    Vp[w[2, 0], :, w[2, 1], 7], Vp[w[-70, 0], :, w[-70, 1], 9] = math.inf, math.nan
    got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), 300, 5)
    n, first = lens[0], start[0]
    assert torch.isinf(got[:, :n, 7]).all()
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    j = len(w) - 70
    p = torch.arange(first, first + n, device="cuda")
    hit[(p >= j) & (p < j + 300)] = True                       # w[j] is a page of the sequence's: it is its last
    assert torch.equal(got[:, :n, 9].isnan(), hit.expand(Hq, n))
    assert got[:, n:].isfinite().all() and got[:, :n, 10:].isfinite().all()


@pytest.mark.parametrize("lens,Hq", [((400, 600), 12), ((3, 2), 4)])
def test_offsets_that_do_not_ascend(lens, Hq):
    """Sequences that overlap have no result, but every access stays in place: 1,500 row tiles where
    the host counted on 100, no memory but out's own written."""
    serve = need_serve()
    lens, start = list(lens), [700, 30]
    q, Kp, Vp, table, cu, start = held(lens, start, 64, Hq, 2, 128, seed=15)
    T = sum(lens)
    wide = np.concatenate([table, np.full((30, table.shape[1]), -1, np.int32), table[:1]])
    bad = torch.tensor([0, lens[0], T] + [0, T] * 15 + [0], dtype=torch.int64, device="cuda")
    starts = start + [0] * 31
    room = torch.full((Hq, 3 * T, 128), 7.0, dtype=F32, device="cuda")
    keep = Kp.clone()
    attend(serve, q, Kp, Vp, ids(wide, torch.int32), bad, ids(starts), out=room[:, T:2 * T])
    serve.page_store(q[:2], q[:2], bad, ids(np.full_like(wide, -1), torch.int32), Kp, Vp, start=ids(starts))
    torch.cuda.synchronize()
    assert (room[:, :T] == 7).all() and (room[:, 2 * T:] == 7).all() and torch.equal(Kp.nan_to_num(9), keep.nan_to_num(9))
