"""Attention over a paged cache where many waves and workgroups share a row's keys: a tile of keys that
is lost or counted twice shows.

Scores are whole numbers in [-4, 0] and the scale times log2 e is 1 in float32, so that softmax weights are
powers of two, values are whole numbers up to 8, and every sum is exact in float32 (multiples of 2^-4 below
2^20).  An output is a quotient then, off by two roundings; exp(scale s) is off 2^s by 4 u.  The bar is 8 u
of the weighted mean of |v|, u = 2^-24; leaving out any 32 neighbouring keys changes an output by more (held of
the reference itself, key tile by key tile)."""
import math

import numpy as np
import pytest

from gpu_common import say, torch
from oracle import serve as o_srv
from serve_common import U, bounds, need_serve
from test_gpu_page import EVERY, a_table, attend, ids

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SCALE = 0.6931471824645996                # the float32 whose product with log2 e is 1


def whole(shape, lo, hi, seed):
    """Whole numbers lo .. hi, bf16."""
    return torch.randint(lo, hi + 1, shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(BF16)


def batch_of(lens, start, page, Hq, Hkv, D, places, seed):
    need = [-(-(p + n) // page) for p, n in zip(start, lens)]
    pages = sum(need) + 2
    table = a_table(need, -(-places // page), pages, seed=seed)
    Kp, Vp = torch.zeros(pages, Hkv, page, D, dtype=BF16, device="cuda"), whole((pages, Hkv, page, D), -8, 8, seed)
    Kp[..., 3] = whole((pages, Hkv, page), -2, 0, seed + 1)
    for i in set(range(pages)) - set(table[table >= 0].tolist()):
        Kp[i], Vp[i] = math.nan, math.nan
    q = torch.zeros(Hq, sum(lens), D, dtype=BF16, device="cuda")
    q[..., 3] = whole((Hq, sum(lens)), 1, 2, seed + 2)
    return q, Kp, Vp, table, bounds(lens), start


def reference(q, Kp, Vp, table, cu, start, window, sink, tiles=False):
    """Outputs and their bars in float64; tiles: that every 32 keys that the sequence's last row attends to matter."""
    Hq, T, D = q.shape
    pages, Hkv, page, _ = Kp.shape
    G = Hq // Hkv
    out, bar = (torch.zeros(Hq, T, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, (a, z) in enumerate(zip(cu.tolist()[:-1], cu.tolist()[1:])):
        if a == z:
            continue
        at = torch.tensor(o_srv.page_places(table[b], page, pages)[:start[b] + z - a], device="cuda")
        p = torch.arange(start[b], start[b] + z - a, device="cuda")[:, None]
        j = torch.arange(len(at), device="cuda")
        keep = (j <= p) & ((j > p - window) | (j < sink))
        for g in range(Hkv):
            k, v = Kp[at[:, 0], g, at[:, 1], 3].double(), Vp[at[:, 0], g, at[:, 1]].double()
            for h in range(g * G, g * G + G):
                w = torch.where(keep, torch.exp(SCALE * q[h, a:z, 3].double()[:, None] * k), 0.0)
                n = w.sum(1, keepdim=True)
                out[h, a:z], bar[h, a:z] = w @ v / n, 8 * U * (w @ v.abs()) / n
            if tiles and len(at) > 64:
                num = torch.nn.functional.pad(w[-1][:, None] * v, (0, 0, 0, -len(j) % 32)).unflatten(0, (-1, 32)).sum(1)
                den = torch.nn.functional.pad(w[-1], (0, -len(j) % 32)).unflatten(0, (-1, 32)).sum(1)
                less = (num.sum(0) - num) / (den.sum() - den)[:, None]
                off = ((less - out[h, z - 1]).abs() / bar[h, z - 1]).amax(1)
                assert bool((off[den > 0] > 1).all()), "a lost tile of keys would pass"
    return out, bar


def unequal(n, most, seed):
    """Lengths of n sequences up to `most`, one that long, some of them short."""
    x = np.random.default_rng(seed).integers(1, most, n)
    x[0], x[1 % n] = most, 5
    return [int(v) for v in x]


# lens, tokens held before, places of a row of the table (0: what the longest needs).  Steps whose keys and values come to
# more than 256 MiB over all places, and less; row tiles in parts and whole ones.
CASES = {
    "one of 33,000": ([1], [33_333], 0),
    "unequal": ([1, 2, 1], [9_000, 12, 20_001], 0),
    "many long": ([1] * 9, unequal(9, 33_000, 1), 33_024),
    "few in wide tables": ([1, 2, 1], [700, 31, 64], 131_072),
    "many of 2,560": ([1] * 161, unequal(161, 2_559, 2), 2_560),
    "chunk": ([70], [33_000], 0),
    "chunks": ([70, 1, 0, 300], [20_000, 9_000, 0, 5_000], 0),
    "chunks beside many": ([40] * 4 + [1] * 260, unequal(264, 2_000, 3), 2_304),
}


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("Hq,Hkv,D,page", [(12, 2, 128, 64), (32, 4, 64, 16)])
def test_every_key_counts(case, Hq, Hkv, D, page):
    serve = need_serve()
    lens, start, places = CASES[case]
    batch = batch_of(lens, start, page, Hq, Hkv, D, places or max(n + p for n, p in zip(lens, start)), seed=len(lens))
    q, Kp, Vp, table, cu, start = batch
    for window, sink in ((EVERY, 0), (5000, 10)):
        got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), window, sink, SCALE)
        want, bar = reference(*batch, window, sink, tiles=len(lens) < 10)
        worst = float(((got.double() - want).abs() / bar.clamp(min=1e-30)).max())
        say(f"{case} {Hq}/{Hkv} D={D} window {window}: off by {worst:.3f} of the bar")
        assert worst <= 1.0
        again = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), window, sink, SCALE)
        assert torch.equal(got, again)                       # nothing depends on which workgroup is first


@pytest.mark.parametrize("lens,start", [([1, 3], [300, 40]), ([20, 1], [300, 900]), ([70, 1], [20, 5]), ([90, 1], [2000, 7])])
def test_the_largest_score_alone_at_a_huge_scale(lens, start):
    """At a scale of 2^100 a row gives the value of its largest score.  Sums under an earlier
    maximum, 2,007 values of up to 8 under weights of up to 2^8, keep a factor of 2^-149 in the pass that keeps
    infinities: below 2^-127.  The matrix unit cuts off such a remnant where it adds the value to it, an ulp
    (2 u) of the value then; the other additions there are of zeros.  The division is a rounding."""
    serve = need_serve()
    q, Kp, Vp, table, cu, start = batch_of(lens, start, 64, 4, 2, 128, max(n + p for n, p in zip(lens, start)), seed=4)
    Kp[..., 3] = 0.0
    for b, (p, n) in enumerate(zip(start, lens)):             # a key's score rises with a permutation of the positions
        at = torch.tensor(o_srv.page_places(table[b], 64, Kp.shape[0])[:p + n], device="cuda")
        score = torch.randperm(p + n, generator=torch.Generator().manual_seed(b)).cuda()
        for g in range(2):
            Kp[at[:, 0], g, at[:, 1], 0], Kp[at[:, 0], g, at[:, 1], 1] = (score // 128).to(BF16), (score % 128).to(BF16)
    q.zero_()
    q[..., 0], q[..., 1] = 128.0, 1.0
    got = attend(serve, q, Kp, Vp, ids(table, torch.int32), cu, ids(start), scale=2.0**100)
    for b, (a, z) in enumerate(zip(cu.tolist()[:-1], cu.tolist()[1:])):
        at = torch.tensor(o_srv.page_places(table[b], 64, Kp.shape[0])[:start[b] + z - a], device="cuda")
        score = torch.randperm(start[b] + z - a, generator=torch.Generator().manual_seed(b))
        for t in range(a, z):
            best = at[int(score[:start[b] + t - a + 1].argmax())]
            for h in range(4):
                v = Vp[best[0], h // 2, best[1]].float()
                assert bool(((got[h, t] - v).abs() <= 3 * U * v.abs() + 2.0**-127).all()), (b, t, h)
