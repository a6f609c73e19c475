"""The 4-bit key/value cache on the GPU: codes and values exactly, the decode step
against float64 over the values the codes stand for."""
import numpy as np
import pytest

from gpu_common import desc_of, say, spec_of, torch
from oracle import decode as o_dec
from oracle import geometry as o_geo
from oracle import serve as o_srv
from serve_common import attn_bar, bounds, head_view, need_serve, replay_checked

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rows(Hkv, T, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(Hkv, T, D, generator=g) * 10.0 ** torch.randint(-3, 3, (Hkv, T, 1), generator=g)).to(dtype).cuda()
            for _ in range(2)]


def same_codes(got, want):
    """Equal but for the sign of a zero, which the value does not show."""
    a, b = o_srv.unpack(got.cpu().numpy()), want
    return bool(((a == b) | ((a & 7 == 0) & (b & 7 == 0))).all())


def test_every_bf16_value_is_quantised_as_defined():
    """Blocks whose first element sets the scale, with every bf16 magnitude below
    it from a few binades in turn; the ends of the exponent range among the scales."""
    serve = need_serve()
    def bits(x):
        return torch.tensor(x, dtype=torch.float32).to(BF16).view(torch.int16).item()
    parts = []
    for top in (7.0, 3.515625, 4.5, 7 * 2.0**-100, 5 * 2.0**100, 3.3e38, 2.0**-120, 1e-38, 9e-41):
        hi = bits(top)
        low = torch.arange(max(0, hi - 31 * 24), hi + 1, dtype=torch.int16)
        low = torch.cat([low, low.new_zeros(-len(low) % 31)]).view(-1, 31)
        block = torch.cat([torch.full((len(low), 1), hi, dtype=torch.int16), low], 1)
        parts += [block, block | torch.tensor(-32768, dtype=torch.int16)]
    x = torch.cat(parts)
    x = torch.cat([x, x.new_zeros(len(x) % 2, 32)]).view(BF16).view(1, -1, 64).cuda()
    T = x.shape[1]
    cache = serve.kv4_cache(1, 1, T, 64)
    serve.kv4_store(x, x.flip(1).contiguous(), bounds([T]), *cache)
    codes, scales = o_srv.quantise(x.double().cpu().numpy())
    assert np.array_equal(cache[2][0, :, :, 0].cpu().numpy(), scales)
    assert np.array_equal(cache[2][0, :, :, 1].cpu().numpy(), scales[:, ::-1])
    assert same_codes(cache[0][0], codes) and same_codes(cache[1][0], codes[:, ::-1])


def test_float32_values_next_to_every_border():
    serve = need_serve()
    edge = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], np.float32)
    near = np.concatenate([edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(9))])
    x = np.zeros((1, 40, 64), np.float32)
    for t in range(40):
        for h in (0, 32):
            x[0, t, h] = 7.0 if t % 2 else np.nextafter(np.float32(7), np.float32(8))
            x[0, t, h + 1:h + 28] = near * np.float32(1 if t % 2 else 2) * np.float32((-1) ** (t // 2))
        x[0, t] *= np.float32(2.0 ** (6 * t - 120))
    xd = torch.tensor(x, device="cuda")
    cache = serve.kv4_cache(1, 1, 40, 64)
    serve.kv4_store(xd, xd, bounds([40]), *cache)
    codes, scales = o_srv.quantise(x.astype(np.float64))
    assert np.array_equal(cache[2][0, :, :, 0].cpu().numpy(), scales) and same_codes(cache[0][0], codes)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,Hkv", [(64, 3), (128, 2)])
def test_store_and_load(dtype, D, Hkv):
    """Packed rows to their positions and back; rows of the cache that no token goes
    to, and tokens without a place in it, stay as they were."""
    serve = need_serve()
    lens, start, L = [70, 0, 1, 33, 20], [5, 0, 99, 80, -3], 100
    T = sum(lens) + 3
    k, v = rows(Hkv, T, D, dtype, seed=D)
    k[0, 3, 5], k[1, 4, D - 1], v[0, 70, 1], v[1, 72, 0] = float("nan"), float("inf"), float("-inf"), 0.0
    v[0, 75] = 0.0
    buf = torch.zeros(T, 2 * Hkv * D, dtype=dtype, device="cuda")
    vv = head_view(buf, Hkv, Hkv, D).copy_(v)                        # a token-major view
    K4, V4, S = serve.kv4_cache(5, Hkv, L, D)
    for t in (K4, V4, S):
        t.fill_(0xA5)
    serve.kv4_store(k, vv, bounds(lens), K4, V4, S, start=torch.tensor(start, device="cuda"))
    want = [torch.full_like(t, 0xA5) for t in (K4, V4, S)]
    place = []
    at = 0
    for b, (n, p) in enumerate(zip(lens, start)):
        for i in range(n):
            if 0 <= p + i < L:
                place.append((at + i, b, p + i))
        at += n
    for i, x in enumerate((k, v)):
        codes, scales = o_srv.quantise(x.double().cpu().numpy())
        for t, b, p in place:
            want[i][b, :, p] = torch.tensor(o_srv.pack(codes[:, t]), device="cuda")
            want[2][b, :, p, i] = torch.tensor(scales[:, t], device="cuda")
    assert torch.equal(S, want[2])
    for got, w in ((K4, want[0]), (V4, want[1])):
        assert same_codes(got, o_srv.unpack(w.cpu().numpy()))
    # back, into strided rows of either type
    for back in (BF16, F32):
        kr = torch.full((Hkv, T, D), 3.0, dtype=back, device="cuda")
        vr = head_view(torch.full((T, Hkv * D + 8), 3.0, dtype=back, device="cuda"), 0, Hkv, D)
        serve.kv4_load(K4, V4, S, bounds(lens), kr, vr, start=torch.tensor(start, device="cuda"))
        for got, x in ((kr, k), (vr, v)):
            val = torch.tensor(o_srv.values(*o_srv.quantise(x.double().cpu().numpy())))
            ref = torch.full((Hkv, T, D), 3.0, dtype=torch.float64)
            for t, _, _ in place:
                ref[:, t] = val[:, t]
            assert torch.equal(got.double().cpu().nan_to_num(nan=-1e9), ref.nan_to_num(nan=-1e9))


def test_cache_positions_count_from_the_clipped_offset():
    serve = need_serve()
    k, v = rows(2, 50, 64, BF16, seed=4)
    far = torch.tensor([-9, 20, 1 << 40], device="cuda")
    want, got = serve.kv4_cache(2, 2, 40, 64), serve.kv4_cache(2, 2, 40, 64)
    serve.kv4_store(k, v, bounds([20, 30]), *want)
    serve.kv4_store(k, v, far, *got)
    back = [[torch.zeros_like(k), torch.zeros_like(v)] for _ in range(2)]
    serve.kv4_load(*want, bounds([20, 30]), *back[0])
    serve.kv4_load(*want, far, *back[1])
    for a, b in zip(got + tuple(back[1]), want + tuple(back[0])):
        assert torch.equal(a, b)


def test_store_of_one_token_a_sequence_and_in_a_graph():
    """A decode step's rows: more sequences than a wave looks at in a step."""
    serve = need_serve()
    B, Hkv, D, L = 150, 2, 128, 50
    k, v = rows(Hkv, B, D, BF16, seed=3)
    cu, pos = torch.arange(B + 1, device="cuda"), torch.arange(B, device="cuda") % L
    cache = serve.kv4_cache(B, Hkv, L, D)
    serve.kv4_store(k, v, cu, *cache, start=pos)
    val = o_srv.values(*o_srv.quantise(k.double().cpu().numpy()))
    for b in (0, 1, 63, 64, 65, 149):
        got = o_srv.values(o_srv.unpack(cache[0][b, :, b % L].cpu().numpy()), cache[2][b, :, b % L, 0].cpu().numpy())
        assert np.array_equal(got, val[:, b])
    assert (cache[2].view(B, Hkv, L, -1).sum((1, 3)) != 0).sum() == B        # one row a sequence
    kr, vr = torch.empty_like(k), torch.empty_like(v)

    def step():
        serve.kv4_store(k, v, cu, *cache, start=pos)
        serve.kv4_load(*cache, cu, kr, vr, start=pos)
    replay_checked(step, [kr, vr], lambda i: (k.mul_(-1.25), pos.copy_((pos + 7) % L)))


def test_cache_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes of codes: its last rows."""
    serve = need_serve()
    B, Hkv, L, D = 3, 1, 1 << 25, 128
    cache = [torch.empty(B, Hkv, L, n, dtype=torch.uint8, device="cuda") for n in (D // 2, D // 2)]
    cache.append(torch.empty(B, Hkv, L, 2, D // 32, dtype=torch.uint8, device="cuda"))
    assert cache[0].numel() > 1 << 32
    k, v = rows(Hkv, 3 * 40, D, BF16, seed=5)
    cu, start = bounds([40] * 3), torch.full((3,), L - 40, device="cuda")
    serve.kv4_store(k, v, cu, *cache, start=start)
    kr, vr = torch.empty_like(k), torch.empty_like(v)
    serve.kv4_load(*cache, cu, kr, vr, start=start)
    assert np.array_equal(kr.double().cpu().numpy(), o_srv.values(*o_srv.quantise(k.double().cpu().numpy())))
    Q = torch.randn(B, 2, D, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    out = step(serve, Q, cache, torch.full((B,), L - 1, device="cuda"), window=40)
    for b in range(B):
        kk, vv = kr[0, 40 * b:40 * b + 40].double(), vr[0, 40 * b:40 * b + 40].double()
        want = torch.softmax(Q[b].double() @ kk.t().contiguous() * D**-0.5, 1) @ vv
        assert ((out[b].double() - want).abs() <= attn_bar(Q[b], kk, vv, 40, D**-0.5, want, BF16, F32)).all()


# ---- decode

def filled(serve, B, Hkv, L, D, seed=0):
    """A cache of random rows and its values [B, Hkv, L, D] in float64."""
    k, v = rows(Hkv, B * L, D, BF16, seed)
    cache = serve.kv4_cache(B, Hkv, L, D)
    serve.kv4_store(k, v, bounds([L] * B), *cache)
    kr, vr = torch.empty_like(k), torch.empty_like(v)
    serve.kv4_load(*cache, bounds([L] * B), kr, vr)
    return cache, *(x.double().view(Hkv, B, L, D).transpose(0, 1).cpu().numpy() for x in (kr, vr))


def step(serve, Q, cache, pos, ptr=None, idx=None, window=0, sink=0, out_dtype=F32, scale=0.0):
    out = torch.full(Q.shape, 5.0, dtype=out_dtype, device="cuda")
    d = serve.kv4_decode_desc(Q, cache[0], out, 0 if idx is None else idx.shape[1], window, sink, scale)
    n = serve.kv4_decode_workspace_bytes(d)
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN wherever it is not written
    serve.kv4_decode_attn(Q, *cache, pos, None if ptr is None else ptr.view(-1), idx, out, ws[:n], d)
    assert (ws[n:] == 0xFF).all()
    return out


def check_step(got, Q, K, V, pos, anchors, window, sink, scale):
    B, Hq, D = Q.shape
    Hkv, L = K.shape[1:3]
    G = Hq // Hkv
    q = Q.double().cpu().numpy()
    worst = 0.0
    for b in range(B):
        t = int(pos[b])
        for g in range(Hkv):
            hs = slice(g * G, (g + 1) * G)
            s = o_dec.step_set(anchors[b][g], t, window, sink) if 0 <= t < L else np.zeros(0, np.int64)
            want = o_dec.decode_attention(q[b, hs], K[b, g], V[b, g], s, scale)
            if len(s) == 0:
                assert (got[b, hs] == 0).all()
                continue
            bar = attn_bar(q[b, hs], K[b, g][s], V[b, g][s], len(s), scale, want, BF16, got.dtype)
            err = np.abs(got[b, hs].double().cpu().numpy() - want)
            worst = max(worst, float((err / bar).max()))
            assert (err <= bar).all(), (b, g)
    say(f"  {worst:.3f} of the bar")


CASES = [
    # Hq, Hkv, D, positions, L, window, sink, ppm (0: no anchor), seeds
    (12, 2, 128, [0, 1, 31, 32, 33, 499], 500, 500, 0, 0, 0),          # every key
    (32, 4, 64, [700, 127, 128, 5], 701, 4096, 0, 0, 0),               # a window wider than the cache
    (8, 8, 64, [400, 3, 250], 512, 0, 0, 20_000, 10),                  # the anchor alone
    (12, 2, 128, [600, 900, 77], 1000, 64, 4, 20_000, 10),             # the Hybrid Anchor
    (6, 1, 128, [300, 10], 400, 33, 16, 0, 0),                         # window and initial tokens
    (4, 4, 128, [300, 0], 301, 0, 0, 0, 0),                            # nothing: zeros
    (7, 1, 64, [511, 512, -1, 1024, 1023], 1024, 1, 1, 10_000, 5),     # positions outside the cache
    (1, 1, 64, [37], 64, 256, 0, 0, 0),
    (16, 2, 128, [2999], 3000, 0, 4, 30_000, 30),
]


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_decode_matches_float64(case, out_dtype):
    serve = need_serve()
    from paper_2607_21927_amd import ris
    Hq, Hkv, D, pos, L, window, sink, ppm, S = case
    say(f"kv4 decode {case} {out_dtype}")
    B = len(pos)
    cache, K, V = filled(serve, B, Hkv, L, D, seed=L)
    Q = torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(L)).to(BF16).cuda()
    ptr = idx = None
    anchors = [[np.zeros(0, np.int64)] * Hkv for _ in pos]
    if ppm:
        sp = spec_of(0, ppm, L, Hkv, S)
        md = desc_of(ris, sp)
        at = [min(max(t - 9, 0), L - 1) for t in pos]                  # frozen nine tokens ago
        stride = max(ris.mask_rows_nnz_bound(md, t, 1) for t in at)
        ptr = torch.empty(B, Hkv + 1, dtype=torch.int64, device="cuda")
        idx = torch.full((B, stride), -1, dtype=torch.int32, device="cuda")
        for b, t in enumerate(at):
            ris.mask_build_rows(md, t, 1, ptr[b], idx[b], col_capacity=stride)
            anchors[b] = [o_geo.row_set(sp, g, t) for g in range(Hkv)]
    got = step(serve, Q, cache, torch.tensor(pos, device="cuda"), ptr, idx, window, sink, out_dtype)
    check_step(got, Q, K, V, pos, anchors, window, sink, D**-0.5)


@pytest.mark.parametrize("B", [1, 40])
def test_decode_long_rows(B):
    """Rows of 30,000 keys and ragged ones, one sequence (many waves a row) and a batch."""
    serve = need_serve()
    say(f"kv4 decode long B={B}")
    Hq, Hkv, D, L = 6, 1, 128, 30_000
    cache, K, V = filled(serve, B, Hkv, L, D, seed=1)
    Q = (torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(2)) * 2).to(BF16).cuda()
    pos = [L - 1 - 701 * b for b in range(B)]
    got = step(serve, Q, cache, torch.tensor(pos, device="cuda"), window=L, scale=0.25)
    check_step(got, Q, K, V, pos, [[np.zeros(0, np.int64)]] * B, L, 0, 0.25)


def test_decode_reads_only_its_set():
    """NaN blocks in rows outside the set do not reach the output; in the set they do."""
    serve = need_serve()
    B, Hq, Hkv, D, L = 2, 6, 2, 128, 300
    cache, K, V = filled(serve, B, Hkv, L, D, seed=4)
    Q = torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(5)).to(BF16).cuda()
    pos = torch.tensor([250, 40], device="cuda")
    clean = step(serve, Q, cache, pos, window=50, sink=2)
    bad = [t.clone() for t in cache]
    bad[2][:, :, 251:] = 255
    bad[2][0, :, 2:201] = 255
    bad[2][1, :, 41:] = 255
    assert torch.equal(step(serve, Q, bad, pos, window=50, sink=2), clean)
    bad[2][0, 0, 230, 1, 2] = 255                # a value block of head group 0
    bad[2][1, 1, 30, 0, 0] = 255                 # a key block
    got = step(serve, Q, bad, pos, window=50, sink=2)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[0, :3, 64:96] = True
    hit[1, 3:] = True
    assert torch.equal(got.isnan(), hit) and torch.equal(got[~hit], clean[~hit])
    # a set of nothing beside row 0, which stands in for keys that are none
    bad[2][0, :, 0] = 255
    assert not step(serve, Q, bad, pos, window=20).isnan()[0, :3].any()


def test_decode_anchor_entries_outside_are_ignored():
    serve = need_serve()
    Hkv, D, L = 1, 64, 200
    cache, K, V = filled(serve, 1, Hkv, L, D, seed=6)
    Q = torch.randn(1, 3, D, generator=torch.Generator().manual_seed(7)).to(BF16).cuda()
    idx = torch.tensor([[-5, 3, 7, 120, 150, 199, 200, 1 << 30]], dtype=torch.int32, device="cuda")
    pos = torch.tensor([150], device="cuda")
    for lo, hi in ((0, 8), (-3, 99)):
        got = step(serve, Q, cache, pos, torch.tensor([[lo, hi]], device="cuda"), idx)
        check_step(got, Q, K, V, [150], [[np.array([3, 7, 120, 150])]], 0, 0, D**-0.5)
    assert (step(serve, Q, cache, pos, torch.tensor([[6, 2]], device="cuda"), idx) == 0).all()


def test_decode_in_a_graph():
    serve = need_serve()
    B, Hq, Hkv, D, L = 3, 12, 2, 128, 4000
    cache, K, V = filled(serve, B, Hkv, L, D, seed=8)
    Q = torch.randn(B, Hq, D, generator=torch.Generator().manual_seed(9)).to(BF16).cuda()
    pos = torch.tensor([3000, 17, 3999], device="cuda")
    out = torch.empty(B, Hq, D, dtype=BF16, device="cuda")
    d = serve.kv4_decode_desc(Q, cache[0], out, window=L)
    ws = torch.empty(serve.kv4_decode_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    replay_checked(lambda: serve.kv4_decode_attn(Q, *cache, pos, None, None, out, ws, d), [out],
                   lambda i: (Q.mul_(-1.1), pos.copy_((pos + 777) % L)))
