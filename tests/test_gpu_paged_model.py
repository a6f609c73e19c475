"""Generation over a cache in pages as it is used: prompts in pieces, several sequences at
different points, a sliding window, weights in 4 bits, steps in a graph.

Bars for bf16 hidden states as in test_gpu_serve_model.py: 13 roundings a layer, each below 2^-9
of the value in the root mean square, in quadrature; twice that is allowed."""
import numpy as np
import pytest

from gpu_common import say, torch
from oracle import geometry as o_geo
from oracle import model as o_model
from oracle import rope as o_rope
from serve_common import bounds, need_serve, replay_checked
from synth import MODELS, model_weights, tokens

pytestmark = pytest.mark.gpu

FACTOR = 2.0


def setup(name, lens, seed=7, **kw):
    from paper_2607_21927_amd import ris
    from paper_2607_21927_amd.model import PrefillModel
    cfg = MODELS[name]
    W = model_weights(cfg, seed=seed)
    W["lm_head"] = np.random.default_rng(seed).standard_normal((cfg.vocab, cfg.hidden)).astype(np.float32) * 0.1
    ids = [tokens(n, cfg.vocab, seed=seed + 1 + i) for i, n in enumerate(lens)]
    rd = ris.rope_desc(ris.ROPE_YARN, cfg.rope_base, orig_max_pos=cfg.native_len, factor=FACTOR)
    return cfg, W, ids, rd, PrefillModel(cfg, W, "cuda", torch.bfloat16, **kw)


def oracle(ids, W, cfg, window=0, sink=0):
    """Dense attention up to each token; under a window, the geometry of local window and first
    tokens with one draw of the smallest density that is its own row's, taken out."""
    spec = o_geo.MaskSpec(mode=0, density_ppm=10**6, seed=0, n_seeds=1, layer=0, N=len(ids), heads=cfg.kv_heads)
    if not window:
        return o_model.prefill(ids, W, cfg, spec, o_rope.YARN, FACTOR)

    def attention(h, L):
        q, k, v = (h @ np.asarray(L[n], np.float64).T + (np.asarray(L["b" + n], np.float64) if cfg.qkv_bias else 0) for n in "qkv")
        q, k, v = (x.reshape(len(ids), -1, cfg.head_dim).transpose(1, 0, 2) for x in (q, k, v))
        q, k = (o_rope.apply(x, o_rope.YARN, cfg.rope_base, 0, FACTOR, cfg.native_len) for x in (q, k))
        G, t = cfg.heads // cfg.kv_heads, np.arange(len(ids))
        keep = (t[None] <= t[:, None]) & ((t[None] > t[:, None] - window) | (t[None] < sink))
        a = np.zeros_like(q)
        for i in range(cfg.heads):
            s = np.where(keep, q[i] @ k[i // G].T * cfg.head_dim**-0.5, -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            a[i] = w @ v[i // G] / w.sum(1, keepdims=True)
        return a.transpose(1, 0, 2).reshape(len(ids), -1) @ np.asarray(L["o"], np.float64).T
    x = np.asarray(W["embed"], np.float64)[ids]
    for L in W["layers"]:
        x = x + attention(o_model.rmsnorm(x, L["ln1"], cfg.eps), L)
        x = x + o_model.mlp_block(o_model.rmsnorm(x, L["ln2"], cfg.eps), L)
    return o_model.rmsnorm(x, W["norm"], cfg.eps)


def held(got, want, cfg, what):
    got = got.double().cpu().numpy()
    bar = 2 * np.sqrt(13 * cfg.layers) * 2.0**-9
    rel, err = np.linalg.norm(got - want) / np.linalg.norm(want), np.abs(got - want).max()
    say(f"  {what}: max {err:.4f}, relative {rel:.4f} (bar {bar:.4f})")
    assert rel <= bar and err <= bar * np.abs(want).max()


def in_pieces(model, cache, ids, rd, cuts, **kw):
    """The sequences' tokens in turns: turn i takes cuts[i][b] tokens of sequence b.  Hidden states
    of every sequence."""
    done, out = [0] * len(ids), [[] for _ in ids]
    for cut in cuts:
        new = [min(n, len(x) - d) for n, x, d in zip(cut, ids, done)]
        cache.reserve([d + n for d, n in zip(done, new)])
        batch = np.concatenate([x[d:d + n] for x, d, n in zip(ids, done, new)])
        h = model.extend(torch.tensor(batch, device="cuda"), bounds(new), torch.tensor(done, device="cuda"), cache, rd, **kw)
        at = 0
        for b, n in enumerate(new):
            out[b].append(h[at:at + n])
            at += n
            done[b] += n
    assert done == [len(x) for x in ids]
    return [torch.cat(h) for h in out]


CUTS = [[70, 1, 0, 5], [1, 1, 64, 1], [0, 100, 2, 60], [200, 200, 200, 200]]


@pytest.mark.parametrize("name,page", [("tiny_qwen2", 64), ("tiny_llama", 16)])
def test_pieces_equal_the_whole(name, page):
    need_serve()
    lens = [130, 120, 71, 66]
    cfg, W, ids, rd, model = setup(name, lens)
    cache = model.paged_cache(4, 256, page=page)
    for b, (h, x) in enumerate(zip(in_pieces(model, cache, ids, rd, CUTS), ids)):
        held(h, oracle(x, W, cfg), cfg, f"{name} sequence {b}")


@pytest.mark.parametrize("name", ["tiny_qwen2", "tiny_llama"])
def test_sliding_window(name):
    """Pages that the window has left are given back and taken by others on the way."""
    need_serve()
    lens, window, sink = [150, 90], 40, 3
    cfg, W, ids, rd, model = setup(name, lens)
    cache = model.paged_cache(2, 256, pages=12, page=16)          # 16 without giving back
    done, out, free = 0, [], []
    for n in (60, 30, 30, 30):
        new = [min(n, len(x) - done) if done < len(x) else 0 for x in ids]
        for b in (0, 1):
            cache.release(b, first=sink, end=max(0, done - window + 1))
        keep = [len(x) if len(x) < done + n else done + n for x in ids]
        free.append(len(cache.free))
        cache.reserve(keep, first=[max(0, done - window + 1)] * 2)
        batch = np.concatenate([x[done:done + m] for x, m in zip(ids, new)])
        h = model.extend(torch.tensor(batch, device="cuda"), bounds(new), torch.tensor([done, done], device="cuda"), cache, rd,
                         window=window, sink=sink)
        out.append(h.split(new))
        done += n
    say(f"  free pages before each turn: {free}")
    for b, x in enumerate(ids):
        held(torch.cat([o[b] for o in out]), oracle(x, W, cfg, window, sink), cfg, f"{name} sequence {b}")


@pytest.mark.parametrize("name", ["tiny_qwen2", "tiny_llama"])
@pytest.mark.parametrize("most", [1024, 16])
def test_weights_in_4_bits(name, most, monkeypatch):
    """The stack on 4-bit weights, few rows and (from 17 on) written out for the library, against
    float64 on the values that they stand for; scores as those values' logits."""
    need_serve()
    from paper_2607_21927_amd.model import W4Weight
    monkeypatch.setattr(W4Weight, "MOST_ROWS", most)
    lens = [300, 40]
    cfg, W, ids, rd, model = setup(name, lens, weight_bits=4)
    cuts = np.cumsum([0, cfg.heads * cfg.head_dim, cfg.kv_heads * cfg.head_dim, cfg.kv_heads * cfg.head_dim])
    for L, layer in zip(W["layers"], model.layers):
        qkv, gu = (layer[n].values().double().cpu().numpy() for n in ("wqkv", "wgu"))
        for n, a, b in zip("qkv", cuts, cuts[1:]):
            assert np.abs(qkv[a:b] - L[n]).max() < 0.02 and not np.array_equal(qkv[a:b], L[n])
            L[n] = qkv[a:b]
        L["gate"], L["up"] = gu[:cfg.inter], gu[cfg.inter:]
        L["o"], L["down"] = (layer[n].values().double().cpu().numpy() for n in ("wo", "wd"))
    cache = model.paged_cache(2, 320)
    for b, (h, x) in enumerate(zip(in_pieces(model, cache, ids, rd, [[280, 30], [1, 1], [5, 1], [14, 8]]), ids)):
        want = oracle(x, W, cfg)
        held(h, want, cfg, f"{name} sequence {b}")
    head = model.lm_head.values().double().cpu()
    for n in (1, 40):
        rows = h[:n].contiguous()
        logits = rows.double().cpu() @ head.t()
        got = model.score(rows, torch.zeros(n, 1, dtype=torch.int64, device="cuda"), top_k=3)
        want = logits.log_softmax(1)
        # logits rounded to bf16: half a step of the largest moves a log probability by twice that at most
        bar = 2 * float(logits.abs().max()) * 2.0**-8
        assert (got["logprob"][:, 0].double().cpu() - want[:, 0]).abs().max() <= bar
        assert (got["top_logprob"][:, 0].double().cpu() - want.max(1).values).abs().max() <= bar


def test_prefill_with_4_bit_weights():
    """The paths that were there take 4-bit weights too."""
    need_serve()
    lens = [50, 33]
    cfg, W, ids, rd, model = setup("tiny_qwen2", lens, weight_bits=4)
    cache = model.paged_cache(2, 64)
    packed = torch.tensor(np.concatenate(ids), device="cuda")
    a = model.prefill_packed(packed, bounds(lens), rd)
    cache.reserve(lens)
    b = model.extend(packed, bounds(lens), torch.zeros(2, dtype=torch.int64, device="cuda"), cache, rd)
    rel = float((a - b).float().norm() / a.float().norm())
    assert rel <= 2 * np.sqrt(13 * cfg.layers) * 2.0**-9                  # another order of the same sums
    old = model.kv4_cache(2, 64)
    model.prefill_packed(packed, bounds(lens), rd, cache=old)
    h = model.decode_step(torch.tensor([1, 2], device="cuda"), torch.tensor(lens, device="cuda"), old, rd)
    assert h.isfinite().all()


def test_pages_are_kept_account_of():
    need_serve()
    _, _, _, _, model = setup("tiny_llama", [1])
    cache = model.paged_cache(3, 100, pages=7, page=16)
    cache.reserve([16, 17, 0])
    table = cache.table.cpu()
    assert table[0, 0] >= 0 and (table[1, :2] >= 0).all() and (table[0, 1:] == -1).all() and (table[2] == -1).all()
    with pytest.raises(RuntimeError):
        cache.reserve([16, 17, 100])
    assert torch.equal(cache.table.cpu(), table) and len(cache.free) == 4
    cache.reserve([40, 17, 32])
    used = cache.table[cache.table >= 0].tolist()
    assert len(used) == len(set(used)) == 7 and not cache.free
    cache.release(0, first=10, end=40)                        # the page of 16 .. 31 alone lies within
    assert len(cache.free) == 1 and cache.table[0].tolist()[1] == -1 and cache.table[0, 2] >= 0
    cache.release(1)
    assert (cache.table[1] == -1).all() and len(cache.free) == 3
    for bad in ([1, 2], [1, 2, 113], [-1, 0, 0]):
        with pytest.raises(ValueError):
            cache.reserve(bad)
    with pytest.raises(ValueError):
        cache.reserve([1, 1, 1], first=[0, -1, 0])
    with pytest.raises(ValueError):
        model.extend(torch.zeros(2, dtype=torch.int64, device="cuda"), bounds([1, 1]), torch.zeros(2, dtype=torch.int64, device="cuda"), cache)


@pytest.mark.parametrize("bits", [16, 4])
def test_token_steps_in_a_graph(bits):
    """Steps of a stack captured twice over one cache and replayed between eager ones."""
    need_serve()
    lens = [60, 5, 31]
    cfg, W, ids, rd, model = setup("tiny_qwen2", lens, weight_bits=bits)
    cache = model.paged_cache(3, 128)
    cache.reserve([100, 100, 100])
    packed = torch.tensor(np.concatenate(ids), device="cuda")
    model.extend(packed, bounds(lens), torch.zeros(3, dtype=torch.int64, device="cuda"), cache, rd)
    tok, pos, one = torch.tensor([3, 4, 5], device="cuda"), torch.tensor(lens, device="cuda"), bounds([1, 1, 1])
    out = torch.zeros(3, cfg.hidden, dtype=torch.bfloat16, device="cuda")
    replay_checked(lambda: out.copy_(model.extend(tok, one, pos, cache, rd)), [out], lambda i: (pos.add_(1), tok.add_(7)))
    best = torch.zeros(3, 2, dtype=torch.int64, device="cuda")

    def step():
        h = model.extend(tok, one, pos, cache, rd, window=20, sink=2)
        best.copy_(model.score(h, top_k=2)["top_ids"])
    replay_checked(step, [best], lambda i: (pos.add_(1), tok.add_(11)))
