"""The serving path as it is used: packed prompts through a stack, their 4-bit cache,
token steps over it, and the log probabilities of what follows.

Bars for the hidden states as in test_gpu_model.py: 5e-5 in float32; in bf16 a layer
rounds its activations 13 times, each off by at most 2^-8 of the value and by less than
2^-9 in the root mean square, which add in quadrature over the layers; twice that is
allowed."""
import numpy as np
import pytest

from gpu_common import say, torch
from oracle import geometry as o_geo
from oracle import model as o_model
from oracle import rope as o_rope
from oracle import serve as o_srv
from serve_common import bounds, need_serve, replay_checked
from synth import MODELS, model_weights, tokens

pytestmark = pytest.mark.gpu

FACTOR = 2.0


def setup(name, dtype, lens, seed=7):
    from paper_2607_21927_amd import ris
    from paper_2607_21927_amd.model import PrefillModel
    cfg = MODELS[name]
    W = model_weights(cfg, seed=seed)
    rng = np.random.default_rng(seed)
    W["lm_head"] = rng.standard_normal((cfg.vocab, cfg.hidden)).astype(np.float32) * 0.1
    ids = tokens(sum(lens), cfg.vocab, seed=seed + 1)
    rd = ris.rope_desc(ris.ROPE_YARN, cfg.rope_base, orig_max_pos=cfg.native_len, factor=FACTOR)
    return cfg, W, ids, rd, PrefillModel(cfg, W, "cuda", dtype)


def dense(ids, W, cfg):
    spec = o_geo.MaskSpec(mode=0, density_ppm=10**6, seed=0, n_seeds=1, layer=0, N=len(ids), heads=cfg.kv_heads)
    return o_model.prefill(ids, W, cfg, spec, o_rope.YARN, FACTOR)


@pytest.mark.parametrize("name", ["tiny_qwen2", "tiny_llama"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_prompts_equal_each_prompt_alone(name, dtype):
    need_serve()
    lens = [50, 1, 0, 130, 33]
    cfg, W, ids, rd, model = setup(name, dtype, lens)
    say(f"packed prefill {name} {dtype}")
    got = model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd).double().cpu().numpy()
    at = 0
    for n in lens:
        if n:
            want = dense(ids[at:at + n], W, cfg)
            err = np.abs(got[at:at + n] - want).max()
            if dtype == torch.float32:
                assert err <= 5e-5
            else:
                bar = 2 * np.sqrt(13 * cfg.layers) * 2.0**-9
                rel = np.linalg.norm(got[at:at + n] - want) / np.linalg.norm(want)
                say(f"  {n}: max {err:.4f}, relative {rel:.4f} (bar {bar:.4f})")
                assert rel <= bar and err <= bar * np.abs(want).max()
        at += n


def test_scores_of_packed_prompts():
    """score_prompts: next-token log probabilities, entropy and alternatives."""
    need_serve()
    lens = [40, 1, 77]
    cfg, W, ids, rd, model = setup("tiny_qwen2", torch.float32, lens)
    out = model.score_prompts(torch.tensor(ids, device="cuda"), bounds(lens), rd, top_k=4)
    at = 0
    for n in lens:
        h = dense(ids[at:at + n], W, cfg)
        logits = h @ np.asarray(W["lm_head"], np.float64).T
        # hidden states within 5e-5, 256 products with weights of 0.1: logits within
        bar = 5e-5 * 4 * np.abs(W["lm_head"]).sum(1).max()
        for i in range(n):
            nxt = [ids[at + i + 1]] if i + 1 < n else [-1]
            lp, ent, top_ids, top = o_srv.logprobs(logits[i], nxt, 4)
            assert abs(out["logprob"][at + i, 0].item() - lp[0]) <= bar
            assert abs(out["entropy"][at + i].item() - ent) <= bar * 10
            got_ids = out["top_ids"][at + i].cpu().numpy()
            assert np.abs(logits[i][got_ids] - logits[i][top_ids]).max() <= 2 * bar
            np.testing.assert_allclose(out["top_logprob"][at + i].cpu().numpy(), top, atol=2 * bar)
        at += n
    # in chunks of rows, and without targets
    h = model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd)
    part = model.score(h, top_k=4, rows=50)
    assert part["logprob"].shape == (118, 0)
    for key in ("entropy", "top_ids", "top_logprob"):
        a, b = part[key].double(), out[key].double()
        assert (a - b).abs().max() <= (0 if key == "top_ids" else 1e-5)


def test_scores_with_offsets_outside_the_tokens():
    """Offsets are clipped to the tokens, in scoring as in the kernels."""
    need_serve()
    lens = [40, 0, 37]
    _, _, ids, rd, model = setup("tiny_qwen2", torch.float32, lens)
    ids_d = torch.tensor(ids, device="cuda")
    want = model.score_prompts(ids_d, bounds(lens), rd, top_k=2)
    got = model.score_prompts(ids_d, torch.tensor([-3, 40, 40, 10**12], device="cuda"), rd, top_k=2)
    for key in want:
        assert torch.equal(got[key], want[key]), key
    assert want["logprob"][39] == 0 and want["logprob"][76] == 0 and want["logprob"][38] < 0


def oracle_step(tok, W, cfg, pos, caches):
    """One token's final hidden state in float64, over the caches [(K, V)] [Hkv, n, D] of the
    layers, whose last row is the token's own (as the GPU quantised it)."""
    x = np.asarray(W["embed"], np.float64)[tok]
    G, D = cfg.heads // cfg.kv_heads, cfg.head_dim
    for L, (K, V) in zip(W["layers"], caches):
        h = o_model.rmsnorm(x, L["ln1"], cfg.eps)
        q = h @ np.asarray(L["q"], np.float64).T + (L["bq"] if cfg.qkv_bias else 0)
        q = o_rope.apply(q.reshape(cfg.heads, 1, D), o_rope.YARN, cfg.rope_base, pos, FACTOR, cfg.native_len)[:, 0]
        a = np.zeros((cfg.heads, D))
        for i in range(cfg.heads):
            s = K[i // G] @ q[i] * D**-0.5
            w = np.exp(s - s.max())
            a[i] = w @ V[i // G] / w.sum()
        x = x + a.reshape(-1) @ np.asarray(L["o"], np.float64).T
        x = x + o_model.mlp_block(o_model.rmsnorm(x, L["ln2"], cfg.eps), L)
    return o_model.rmsnorm(x, W["norm"], cfg.eps)


@pytest.mark.parametrize("name", ["tiny_qwen2", "tiny_llama"])
def test_prompts_cache_steps_and_scores_together(name):
    """Prompts fill the cache, three steps follow, each against a float64 step over
    the values that the cache holds; the cache's values are the prompts' own keys and
    values to within a step of their codes."""
    serve = need_serve()
    lens, L = [60, 5, 31], 80
    cfg, W, ids, rd, model = setup(name, torch.bfloat16, lens)
    say(f"generation {name}")
    cache = model.kv4_cache(3, L)
    h = model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd, cache=cache)
    last = (bounds(lens)[1:] - 1)
    for step in range(3):
        best = model.score(h[last] if step == 0 else h, top_k=1)
        tok = best["top_ids"][:, 0]
        assert (best["top_logprob"] <= 0).all() and (tok >= 0).all()
        pos = torch.tensor([n + step for n in lens], device="cuda")
        h = model.decode_step(tok, pos, cache, rd)
        for b, n in enumerate(lens):
            rows = n + step + 1
            caches = []
            for K4, V4, S in cache.layers:
                k, v = (torch.empty(cfg.kv_heads, rows, cfg.head_dim, dtype=torch.float32, device="cuda") for _ in range(2))
                serve.kv4_load(K4[b:b + 1], V4[b:b + 1], S[b:b + 1], bounds([rows]), k, v)
                caches.append((k.double().cpu().numpy(), v.double().cpu().numpy()))
            want = oracle_step(int(tok[b]), W, cfg, n + step, caches)
            got = h[b].double().cpu().numpy()
            bar = 2 * np.sqrt(13 * cfg.layers) * 2.0**-9
            rel = np.linalg.norm(got - want) / np.linalg.norm(want)
            say(f"  step {step} sequence {b}: relative {rel:.4f} (bar {bar:.4f})")
            assert rel <= bar
    # layer 0's keys and values of a prompt, from the embeddings alone
    L0 = W["layers"][0]
    x = o_model.rmsnorm(np.asarray(W["embed"], np.float64)[ids[:60]], L0["ln1"], cfg.eps)
    k = torch.empty(cfg.kv_heads, 60, cfg.head_dim, dtype=torch.float32, device="cuda")
    v = torch.empty_like(k)
    K4, V4, S = (t[:1] for t in cache.layers[0])
    serve.kv4_load(K4, V4, S, bounds([60]), k, v)
    for w, bias, got, i in (("k", "bk", k, 0), ("v", "bv", v, 1)):
        y = x @ np.asarray(L0[w], np.float64).T + (L0[bias] if cfg.qkv_bias else 0)
        y = y.reshape(60, cfg.kv_heads, cfg.head_dim).transpose(1, 0, 2)
        if w == "k":
            y = o_rope.apply(y, o_rope.YARN, cfg.rope_base, 0, FACTOR, cfg.native_len)
        step = np.repeat(2.0 ** (S[0, :, :60, i].cpu().numpy().astype(float) - 127), 32, axis=-1)
        # a step of the code, and what three bf16 roundings move the value by
        assert (np.abs(got.cpu().numpy() - y) <= step + 3 * 2.0**-8 * np.abs(y).max()).all()


def test_anchored_steps():
    """decode_step over the Hybrid Anchor of every layer: with every key in the anchor, it
    is the dense step; with some, only they, the window and the initial tokens count."""
    need_serve()
    from paper_2607_21927_amd import ris
    lens, L = [60, 45], 64
    cfg, W, ids, rd, model = setup("tiny_qwen2", torch.bfloat16, lens)
    cache = model.kv4_cache(2, L)
    model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd, cache=cache)
    tok, pos = torch.tensor([3, 4], device="cuda"), torch.tensor(lens, device="cuda")

    def anchors(ppm):
        out = []
        for l in range(cfg.layers):
            md = ris.mask_desc(ris.STOCHASTIC, ppm, L, cfg.kv_heads, n_seeds=2, layer=l)
            stride = max(ris.mask_rows_nnz_bound(md, n, 1) for n in lens)
            ptr = torch.empty(2, cfg.kv_heads + 1, dtype=torch.int64, device="cuda")
            idx = torch.zeros(2, stride, dtype=torch.int32, device="cuda")
            for b, n in enumerate(lens):
                ris.mask_build_rows(md, n, 1, ptr[b], idx[b], col_capacity=stride)
            out.append((ptr.view(-1), idx))
        return out
    dense_h = model.decode_step(tok, pos, cache, rd)
    full = model.decode_step(tok, pos, cache, rd, anchors=anchors(10**6), window=4, sink=2)
    rel = float((full - dense_h).float().norm() / dense_h.float().norm())
    say(f"  all keys in the anchor: relative difference {rel:.2e}")
    assert rel <= 2 * np.sqrt(13 * cfg.layers) * 2.0**-9              # another order of the same sums
    some = model.decode_step(tok, pos, cache, rd, anchors=anchors(100_000), window=4, sink=2)
    assert not torch.equal(some, dense_h) and torch.isfinite(some.float()).all()


def test_steps_in_a_graph():
    """rope, store, decode and scores captured together and replayed as positions advance."""
    serve = need_serve()
    from paper_2607_21927_amd import ris
    B, Hq, Hkv, D, L, V = 4, 12, 2, 128, 600, 5000
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(B, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16).cuda()
    head = (torch.randn(V, Hq * D, generator=g) * 0.02).to(torch.bfloat16).cuda()
    cu, pos = torch.arange(B + 1, device="cuda"), torch.tensor([0, 130, 64, 500], device="cuda")
    cache = serve.kv4_cache(B, Hkv, L, D)
    k, v = (torch.randn(Hkv, B * L, D, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    serve.kv4_store(k, v, bounds([L] * B), *cache)
    rd = ris.rope_desc(ris.ROPE_YARN, 1e6, orig_max_pos=32768, factor=2.0)
    rot = torch.empty(Hq + Hkv, B, D, dtype=torch.bfloat16, device="cuda")
    q, out = (torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dd = serve.kv4_decode_desc(q, cache[0], out, window=L)
    ws = torch.empty(serve.kv4_decode_workspace_bytes(dd), dtype=torch.uint8, device="cuda")
    logits = torch.empty(B, V, dtype=torch.bfloat16, device="cuda")
    ld = serve.logprob_desc(logits, 0, 3)
    ws2 = torch.empty(serve.logprobs_workspace_bytes(ld), dtype=torch.uint8, device="cuda")
    ent, ids, top = torch.empty(B, device="cuda"), torch.empty(B, 3, dtype=torch.int64, device="cuda"), torch.empty(B, 3, device="cuda")

    def step():
        view = qkv.transpose(0, 1)
        serve.rope_packed(view[:Hq + Hkv], rot, cu, rd, start=pos)
        serve.kv4_store(rot[Hq:], view[Hq + Hkv:], cu, *cache, start=pos)
        q.copy_(rot[:Hq].transpose(0, 1))
        serve.kv4_decode_attn(q, *cache, pos, None, None, out, ws, dd)
        torch.mm(out.view(B, Hq * D), head.t(), out=logits)
        serve.logprobs(logits, None, None, ent, ids, top, ws2, ld)
    replay_checked(step, [out, ent, ids, top], lambda i: (pos.add_(1), qkv.mul_(-1.05)))
