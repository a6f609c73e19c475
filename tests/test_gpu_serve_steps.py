"""Token steps over the 4-bit cache: what they refuse, and the Hybrid Anchor's set
against float64.  Bars as in ``test_gpu_serve_model``."""
import numpy as np
import pytest

from gpu_common import desc_of, say, spec_of, torch
from oracle import decode as o_dec
from oracle import geometry as o_geo
from serve_common import bounds, need_serve
from test_gpu_serve_model import oracle_step, setup

pytestmark = pytest.mark.gpu


def test_a_refused_step_leaves_the_cache():
    """The step reads bf16 queries alone; the cache takes float32 rows."""
    need_serve()
    from paper_2607_21927_amd import ris
    lens = [9, 4]
    cfg, W, ids, rd, model = setup("tiny_qwen2", torch.float32, lens)
    cache = model.kv4_cache(2, 16)
    model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd, cache=cache)
    before = [[t.clone() for t in layer] for layer in cache.layers]
    with pytest.raises(ris.RisError):
        model.decode_step(torch.tensor([1, 2], device="cuda"), torch.tensor(lens, device="cuda"), cache, rd)
    assert all(torch.equal(a, b) for x, y in zip(before, cache.layers) for a, b in zip(x, y))


@pytest.mark.parametrize("name,window,sink", [("tiny_qwen2", 4, 2), ("tiny_llama", 7, 0)])
def test_anchored_steps_match_float64(name, window, sink):
    serve = need_serve()
    from paper_2607_21927_amd import ris
    lens, L = [60, 45], 64
    cfg, W, ids, rd, model = setup(name, torch.bfloat16, lens)
    cache = model.kv4_cache(2, L)
    model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd, cache=cache)
    tok, pos = torch.tensor([3, 4], device="cuda"), torch.tensor(lens, device="cuda")
    anchors, rows = [], []
    for l in range(cfg.layers):
        sp = spec_of(0, 100_000, L, cfg.kv_heads, 2, layer=l)
        md = desc_of(ris, sp)
        stride = max(ris.mask_rows_nnz_bound(md, n, 1) for n in lens)
        ptr = torch.empty(2, cfg.kv_heads + 1, dtype=torch.int64, device="cuda")
        idx = torch.zeros(2, stride, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lens):
            ris.mask_build_rows(md, n, 1, ptr[b], idx[b], col_capacity=stride)
        anchors.append((ptr.view(-1), idx))
        rows.append([[o_geo.row_set(sp, g, n) for g in range(cfg.kv_heads)] for n in lens])
    h = model.decode_step(tok, pos, cache, rd, anchors=anchors, window=window, sink=sink).double().cpu().numpy()
    for b, n in enumerate(lens):
        caches = []
        for l, (K4, V4, S) in enumerate(cache.layers):
            k, v = (torch.empty(cfg.kv_heads, n + 1, cfg.head_dim, device="cuda") for _ in range(2))
            serve.kv4_load(K4[b:b + 1], V4[b:b + 1], S[b:b + 1], bounds([n + 1]), k, v)
            sets = [o_dec.step_set(rows[l][b][g], n, window, sink) for g in range(cfg.kv_heads)]
            assert max(len(s) for s in sets) < n
            caches.append([[x[g].double().cpu().numpy()[s] for g, s in enumerate(sets)] for x in (k, v)])
        want = oracle_step(int(tok[b]), W, cfg, n, caches)
        bar = 2 * np.sqrt(13 * cfg.layers) * 2.0**-9
        rel = np.linalg.norm(h[b] - want) / np.linalg.norm(want)
        say(f"  sequence {b}: relative {rel:.4f} (bar {bar:.4f})")
        assert rel <= bar


def test_captured_steps():
    """A step captured once and replayed as tokens and positions move on, with eager steps
    over the same cache and a second captured step in between."""
    need_serve()
    lens, L = [30, 5, 17], 64
    cfg, W, ids, rd, model = setup("tiny_qwen2", torch.bfloat16, lens)
    cache = model.kv4_cache(3, L)
    model.prefill_packed(torch.tensor(ids, device="cuda"), bounds(lens), rd, cache=cache)
    tok, pos = torch.tensor([3, 4, 5], device="cuda"), torch.tensor(lens, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        model.decode_step(tok, pos, cache, rd)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(model.decode_step(tok, pos, cache, rd))
    for step in range(4):
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        got = outs[step % 2].clone()
        want = model.decode_step(tok, pos, cache, rd)          # stores the same row again
        torch.cuda.synchronize()
        assert torch.equal(got, want), step
        tok.add_(7).remainder_(cfg.vocab)
        pos.add_(1)
