"""Model-level prefill: a LLaMA / Qwen2 decoder stack whose attention is the
RIS hot path.

The paper replaces only the attention of the host model and leaves its
weights and every other layer as they are (Methods, opening of "The RIS
Implementation").  Per layer:

    ris_rmsnorm (fused residual add) -> QKV GEMM -> head-major V
    -> ris_rope_from on Q and K (head-major layout and rotation in one pass)
    -> ris_mask_build (this layer's geometry)
    -> ris_sparse_attn -> O GEMM -> ris_rmsnorm (fused residual add)
    -> gate/up GEMM -> ris_swiglu -> down GEMM

GEMMs are plain library GEMMs (torch.nn.functional.linear on the vendor
BLAS, weights kept [out, in] contiguous: activations times transposed
weights is the layout the library's bf16 GEMMs run fastest in, 13-16% ahead
of pre-transposed [in, out] weights at these shapes); every other step runs
in the library's kernels.  The stack
returns the final normalised hidden states.

Around that pass (``serve``): ``prefill_packed`` runs prompts of different
lengths through the stack at full density, the paper's dense baseline, and can
fill a 4-bit key/value cache; ``decode_step`` generates over that cache; ``score``
and ``score_prompts`` give log probabilities of tokens under the LM head.
``extend`` takes any number of new tokens of each sequence over a cache in pages:
prompts in pieces, drafts, single tokens, or all of them in one batch, with a sliding
window if asked.  With ``weight_bits=4`` the projections are held in 4 bits.
"""
import torch
import torch.nn.functional as F

from . import ris, serve


class PrefillModel:
    """A decoder stack on one GPU.

    cfg: a model configuration with fields hidden, heads, kv_heads, head_dim,
    inter, layers, eps, qkv_bias, vocab.  weights: the dict layout of
    ``synth.model_weights`` (numpy arrays or tensors; linear weights
    [out, in]); they are copied to the device in ``dtype``.  The LM head is
    ``weights["lm_head"]`` [vocab, hidden], or the embedding where the weights tie
    the two.  weight_bits 4: the layers' projections and the LM head are quantised to 4
    bits (``serve.w4_pack``); the embedding, norms and biases stay as they are.
    """

    def __init__(self, cfg, weights, device="cuda", dtype=torch.bfloat16, weight_bits=16):
        if weight_bits not in (4, 16):
            raise ValueError("weight_bits must be 4 or 16")
        self.cfg = cfg
        self.dtype = dtype
        self.device = torch.device(device)

        def t(a):
            return torch.as_tensor(a).to(device=self.device, dtype=dtype).contiguous()

        held = (lambda w: w) if weight_bits == 16 else W4Weight
        self.embed = t(weights["embed"])
        self.lm_head = held(t(weights["lm_head"]) if "lm_head" in weights else self.embed)
        self.layers = []
        for L in weights["layers"]:
            layer = {
                "wqkv": held(torch.cat([t(L["q"]), t(L["k"]), t(L["v"])], 0).contiguous()),   # [(Hq + 2 Hkv) D, hidden]
                "bqkv": torch.cat([t(L["bq"]), t(L["bk"]), t(L["bv"])]) if cfg.qkv_bias else None,
                "wo": held(t(L["o"])),                                                  # [hidden, Hq D]
                "wgu": held(torch.cat([t(L["gate"]), t(L["up"])], 0).contiguous()),    # [2 I, hidden]
                "wd": held(t(L["down"])),                                               # [hidden, I]
                "ln1": t(L["ln1"]),
                "ln2": t(L["ln2"]),
            }
            self.layers.append(layer)
        self.norm = t(weights["norm"])
        self._csr = None

    def _csr_buffers(self, desc):
        cap = ris.mask_nnz_bound(desc)             # the bound does not depend on the layer
        rows = desc.heads * desc.N + 1
        if self._csr is None or self._csr[1].numel() < cap or self._csr[0].numel() != rows:
            self._csr = (torch.empty(rows, dtype=torch.int64, device=self.device),
                         torch.empty(max(cap, 1), dtype=torch.int32, device=self.device))
        return self._csr[0], self._csr[1], cap

    def attention(self, h, layer, l, mask, rope_desc, algo, timers=None):
        cfg = self.cfg
        N, D, Hq, Hkv = h.shape[0], cfg.head_dim, cfg.heads, cfg.kv_heads
        qkv = linear(h, layer["wqkv"], layer["bqkv"])
        v = qkv[:, (Hq + Hkv) * D:].view(N, Hkv, D).transpose(0, 1).contiguous()
        if timers:
            timers.mark("proj")
        # Q and K: head-major layout and rotation in one pass over the
        # projection output (ris_rope_from reads the strided head columns).
        qv = qkv[:, :Hq * D].view(N, Hq, D).transpose(0, 1)
        kv = qkv[:, Hq * D:(Hq + Hkv) * D].view(N, Hkv, D).transpose(0, 1)
        if rope_desc is not None:
            q = ris.rope_from(qv, torch.empty(Hq, N, D, dtype=qkv.dtype, device=qkv.device), rope_desc)
            k = ris.rope_from(kv, torch.empty(Hkv, N, D, dtype=qkv.dtype, device=qkv.device), rope_desc)
        else:
            q, k = qv.contiguous(), kv.contiguous()
        desc = ris.mask_desc(mask["mode"], mask["density_ppm"], N, Hkv, n_seeds=mask["n_seeds"],
                             seed=mask.get("seed", 0), layer=l, block=mask.get("block", 0),
                             window=mask.get("window", 0), anchor=mask.get("anchor", 0))
        row_ptr, col_idx, cap = self._csr_buffers(desc)
        if timers:
            timers.mark("rope")
        ris.mask_build(desc, row_ptr, col_idx, col_capacity=cap)
        if timers:
            timers.mark("geometry")
        out = torch.empty_like(q)
        ris.sparse_attn(q, k, v, row_ptr, col_idx, out,
                        ris.attn_desc(q, k, out, mode=mask["mode"], block=mask.get("block", 0), algo=algo))
        if timers:
            timers.mark("attention")
        a = out.transpose(0, 1).reshape(N, Hq * D)
        return linear(a, layer["wo"])

    def mlp(self, h, layer):
        m = torch.empty(h.shape[0], self.cfg.inter, dtype=self.dtype, device=self.device)
        wgu = layer["wgu"]
        if isinstance(wgu, W4Weight) and wgu.direct(h) and self.cfg.inter % 16 == 0:
            serve.w4_linear(h, *wgu.tiles, m, gated=True)
        else:
            ris.swiglu(linear(h, wgu), m)
        return linear(m, layer["wd"])

    def prefill(self, ids, mask, rope_desc=None, algo=ris.ATTN_AUTO, timers=None):
        """Final hidden states [N, hidden] for token ids (a device int64 tensor).

        mask: geometry parameters {mode, density_ppm, n_seeds[, seed, block,
        window, anchor]}; layer l uses layer index l.  rope_desc: from
        ``ris.rope_desc`` (None: no rotation).  timers: optional object with
        ``mark(name)`` called after each phase (for profiling).
        """
        cfg = self.cfg
        res = self.embed[ids].contiguous()                 # the residual stream
        h = torch.empty_like(res)
        ris.rmsnorm(res, self.layers[0]["ln1"], h, cfg.eps)
        for l, layer in enumerate(self.layers):
            a = self.attention(h, layer, l, mask, rope_desc, algo, timers)
            ris.rmsnorm(a, layer["ln2"], h, cfg.eps, residual=res)
            m = self.mlp(h, layer)
            nxt = self.layers[l + 1]["ln1"] if l + 1 < len(self.layers) else self.norm
            ris.rmsnorm(m, nxt, h, cfg.eps, residual=res)
            if timers:
                timers.mark("proj")
        return h

    # ---- packed prompts, generation over the 4-bit cache, scoring

    def kv4_cache(self, batch, max_len):
        """A 4-bit key/value cache for ``batch`` sequences of up to ``max_len``
        tokens, one (K4, V4, S) per layer."""
        return KV4Cache(self, batch, max_len)

    def _packed_qkv(self, h, layer, cu_seqlens, rope_desc, start):
        """Rotated Q [Hq, T, D] and K [Hkv, T, D], and V as a view of the projection."""
        cfg = self.cfg
        T, D, Hq, Hkv = h.shape[0], cfg.head_dim, cfg.heads, cfg.kv_heads
        qkv = linear(h, layer["wqkv"], layer["bqkv"]).view(T, Hq + 2 * Hkv, D).transpose(0, 1)
        qk = qkv[:Hq + Hkv]
        if rope_desc is not None:
            qk = serve.rope_packed(qk, torch.empty(Hq + Hkv, T, D, dtype=qkv.dtype, device=qkv.device), cu_seqlens,
                                   rope_desc, start=start)
        return qk[:Hq], qk[Hq:], qkv[Hq + Hkv:]

    def _stack(self, ids, attention, timers=None):
        """The decoder stack around ``attention(l, layer, h)`` [T, Hq D]."""
        cfg = self.cfg
        res = self.embed[ids].contiguous()
        h = torch.empty_like(res)
        ris.rmsnorm(res, self.layers[0]["ln1"], h, cfg.eps)
        for l, layer in enumerate(self.layers):
            a = linear(attention(l, layer, h), layer["wo"])
            ris.rmsnorm(a, layer["ln2"], h, cfg.eps, residual=res)
            m = self.mlp(h, layer)
            nxt = self.layers[l + 1]["ln1"] if l + 1 < len(self.layers) else self.norm
            ris.rmsnorm(m, nxt, h, cfg.eps, residual=res)
            if timers:
                timers.mark("proj")
        return h

    def prefill_packed(self, ids, cu_seqlens, rope_desc=None, cache=None, timers=None):
        """Final hidden states [T, hidden] of prompts packed into ``ids`` [T], with
        dense causal attention within each prompt and positions from 0.

        cu_seqlens: device int64 offsets [batch + 1].  rope_desc: as in ``prefill``,
        with the factor given for linear and YaRN.  cache: a ``kv4_cache`` of as
        many sequences, which receives the prompts' keys and values (those of tokens
        from its max_len on are left out).  Rows of tokens outside every prompt hold
        nothing of use.
        """
        cfg = self.cfg
        T, D, Hq = ids.shape[0], cfg.head_dim, cfg.heads

        def attention(l, layer, h):
            q, k, v = self._packed_qkv(h, layer, cu_seqlens, rope_desc, None)
            if timers:
                timers.mark("rope")
            if cache is not None:
                serve.kv4_store(k, v, cu_seqlens, *cache.layers[l])
            a = torch.empty(T, Hq * D, dtype=h.dtype, device=h.device)
            out = a.view(T, Hq, D).transpose(0, 1)
            serve.prompt_attn(q, k, v, cu_seqlens, out, serve.prompt_desc(q, k, v, out, cu_seqlens))
            if timers:
                timers.mark("attention")
            return a

        return self._stack(ids, attention, timers)

    def decode_step(self, ids, pos, cache, rope_desc=None, anchors=None, window=None, sink=0):
        """Final hidden states [batch, hidden] of one new token a sequence: ids
        [batch] at positions pos [batch] (device int64), whose keys and values join
        the cache before the step attends to it; a sequence at max_len or beyond has no
        place there, and its state is of no use.

        window None attends to every token of the cache.  anchors: per layer the
        (anchor_ptr, anchor_idx) that ``ris.mask_build_rows`` wrote for the sequences
        (anchor_idx [batch, stride]), with the local window and initial tokens of the
        Hybrid Anchor.  bf16 models only.
        """
        cfg = self.cfg
        B, D, Hq = ids.shape[0], cfg.head_dim, cfg.heads
        if ids.shape != (cache.batch,) or pos.numel() != B:
            raise ValueError(f"ids and pos must hold one entry for each of the cache's {cache.batch} sequences")

        def attention(l, layer, h):
            q, k, v = self._packed_qkv(h, layer, cache.cu, rope_desc, pos)
            ptr, idx = anchors[l] if anchors is not None else (None, None)
            q = q.transpose(0, 1).contiguous()
            out = torch.empty(B, Hq, D, dtype=h.dtype, device=h.device)
            desc = serve.kv4_decode_desc(q, cache.layers[l][0], out, idx.shape[1] if idx is not None else 0,
                                         window=cache.max_len if window is None else window, sink=sink)
            workspace = cache.workspace(desc)              # refuses what the step cannot do before the cache changes
            serve.kv4_store(k, v, cache.cu, *cache.layers[l], start=pos)
            serve.kv4_decode_attn(q, *cache.layers[l], pos, ptr, idx, out, workspace, desc)
            return out.view(B, Hq * D)

        return self._stack(ids, attention)

    def paged_cache(self, batch, max_len, pages=None, page=64):
        """A cache in pages of ``page`` tokens for ``batch`` sequences of up to ``max_len``
        tokens that share ``pages`` pages (None: as many as all of them can need)."""
        return PagedCache(self, batch, max_len, pages, page)

    def extend(self, ids, cu_seqlens, start, cache, rope_desc=None, window=None, sink=0):
        """Final hidden states [T, hidden] of new tokens ids [T] packed by cu_seqlens
        [batch + 1], the first one of sequence b at position start[b] (device int64):
        their keys and values join the ``paged_cache``, whose table has to name their pages
        (``cache.reserve``), and each token attends to its sequence up to itself, or to
        its last ``window`` tokens and the ``sink`` first ones.  Rows of tokens outside
        every sequence hold nothing of use.  bf16 models only.
        """
        cfg = self.cfg
        T, D, Hq, Hkv = ids.shape[0], cfg.head_dim, cfg.heads, cfg.kv_heads
        if cu_seqlens.numel() != cache.batch + 1 or start.numel() != cache.batch:
            raise ValueError(f"cu_seqlens and start must be those of the cache's {cache.batch} sequences")

        def attention(l, layer, h):
            qkv = linear(h, layer["wqkv"], layer["bqkv"]).view(T, Hq + 2 * Hkv, D).transpose(0, 1)
            q, k, v = qkv[:Hq], qkv[Hq:Hq + Hkv], qkv[Hq + Hkv:]
            a = torch.empty(T, Hq * D, dtype=h.dtype, device=h.device)
            out = a.view(T, Hq, D).transpose(0, 1)
            Kp, Vp = cache.layers[l]
            desc = serve.page_attn_desc(q, Kp, cache.table, cu_seqlens, out, window=window, sink=sink)
            # refuses what the step cannot do before the cache changes
            workspace = torch.empty(serve.page_attn_workspace_bytes(desc), dtype=torch.uint8, device=h.device)
            turned = dict(q=q, q_out=q) if rope_desc is not None else {}
            serve.page_store(k, v, cu_seqlens, cache.table, Kp, Vp, start=start, rope=rope_desc, **turned)
            serve.page_attn(q, Kp, Vp, cache.table, cu_seqlens, out, workspace, desc, start=start)
            return a

        return self._stack(ids, attention)

    def score(self, h, targets=None, top_k=0, rows=2048):
        """Log probabilities under the LM head at hidden states h [n, hidden]: of
        the tokens ``targets`` [n, m] (negative: padding, 0), with the entropy and
        the ``top_k`` likeliest tokens.  Logits exist for ``rows`` states at a time.
        Returns dict(logprob [n, m], entropy [n], top_ids, top_logprob [n, top_k])."""
        n, m = h.shape[0], 0 if targets is None else targets.shape[1]
        out = dict(logprob=torch.empty(n, m, dtype=torch.float32, device=h.device),
                   entropy=torch.empty(n, dtype=torch.float32, device=h.device),
                   top_ids=torch.empty(n, top_k, dtype=torch.int64, device=h.device),
                   top_logprob=torch.empty(n, top_k, dtype=torch.float32, device=h.device))
        if targets is not None:
            targets = targets.contiguous()
        for r in range(0, n, rows):
            logits = linear(h[r:r + rows], self.lm_head)
            desc = serve.logprob_desc(logits, m, top_k)
            ws = torch.empty(serve.logprobs_workspace_bytes(desc), dtype=torch.uint8, device=h.device)
            serve.logprobs(logits, targets[r:r + rows] if m else None, *(out[x][r:r + rows] for x in (
                "logprob", "entropy", "top_ids", "top_logprob")), ws, desc)
        return out

    def score_prompts(self, ids, cu_seqlens, rope_desc=None, top_k=0):
        """``score`` of every next token of packed prompts: entry t is about the token
        after ids[t] in its prompt; a prompt's last token has none (log probability
        0), so a sum over a prompt's entries is the prompt's log probability."""
        T = ids.shape[0]
        at = torch.arange(1, T + 1, device=ids.device)
        ends = torch.zeros(T + 1, dtype=torch.bool, device=ids.device)
        ends[cu_seqlens.clamp(0, T)] = True        # as the kernels read them
        none = ends[1:] | (at <= cu_seqlens[0]) | (at > cu_seqlens[-1])
        targets = torch.where(none, -1, ids.roll(-1))
        return self.score(self.prefill_packed(ids, cu_seqlens, rope_desc), targets[:, None], top_k)


def linear(x, w, bias=None):
    """x W^T + bias for rows x and a weight [out, in], held in 16 or 32 bits or as a ``W4Weight``."""
    return w(x, bias) if isinstance(w, W4Weight) else F.linear(x, w, bias)


class W4Weight:
    """A weight matrix held in 4 bits (codes and scales of ``serve.w4_weight``)."""

    # Rows up to which the product reads the 4-bit weights itself.  For more they are written out, in every call, for
    # a library product.  By itself, and written out + library, us, bf16: 17,920 outputs of 1,536 inputs, 1,024 rows 65 and
    # 22 + 63, 1,536 101 and 22 + 69, 2,048 141 and 22 + 111; 151,936 of 1,536, 1,024 rows 544 and 189 + 441, 2,048 1,195 and
    # 189 + 746; 1,536 of 8,960, 1,024 45 and 14 + 42, 2,048 78 and 14 + 59; 2,048 of 1,536, 2,048 21 and 6 + 19.  The library
    # draws level between 1,024 and 2,048 rows.  float32 has the same line, though the product by itself takes half
    # as long at every number of rows (17,920 of 1,536, 1,024 rows 168 and 38 + 410, 4,096 720 and 38 + 1,578).
    MOST_ROWS = 1024

    def __init__(self, w):
        if w.shape[1] * w.element_size() % 16:
            raise ValueError("a weight in 4 bits needs rows of inputs that are multiples of 16 bytes")
        self.shape, self.dtype = w.shape, w.dtype
        self.tiles = serve.w4_weight(*w.shape, device=w.device)
        serve.w4_pack(w, *self.tiles)

    def direct(self, x):
        return x.shape[0] <= self.MOST_ROWS

    def values(self):
        """The matrix of the values that it stands for."""
        return serve.w4_load(*self.tiles, torch.empty(self.shape, dtype=self.dtype, device=self.tiles[0].device))

    def __call__(self, x, bias=None):
        if not self.direct(x):
            return F.linear(x, self.values(), bias)
        out = torch.empty(x.shape[0], self.shape[0], dtype=x.dtype, device=x.device)
        return serve.w4_linear(x, *self.tiles, out, bias=bias)


class PagedCache:
    """The layers' pages of a batch of sequences and the block table that names them
    (``PrefillModel.paged_cache``).  Which pages are free is kept on the host."""

    def __init__(self, model, batch, max_len, pages=None, page=64):
        cfg = model.cfg
        self.batch, self.page = batch, page
        self.max_pages = -(-max_len // page)
        pages = batch * self.max_pages if pages is None else pages
        self.layers = [serve.page_cache(pages, cfg.kv_heads, page, cfg.head_dim, model.device) for _ in model.layers]
        self.table = torch.full((batch, self.max_pages), -1, dtype=torch.int32, device=model.device)
        self.free = list(range(pages - 1, -1, -1))
        self.held = [{} for _ in range(batch)]          # of a sequence: entry of the table -> page

    def reserve(self, lens, first=None):
        """Pages for the positions below lens[b] of every sequence b (host integers; those
        that it has stay), but for those before first[b] alone, which a window has left.
        Raises, taking none, where there are not enough."""
        first = [0] * self.batch if first is None else first
        if len(lens) != self.batch or any(not 0 <= n <= self.max_pages * self.page for n in lens):
            raise ValueError(f"lens must hold {self.batch} lengths of at most {self.max_pages * self.page}")
        if len(first) != self.batch or any(f < 0 for f in first):
            raise ValueError(f"first must hold {self.batch} positions")
        need = [[i for i in range(f // self.page, -(-n // self.page)) if i not in held]
                for n, f, held in zip(lens, first, self.held)]
        if sum(map(len, need)) > len(self.free):
            raise RuntimeError(f"{sum(map(len, need))} pages are needed and {len(self.free)} free")
        for b, entries in enumerate(need):
            for i in entries:
                self.held[b][i] = self.free.pop()
            self._write(b, entries, [self.held[b][i] for i in entries])

    def release(self, b, first=0, end=None):
        """Give back the pages of sequence b that hold positions [first, end) alone (end
        None: to the last one): all of them, or those that a window has left."""
        last = self.max_pages if end is None else end // self.page
        entries = [i for i in self.held[b] if -(-first // self.page) <= i < last]
        self.free += [self.held[b].pop(i) for i in entries]
        self._write(b, entries, [-1] * len(entries))

    def _write(self, b, entries, pages):
        if entries:
            at, to = (torch.tensor(v, device=self.table.device) for v in (entries, pages))
            self.table[b, at] = to.to(torch.int32)


class KV4Cache:
    """The layers' 4-bit caches of a batch of sequences (``PrefillModel.kv4_cache``)."""

    def __init__(self, model, batch, max_len):
        cfg = model.cfg
        self.batch, self.max_len = batch, max_len
        self.layers = [serve.kv4_cache(batch, cfg.kv_heads, max_len, cfg.head_dim, model.device) for _ in model.layers]
        self.cu = torch.arange(batch + 1, dtype=torch.int64, device=model.device)   # one token a sequence

    def workspace(self, desc):
        """Device scratch of one decode call, of its own: steps on two streams, or in two
        captured graphs that are replayed side by side, do not meet in it."""
        return torch.empty(serve.kv4_decode_workspace_bytes(desc), dtype=torch.uint8, device=self.cu.device)
