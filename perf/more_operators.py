"""What a generation step over a paged cache is made of, as measurable cases.

Kinds of pass:

store   keys and values of new tokens into the pages of a cache, keys and queries rotated to their positions on the way
attn    attention of the sequences' new tokens (one, a few, or a long chunk each) over the paged cache, with a sliding
        window and a few first tokens that stay visible
linear  products of a few rows with weights held in 4 bits, with a bias or with the gated activation of both halves

``run`` computes them in plain torch where ``own`` is false, and through ``paper_2607_21927_amd.serve`` where it is true.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# query heads, key/value heads, head dimension of the host models' layers
QWEN2 = dict(Hq=12, Hkv=2, D=128)
TINYLLAMA = dict(Hq=32, Hkv=4, D=64)
EVERY = 1 << 30                                  # a window that leaves out nothing
BLOCK = 32                                       # inputs that share a scale in the 4-bit weights
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what the codes 0..7 stand for; 8..15 are their negatives


def _store(name, shape, B, T, start, page, rope="yarn", base=1e6, native=32768, factor=2.0):
    c = dict(kind="store", B=B, T=T, mix="even", start=start, page=page, rope=rope, base=base, native=native, factor=factor,
             **shape)
    return dict(c, name=name) if name else c


def _attn(name, shape, B, T, start, page, window=EVERY, sink=0, mix="even"):
    c = dict(kind="attn", B=B, T=T, mix=mix, start=start, page=page, window=window, sink=sink, **shape)
    return dict(c, name=name) if name else c


def _linear(name, rows, inputs, outputs, dtype="bf16", bias=False, gated=False):
    c = dict(kind="linear", rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, bias=bias, gated=gated)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a generation step's new tokens: 32 sequences at long positions (latency)
        _store("store_step_b32", QWEN2, 32, 32, 40_000, 64),
        # five prompts of the Qwen2-1.5B layer, 64k tokens together, at twice its native window
        _store("store_qwen2_64k", QWEN2, 5, 65536, 0, 64),
        # one sequence's next token over 33,000 keys (latency)
        _attn("attn_step_b1", QWEN2, 1, 1, 33_000, 64),
        # a batch of long sequences, one token each: every key is read
        _attn("attn_step_b32", QWEN2, 32, 32, 65_000, 64),
        # many TinyLlama sequences that attend to their last 1,024 tokens and first 4 alone, small pages
        _attn("attn_step_window", TINYLLAMA, 48, 48, 16_000, 16, window=1024, sink=4),
        # one sequence's prompt joins 31 that generate: 600 new tokens and one token each
        _attn("attn_mixed", QWEN2, 32, 631, 9_000, 64, mix="one"),
        # a long document in pieces: 2,048 new tokens after 30,000
        _attn("attn_chunk_2k", QWEN2, 1, 2048, 30_000, 64),
        # 16k new tokens in three sequences under a window of 4,096 and four first tokens
        _attn("attn_window_16k", QWEN2, 3, 16_384, 12_000, 256, window=4096, sink=4),
        # one token through a layer's query, key and value projection, with its bias (latency)
        _linear("linear_qkv_1", 1, 1536, 2048, bias=True),
        # 32 tokens through both projections and the activation of a feed-forward block
        _linear("linear_gated_32", 32, 1536, 17920, gated=True),
        # a few tokens through the projection back, in float32
        _linear("linear_down_f32", 5, 8960, 1536, dtype="f32"),
        # 64 tokens against the whole vocabulary
        _linear("linear_vocab_64", 64, 1536, 151936),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    kind = rng.choice(["store", "attn", "attn", "attn", "attn", "linear", "linear"])
    shape = rng.choice([QWEN2, TINYLLAMA, dict(Hq=16, Hkv=2, D=128), dict(Hq=8, Hkv=8, D=64), dict(Hq=15, Hkv=5, D=64)])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    if kind == "store":
        B = _log(rng, 1, 64)
        return _store(None, shape, B, _log(rng, B, 65536), rng.choice([0, 0, 1000, 50_000]), page,
                      rope=rng.choice(["none", "plain", "linear", "yarn"]), base=rng.choice([1e4, 1e6]),
                      native=rng.choice([2048, 32768]), factor=rng.choice([1.5, 2.0, 8.0]))
    if kind == "attn":
        form = rng.choice(["step", "step", "few", "chunk", "one"])
        B = _log(rng, 1, 64)
        T = {"step": B, "few": B * rng.randint(2, 8), "chunk": _log(rng, max(B, 64), 16_384), "one": B - 1 + _log(rng, 2, 4096)}
        window, sink = rng.choice([(EVERY, 0), (EVERY, 0), (rng.choice([128, 1000, 4096]), rng.choice([0, 4, 100]))])
        return _attn(None, shape, B, T[form], rng.choice([0, _log(rng, 1, 65_000)]), page, window, sink,
                     mix="one" if form == "one" else "even")
    inputs, outputs = rng.choice([(1536, 2048), (1536, 1536), (8960, 1536), (2048, 2560), (2048, 2048), (5632, 2048),
                                  (1536, 17920), (2048, 11264), (1536, 151936), (2048, 32000),
                                  (_log(rng, 64, 9000), _log(rng, 64, 20_000))])
    gated = (inputs, outputs) in ((1536, 17920), (2048, 11264)) and rng.random() < 0.7
    return _linear(None, rng.choice([1, 1, _log(rng, 1, 16), _log(rng, 1, 256)]), inputs, outputs,
                   dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), bias=rng.random() < 0.3 and not gated, gated=gated)


def _size(c):
    """Bytes and operations of a pass; of the plain form's scores, every token of a sequence against every place."""
    w = work(c)
    return [w["bytes"], w["flops"], c["B"] * c["Hq"] * max(_lens(c)) * _places(c) if c["kind"] == "attn" else 0]


def draw(rng):
    most = [max(v) for v in zip(*(_size(c) for c in listed()))]
    while True:
        c = _drawn(rng)
        if all(a <= b for a, b in zip(_size(c), most)):
            return c


# ---------------------------------------------------------------------------
# What a program has in hand before the call
# ---------------------------------------------------------------------------
def _lens(c):
    """New tokens of the sequences, one at least: the case's own, whatever the seed."""
    B, T = c["B"], c["T"]
    if c["mix"] == "one":
        return [T - B + 1] + [1] * (B - 1)
    rng = random.Random(T * 1_000_003 + B)
    w = [rng.uniform(0.2, 1.0) for _ in range(B)]
    n = [1 + int((T - B) * x / sum(w)) for x in w]
    n[rng.randrange(B)] += T - sum(n)
    return n


def _starts(c):
    """Tokens that the cache holds before the new ones: up to c["start"], the first sequence's as many."""
    rng = random.Random(c["start"] * 1_000_003 + c["B"])
    return [c["start"] if b == 0 else int(c["start"] * rng.uniform(0.25, 1.0)) for b in range(c["B"])]


def _places(c):
    """Tokens that a row of the block table can name."""
    most = max(a + n for a, n in zip(_starts(c), _lens(c)))
    return (most + c["page"] - 1) // c["page"] * c["page"]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(generator=g).to(dtype)


def _ids(v, dtype=torch.int64):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _heads(buf, first, heads, D):
    """Head-major view [heads, T, D] of head columns of a token-major projection output."""
    return buf[:, first * D:(first + heads) * D].unflatten(1, (heads, D)).transpose(0, 1)


def _table(c, g):
    """Block table [B, pages of a sequence] int32 whose pages lie anywhere among all; -1 behind a sequence's last page."""
    need = [(a + n + c["page"] - 1) // c["page"] for a, n in zip(_starts(c), _lens(c))]
    ids = torch.randperm(sum(need) + 8, generator=g, device="cuda")[:sum(need)].to(torch.int32)
    table = torch.full((c["B"], _places(c) // c["page"]), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(table.shape[1], device="cuda") < _ids(need)[:, None]] = ids
    return table, sum(need) + 8


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(c=c)
    if own:
        from paper_2607_21927_amd import ris, serve
        s["serve"] = serve
    if c["kind"] == "linear":
        rows, K, N, dt = c["rows"], c["inputs"], c["outputs"], DTYPES[c["dtype"]]
        s["x"] = _randn(g, rows, (K + 7) // 8 * 8, dtype=dt)[:, :K]
        s["C"], s["S"] = _lay_out(*_quantise(torch.nn.functional.pad(
            _randn(g, N, K, dtype=torch.float32) * 0.02, (0, -K % 128, 0, -N % 16))))
        s["bias"] = _randn(g, N, dtype=dt) if c["bias"] else None
        s["out"] = torch.empty(rows, N // 2 if c["gated"] else N, dtype=dt, device="cuda")
        return s
    Hq, Hkv, D, T, page = c["Hq"], c["Hkv"], c["D"], c["T"], c["page"]
    s["cu_d"] = torch.nn.functional.pad(_ids(_lens(c)).cumsum(0), (1, 0))
    s["start_d"] = _ids(_starts(c))
    s["table"], pages = _table(c, g)
    # what the projection of a layer gives: token-major, the heads of Q, K and V side by side
    s["qkv"] = _randn(g, T, (Hq + 2 * Hkv) * D)
    s["q"], s["k"], s["v"] = (_heads(s["qkv"], a, n, D) for a, n in ((0, Hq), (Hq, Hkv), (Hq + Hkv, Hkv)))
    if c["kind"] == "store":
        s["Kp"], s["Vp"] = (torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["out"] = torch.empty(T, Hq * D, dtype=torch.bfloat16, device="cuda")
        if own and c["rope"] != "none":
            kind = {"plain": ris.ROPE_PLAIN, "linear": ris.ROPE_LINEAR, "yarn": ris.ROPE_YARN}[c["rope"]]
            s["rd"] = ris.rope_desc(kind, c["base"], orig_max_pos=c["native"], factor=c["factor"])
        return s
    s["Kp"], s["Vp"] = (_randn(g, pages, Hkv, page, D) for _ in range(2))
    # a few dimensions of a layer's keys are several times the others
    s["Kp"][..., torch.randint(0, D, (D // 32,), generator=g, device="cuda")] *= 4.0
    s["out"] = torch.empty(T, Hq * D, dtype=torch.bfloat16, device="cuda")       # token-major, as the next product reads it
    if own:
        s["ad"] = serve.page_attn_desc(s["q"], s["Kp"], s["table"], s["cu_d"], _heads(s["out"], 0, Hq, D),
                                       window=c["window"], sink=c["sink"])
        s["ws"] = torch.empty(serve.page_attn_workspace_bytes(s["ad"]), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    c, serve = s["c"], s["serve"]
    if c["kind"] == "store":
        serve.page_store(s["k"], s["v"], s["cu_d"], s["table"], s["Kp"], s["Vp"], start=s["start_d"], q=s["q"],
                         q_out=_heads(s["out"], 0, c["Hq"], c["D"]), rope=s.get("rd"))
        return dict(q=s["out"], k=s["Kp"], v=s["Vp"])
    if c["kind"] == "attn":
        serve.page_attn(s["q"], s["Kp"], s["Vp"], s["table"], s["cu_d"], _heads(s["out"], 0, c["Hq"], c["D"]), s["ws"],
                        s["ad"], start=s["start_d"])
        return s["out"]
    return serve.w4_linear(s["x"], s["C"], s["S"], s["out"], bias=s["bias"], gated=c["gated"])


def _run_plain(s):
    return dict(store=_plain_store, attn=_plain_attn, linear=_plain_linear)[s["c"]["kind"]](s)


def _frequencies(c):
    """Rotary frequencies (float64) and the factor on cos and sin."""
    D, f = c["D"], c["factor"]
    inv = 1.0 / c["base"] ** (torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    if c["rope"] == "linear":
        return inv / f, 1.0
    if c["rope"] == "yarn":
        lo, hi = (D * math.log(c["native"] / (turns * 2 * math.pi)) / (2 * math.log(c["base"])) for turns in (32, 1))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), D - 1)
        t = ((torch.arange(D // 2, dtype=torch.float64, device="cuda") - lo) / (hi - lo if hi != lo else 0.001)).clamp(0, 1)
        return t * inv / f + (1 - t) * inv, 0.1 * math.log(f) + 1 if f > 1 else 1.0
    return inv, 1.0


def _tokens(s):
    """Sequence and position of every new token."""
    T, cu = s["c"]["T"], s["cu_d"]
    seq = torch.arange(s["c"]["B"], device="cuda").repeat_interleave(cu[1:] - cu[:-1], output_size=T)
    return seq, torch.arange(T, device="cuda") - cu[seq] + s["start_d"][seq]


def _plain_store(s):
    c = s["c"]
    seq, pos = _tokens(s)

    def rotated(x):
        if c["rope"] == "none":
            return x
        inv, m = _frequencies(c)
        ang = pos[:, None].double() * inv            # float32 angles of far positions lose the turn's fraction
        cos, sin = (ang.cos() * m).float(), (ang.sin() * m).float()
        x0, x1 = x.float().chunk(2, -1)
        return torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).to(x.dtype)
    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    s["Kp"][page, :, slot] = rotated(s["k"]).transpose(0, 1)
    s["Vp"][page, :, slot] = s["v"].transpose(0, 1)
    s["out"].copy_(rotated(s["q"]).transpose(0, 1).flatten(1))
    return dict(q=s["out"], k=s["Kp"], v=s["Vp"])


def _plain_attn(s):
    c = s["c"]
    B, Hkv, G, D, T = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"], c["T"]
    seq, pos = _tokens(s)
    at = torch.arange(T, device="cuda") - s["cu_d"][seq]
    most = max(_lens(c))
    # the sequences padded to one length; [B, Hkv, places, D] of the pages, absent ones as page 0
    q = torch.zeros(B, most, Hkv, G, D, device="cuda")
    q[seq, at] = s["q"].transpose(0, 1).unflatten(1, (Hkv, G)).float()
    p = torch.full((B, most), -1, dtype=torch.int64, device="cuda")
    p[seq, at] = pos
    k, v = (s[x][s["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3).float() for x in ("Kp", "Vp"))
    q = (q * D ** -0.5).permute(0, 2, 3, 1, 4).flatten(2, 3)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).unflatten(2, (G, most))
    j, p = torch.arange(k.shape[2], device="cuda"), p[:, :, None]
    out_of_sight = (j > p) | ((j <= p - c["window"]) & (j >= c["sink"]))
    x.masked_fill_(out_of_sight[:, None, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    z = x.sum(-1)
    o = (torch.matmul(x.flatten(2, 3), v).unflatten(2, (G, most)) / z[..., None]).permute(0, 3, 1, 2, 4)
    return o[seq, at].flatten(1).to(s["out"].dtype)


def _quantise(x):
    """Codes [.., K / 2] and scale bytes [.., K / 32] of float32 values: the scale 2^e of 32 inputs is the least with no
    magnitude above 7 times it, e in [-124, 125]; a magnitude goes to the nearest of E2M1, halfway to the even code, and
    above 6 to 6.  The low half of a byte is the even input."""
    b = x.unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))           # m 2^e, m in [0.5, 1)
    e = torch.where(m > 7 / 8, e - 2, e - 3).clamp(-124, 125)    # 7 2^(e - 3) = (7 / 8) 2^e
    e = torch.where(m == 0, -124, e)
    a = torch.ldexp(b.abs(), -e)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(b)).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (e + 127).squeeze(-1).to(torch.uint8)


def _lay_out(codes, scales):
    """Codes [N, K / 2] and scales [N, K / 32] (N a multiple of 16, K of 128) in tiles of 16 outputs x 128 inputs: codes
    [N / 16, K / 128, 4 blocks, 16 outputs, 16 bytes], scales of four tiles side by side [N / 16, K / 512, 4, 16, 4]."""
    codes = codes.view(codes.shape[0] // 16, 16, -1, 4, 16).permute(0, 2, 3, 1, 4).contiguous()
    scales = torch.nn.functional.pad(scales, (0, -scales.shape[1] % 16))
    return codes, scales.view(scales.shape[0] // 16, 16, -1, 4, 4).permute(0, 2, 4, 1, 3).contiguous()


def _weights(s, dtype=torch.float32):
    """[N, K] of the laid-out weights."""
    N, K = s["c"]["outputs"], s["c"]["inputs"]
    codes = s["C"].permute(0, 3, 1, 2, 4).reshape(s["C"].shape[0] * 16, -1)
    scales = s["S"].permute(0, 3, 1, 4, 2).reshape(codes.shape[0], -1)[:, :codes.shape[1] // 16]
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=dtype, device="cuda")
    w = torch.stack([lut[(codes & 15).int()], lut[(codes >> 4).int()]], -1).flatten(1)
    return torch.ldexp(w.unflatten(1, (-1, BLOCK)), scales.int().unsqueeze(-1) - 127).flatten(1)[:N, :K]


def _plain_linear(s):
    y = s["x"].float() @ _weights(s).t()
    if s["bias"] is not None:
        y += s["bias"].float()
    if s["c"]["gated"]:
        gate, up = y.chunk(2, 1)
        y = gate / (1 + (-gate).exp()) * up
    return y.to(s["out"].dtype)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def _seen(c, p):
    """Keys that a token at position p attends to."""
    near = min(p + 1, c["window"])
    return near + min(c["sink"], p + 1 - near)


def work(case):
    c = case
    if c["kind"] == "linear":
        e, out = 4 if c["dtype"] == "f32" else 2, c["outputs"] // (2 if c["gated"] else 1)
        return dict(bytes=c["inputs"] * c["outputs"] * (0.5 + 1 / BLOCK) + e * c["rows"] * (c["inputs"] + out)
                    + e * c["outputs"] * c["bias"], flops=2.0 * c["rows"] * c["inputs"] * c["outputs"])
    if c["kind"] == "store":
        return dict(bytes=4.0 * (c["Hq"] + 2 * c["Hkv"]) * c["T"] * c["D"], flops=3.0 * (c["Hq"] + c["Hkv"]) * c["T"] * c["D"])
    pairs = keys = 0
    for a, n in zip(_starts(c), _lens(c)):
        pairs += sum(_seen(c, p) for p in range(a, a + n))
        first = max(0, a + 1 - c["window"])                    # of the first token's window
        keys += a + n - first + min(c["sink"], first)
    return dict(bytes=4.0 * c["Hkv"] * c["D"] * keys + 4.0 * c["T"] * c["Hq"] * c["D"], flops=4.0 * c["Hq"] * c["D"] * pairs)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "linear":
        lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64, device="cuda")
        cols = []
        for n in range(0, s["C"].shape[0], 256):                # 4,096 outputs at a time
            by = s["C"][n:n + 256].long()                       # tile, chunk, block, output, byte
            w = torch.stack([lut[by % 16], lut[by // 16]], -1).flatten(-2)
            sc = s["S"][n:n + 256].double().permute(0, 1, 4, 2, 3).flatten(1, 2)[:, :by.shape[1]]
            w = (w * 2.0 ** (sc - 127).unsqueeze(-1)).permute(0, 3, 1, 2, 4).flatten(2).flatten(0, 1)
            cols.append(s["x"].double() @ w[:, :c["inputs"]].t().contiguous())
        y = torch.cat(cols, 1)[:, :c["outputs"]]
        if s["bias"] is not None:
            y = y + s["bias"].double()
        half = c["outputs"] // 2
        return y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:] if c["gated"] else y
    lens, starts = _lens(c), _starts(c)
    if c["kind"] == "store":
        D, f, freq, m = c["D"], c["factor"], [], 1.0
        for i in range(D // 2):
            w = c["base"] ** (-2.0 * i / D)
            if c["rope"] == "linear":
                w /= f
            if c["rope"] == "yarn":
                m = 1.0 + 0.1 * math.log(f) if f > 1 else 1.0
                edge = [D * math.log(c["native"] / (2 * math.pi * turns)) / (2 * math.log(c["base"])) for turns in (32, 1)]
                lo, hi = max(0, math.floor(edge[0])), min(D - 1, math.ceil(edge[1]))
                ramp = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001)))
                w = w * (1 - ramp) + w / f * ramp
            freq.append(w if c["rope"] != "none" else 0.0)
        freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
        Kp, Vp, q, a = s["Kp"].double(), s["Vp"].double(), [], 0
        for b, (n, p) in enumerate(zip(lens, starts)):
            turn = torch.polar(torch.full((), m, dtype=torch.float64, device="cuda"),
                               torch.arange(p, p + n, dtype=torch.float64, device="cuda")[:, None] * freq)

            def rotate(x):
                y = torch.complex(x[..., :D // 2].double().contiguous(), x[..., D // 2:].double().contiguous()) * turn
                return torch.cat([y.real, y.imag], -1)
            q.append(rotate(s["q"][:, a:a + n]).transpose(0, 1).flatten(1))
            row = s["table"][b].long().repeat_interleave(c["page"])[p:p + n]
            slot = torch.arange(p, p + n, device="cuda") % c["page"]
            for h in range(c["Hkv"]):
                Kp[row, h, slot] = rotate(s["k"][h, a:a + n])
                Vp[row, h, slot] = s["v"][h, a:a + n].double()
            a += n
        return dict(q=torch.cat(q), k=Kp, v=Vp)
    out = torch.zeros(c["T"], c["Hq"] * c["D"], dtype=torch.float64, device="cuda")
    a = 0
    for b, (n, p) in enumerate(zip(lens, starts)):
        pages = s["table"][b, :(p + n + c["page"] - 1) // c["page"]].long()
        for h in range(c["Hq"]):
            g = h * c["Hkv"] // c["Hq"]
            k, v = (s[x][pages, g].flatten(0, 1)[:p + n].double() for x in ("Kp", "Vp"))
            for i in range(0, n, 4096):
                e = min(n, i + 4096)
                w = s["q"][h, a + i:a + e].double() @ k.t().contiguous() / math.sqrt(c["D"])
                back = torch.arange(p + i, p + e, device="cuda")[:, None] - torch.arange(p + n, device="cuda")
                w[(back < 0) | ((back >= c["window"]) & (torch.arange(p + n, device="cuda") >= c["sink"]))] = -math.inf
                out[a + i:a + e, h * c["D"]:(h + 1) * c["D"]] = w.softmax(1) @ v
        a += n
    return out
