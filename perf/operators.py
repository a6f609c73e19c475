"""The serving operators, as measurable cases.

Kinds of pass:

rope    rotation of the query and key heads of packed prompts (or of one new token a sequence): positions restart with
        every sequence
prompt  dense attention over packed prompts of different lengths
cache   keys and values of packed prompts (or of one new token a sequence) into the 4-bit cache, and the rows back as
        the values they stand for
decode  one generated token for every sequence of a batch over the 4-bit cache
score   log probabilities of given tokens, entropy and top alternatives from rows of logits

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
BLOCK = 32                                       # dimensions that share a scale in the 4-bit cache
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what the codes 0..7 stand for; 8..15 are their negatives


def _rope(name, shape, B, T, rope, start=0, dtype="bf16", base=1e6, native=32768, factor=2.0):
    c = dict(kind="rope", B=B, T=T, rope=rope, start=start, dtype=dtype, base=base, native=native, factor=factor, **shape)
    return dict(c, name=name) if name else c


def _prompt(name, shape, B, T, dtype="bf16", causal=True):
    c = dict(kind="prompt", B=B, T=T, dtype=dtype, causal=causal, **shape)
    return dict(c, name=name) if name else c


def _cache(name, shape, B, T, max_len, start=0, dtype="bf16"):
    c = dict(kind="cache", B=B, T=T, max_len=max_len, start=start, dtype=dtype, **shape)
    return dict(c, name=name) if name else c


def _decode(name, shape, B, t_max, anchor, window, sink):
    c = dict(kind="decode", B=B, t_max=t_max, anchor=anchor, window=window, sink=sink, **shape)
    return dict(c, name=name) if name else c


def _score(name, rows, vocab, targets, top, dtype="bf16", banned=0.0):
    c = dict(kind="score", rows=rows, vocab=vocab, targets=targets, top=top, dtype=dtype, banned=banned)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step's rotation: one new token for 32 sequences at long positions (latency)
        _rope("rope_step_b32", QWEN2, 32, 32, "yarn", start=40_000),
        # the rotation of a 64k batch of prompts of the Qwen2-1.5B layer, at twice its native window
        _rope("rope_qwen2_64k", QWEN2, 5, 65536, "yarn"),
        # five answer options of a question, a few dozen tokens each (latency)
        _prompt("prompt_options", QWEN2, 5, 437),
        # a serving batch: nine prompts of different lengths, 32k tokens together
        _prompt("prompt_qwen2_32k", QWEN2, 9, 32768),
        # one long document through the TinyLlama-1.1B layer: the dense baseline of the sparse 64k pass
        _prompt("prompt_tinyllama_64k", TINYLLAMA, 1, 65536),
        # prompts in float32, as the paper's own engine computes
        _prompt("prompt_f32_5k", dict(Hq=4, Hkv=2, D=64), 3, 5003, dtype="f32"),
        # a decode step's new tokens into the cache
        _cache("cache_step_b32", QWEN2, 32, 32, 4096, start=3000),
        # a batch of prompts into the cache
        _cache("cache_qwen2_64k", QWEN2, 5, 65536, 40_000),
        # one sequence under the full geometry at 64k: anchor of 70 seeds at 1%, window, initial tokens
        _decode("decode_qwen2_64k_b1", QWEN2, 1, 65536, 0.505, 1024, 4),
        # a batch of long sequences, every key (the dense step)
        _decode("decode_qwen2_64k_b32_dense", QWEN2, 32, 65536, 0.0, 65536, 0),
        # the options of one question at its last token, top alternatives beside them (latency)
        _score("score_options", 1, 151936, 5, 5),
        # every token of a batch of prompts scored
        _score("score_4k_tokens", 4096, 151936, 1, 20),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    kind = rng.choice(["rope", "prompt", "prompt", "prompt", "cache", "decode", "decode", "decode", "score", "score"])
    shape = rng.choice([QWEN2, TINYLLAMA, dict(Hq=16, Hkv=2, D=128), dict(Hq=8, Hkv=8, D=64), dict(Hq=12, Hkv=4, D=64)])
    if kind == "rope":
        B = _log(rng, 1, 64)
        return _rope(None, shape, B, _log(rng, B, 65536), rng.choice(["plain", "linear", "yarn"]),
                     start=rng.choice([0, 0, 30_000]), dtype=rng.choice(["bf16", "bf16", "f32"]), base=rng.choice([1e4, 1e6]),
                     native=rng.choice([2048, 32768]), factor=rng.choice([1.5, 2.0, 8.0]))
    if kind == "prompt":
        f32 = rng.random() < 0.2
        B = _log(rng, 1, 32)
        return _prompt(None, shape, B, _log(rng, max(B, 64), 6000 if f32 else 65536), dtype="f32" if f32 else "bf16",
                       causal=rng.random() < 0.85)
    if kind == "cache":
        B = _log(rng, 1, 64)
        T = _log(rng, B, 65536)
        start = rng.choice([0, 0, 1000])
        return _cache(None, shape, B, T, start + T + rng.randrange(200), start=start, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "decode":
        B, t_max, dense = _log(rng, 1, 48), _log(rng, 1, 65536), rng.random() < 0.4
        return _decode(None, shape, B, t_max, 0.0 if dense else rng.choice([0.01, 0.1, 0.505]),
                       65536 if dense else rng.choice([0, 256, 1024]), 0 if dense else rng.choice([0, 4, 16]))
    return _score(None, _log(rng, 1, 4096), rng.choice([32000, 151936, 50257, _log(rng, 500, 150_000)]),
                  rng.choice([0, 1, 1, 5]), rng.choice([0, 1, 5, 20]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                  banned=rng.choice([0.0, 0.0, 0.3]))


def _size(c):
    """Bytes of the state and of the pass, operations (float32 products run on units 16 times slower)."""
    w = work(c)
    state = w["bytes"]
    if c["kind"] == "cache":
        state = c["B"] * c["Hkv"] * c["max_len"] * c["D"]
    if c["kind"] == "decode":
        state = c["B"] * c["Hkv"] * c["t_max"] * c["D"]
    return [w["bytes"], w["flops"] * (16 if c.get("dtype") == "f32" else 1), state]


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
    """Lengths of the packed sequences, one token at least: the case's own, whatever the seed."""
    B, T = c["B"], c["T"]
    rng = random.Random(T * 1_000_003 + B)
    w = [rng.uniform(0.2, 1.0) for _ in range(B)]
    n = [1 + int((T - B) * x / sum(w)) for x in w]
    n[rng.randrange(B)] += T - sum(n)
    return n


def _positions(c):
    """Position of the newest token of each sequence of a decode step."""
    rng = random.Random(c["t_max"] * 1_000_003 + c["B"])
    return [c["t_max"] - 1 if b == 0 else int((c["t_max"] - 1) * rng.uniform(0.25, 1.0)) for b in range(c["B"])]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(generator=g).to(dtype)


def _bounds(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _ids(v):
    return torch.tensor(v, dtype=torch.int64, device="cuda")


def _heads(buf, first, heads, D):
    """Head-major view [heads, T, D] of head columns of a token-major projection output."""
    return buf[:, first * D:(first + heads) * D].unflatten(1, (heads, D)).transpose(0, 1)


def _outliers(g, D):
    """A few dimensions of a layer's keys are several times the others."""
    s = torch.ones(D, device="cuda")
    s[torch.randint(0, D, (D // 32,), generator=g, device="cuda")] = 4.0
    return s


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(c=c)
    if own:
        from paper_2607_21927_amd import ris, serve
        s["serve"] = serve
    if c["kind"] in ("rope", "prompt", "cache"):
        dt = DTYPES[c["dtype"]]
        s["cu"] = _bounds(_lens(c))
        s["cu_d"] = _ids(s["cu"])
        Hq, Hkv, D, T = c["Hq"], c["Hkv"], c["D"], c["T"]
        # what the projection of a layer gives: token-major, the heads of Q, K and V side by side
        s["qkv"] = _randn(g, T, (Hq + 2 * Hkv) * D, dtype=dt)
    if c["kind"] == "rope":
        s["src"] = _heads(s["qkv"], 0, Hq + Hkv, D)
        s["start"] = [c["start"] + 131 * b for b in range(c["B"])]
        s["start_d"] = _ids(s["start"])
        if own:
            kind = {"plain": ris.ROPE_PLAIN, "linear": ris.ROPE_LINEAR, "yarn": ris.ROPE_YARN}[c["rope"]]
            s["rd"] = ris.rope_desc(kind, c["base"], orig_max_pos=c["native"], factor=c["factor"])
            s["out"] = torch.empty(Hq + Hkv, T, D, dtype=dt, device="cuda")
    elif c["kind"] == "prompt":
        s["q"], s["k"] = (_heads(s["qkv"], a, n, D).contiguous() for a, n in ((0, Hq), (Hq, Hkv)))
        s["v"] = _heads(s["qkv"], Hq + Hkv, Hkv, D)
        if own:
            s["out"] = torch.empty(T, Hq * D, dtype=dt, device="cuda")      # token-major, as the next product reads it
            s["pd"] = serve.prompt_desc(s["q"], s["k"], s["v"], _heads(s["out"], 0, Hq, D), s["cu_d"],
                                        causal=int(c["causal"]))
    elif c["kind"] == "cache":
        s["qkv"][:, Hq * D:(Hq + Hkv) * D] *= _outliers(g, D).repeat(Hkv).to(dt)
        s["k"] = _heads(s["qkv"], Hq, Hkv, D).contiguous()
        s["v"] = _heads(s["qkv"], Hq + Hkv, Hkv, D)
        s["start"] = [min(c["start"] + 7 * b, c["max_len"] - n) for b, n in enumerate(_lens(c))]
        s["start_d"] = _ids(s["start"])
        s["K4"], s["V4"] = (torch.zeros(c["B"], Hkv, c["max_len"], D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
        s["S"] = torch.zeros(c["B"], Hkv, c["max_len"], 2, D // BLOCK, dtype=torch.uint8, device="cuda")
        if own:
            s["kr"], s["vr"] = (torch.empty(Hkv, T, D, dtype=dt, device="cuda") for _ in range(2))
    elif c["kind"] == "decode":
        B, Hq, Hkv, D, L = c["B"], c["Hq"], c["Hkv"], c["D"], c["t_max"] + 16
        s["Q"] = _randn(g, B, Hq, D)
        s["pos"] = _positions(c)
        s["pos_d"] = _ids(s["pos"])
        s["K4"], s["V4"] = (torch.empty(B, Hkv, L, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
        s["S"] = torch.empty(B, Hkv, L, 2, D // BLOCK, dtype=torch.uint8, device="cuda")
        out = _outliers(g, D)
        for b in range(B):
            for i, codes in enumerate((s["K4"], s["V4"])):
                x = _randn(g, Hkv, L, D, dtype=torch.float32)
                codes[b], s["S"][b, :, :, i] = _quantise(x * out if i == 0 else x)
        s["ptr"], s["idx"], s["stride"] = _anchors(c, s["pos"], g)
        if own:
            s["out"] = torch.empty_like(s["Q"])
            s["dd"] = serve.kv4_decode_desc(s["Q"], s["K4"], s["out"], s["stride"], window=c["window"], sink=c["sink"])
            s["ws"] = torch.empty(serve.kv4_decode_workspace_bytes(s["dd"]), dtype=torch.uint8, device="cuda")
    else:
        rows, V, n, k = c["rows"], c["vocab"], c["targets"], c["top"]
        dt = DTYPES[c["dtype"]]
        s["logits"] = torch.empty(rows, V, dtype=dt, device="cuda")
        for r in range(0, rows, 512):
            # most tokens unlikely, a few plausible ones
            x = _randn(g, min(512, rows - r), V, dtype=torch.float32) * 2.5
            x[torch.rand(x.shape, generator=g, device="cuda") < 20.0 / V] += 8.0
            if c["banned"]:
                x[torch.rand(x.shape, generator=g, device="cuda") < c["banned"]] = -math.inf
            s["logits"][r:r + 512] = x.to(dt)
        s["targets"] = torch.randint(0, V, (rows, n), generator=g, device="cuda")
        if own:
            s["logprob"] = torch.empty(rows, n, dtype=torch.float32, device="cuda")
            s["entropy"] = torch.empty(rows, dtype=torch.float32, device="cuda")
            s["ids"] = torch.empty(rows, k, dtype=torch.int64, device="cuda")
            s["top"] = torch.empty(rows, k, dtype=torch.float32, device="cuda")
            s["ld"] = serve.logprob_desc(s["logits"], n, k)
            s["ws"] = torch.empty(serve.logprobs_workspace_bytes(s["ld"]), dtype=torch.uint8, device="cuda")
    return s


def _anchors(c, pos, g):
    """Frozen key sets of the sequences as CSR rows in slices of one size, ascending; each key with the given chance."""
    B, Hkv = c["B"], c["Hkv"]
    ptr = torch.zeros(B, Hkv + 1, dtype=torch.int64, device="cuda")
    if not c["anchor"]:
        return ptr.view(-1), torch.zeros(1, dtype=torch.int32, device="cuda"), 0
    rows = []
    for b, t in enumerate(pos):
        keep = torch.rand(Hkv, max(1, t - 5), generator=g, device="cuda") < c["anchor"]    # frozen a few tokens ago
        ptr[b, 1:] = keep.sum(1).cumsum(0)
        rows.append(keep.nonzero()[:, 1].to(torch.int32))
    # sized by a bound that does not depend on the draw, as a program does
    stride = Hkv * max(1, min(c["t_max"], int(c["t_max"] * c["anchor"] * 1.4) + 64))
    idx = torch.zeros(B, stride, dtype=torch.int32, device="cuda")
    for b, r in enumerate(rows):
        idx[b, :r.numel()] = r
    return ptr.view(-1), idx.view(-1), stride


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    c, serve = s["c"], s["serve"]
    if c["kind"] == "rope":
        return serve.rope_packed(s["src"], s["out"], s["cu_d"], s["rd"], start=s["start_d"])
    if c["kind"] == "prompt":
        out = _heads(s["out"], 0, c["Hq"], c["D"])
        serve.prompt_attn(s["q"], s["k"], s["v"], s["cu_d"], out, s["pd"])
        return s["out"]
    if c["kind"] == "cache":
        serve.kv4_store(s["k"], s["v"], s["cu_d"], s["K4"], s["V4"], s["S"], start=s["start_d"])
        serve.kv4_load(s["K4"], s["V4"], s["S"], s["cu_d"], s["kr"], s["vr"], start=s["start_d"])
        return dict(k=s["kr"], v=s["vr"])
    if c["kind"] == "decode":
        return serve.kv4_decode_attn(s["Q"], s["K4"], s["V4"], s["S"], s["pos_d"], s["ptr"], s["idx"], s["out"], s["ws"],
                                     s["dd"])
    serve.logprobs(s["logits"], s["targets"], s["logprob"], s["entropy"], s["ids"], s["top"], s["ws"], s["ld"])
    return dict(logprob=s["logprob"], entropy=s["entropy"], ids=s["ids"], top=s["top"])


def _run_plain(s):
    c = s["c"]
    if c["kind"] == "rope":
        return _plain_rope(s)
    if c["kind"] == "prompt":
        return _plain_prompt(s)
    if c["kind"] == "cache":
        seq, pos = _token_places(s)
        back = []
        for i, (x, codes) in enumerate(((s["k"], s["K4"]), (s["v"], s["V4"]))):
            q, e = _quantise(x.float())
            codes[seq, :, pos], s["S"][seq, :, pos, i] = q.transpose(0, 1), e.transpose(0, 1)
            back.append(_values(codes[seq, :, pos], s["S"][seq, :, pos, i]).transpose(0, 1).to(x.dtype))
        return dict(k=back[0], v=back[1])
    if c["kind"] == "decode":
        return _plain_decode(s)
    return _plain_score(s)


def _frequencies(c):
    """Rotary frequencies (float64) and the factor on cos and sin."""
    D, f = c["D"], c["factor"]
    inv = 1.0 / c["base"] ** (torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    if c["rope"] == "linear":
        return inv / f, 1.0
    if c["rope"] == "yarn":
        def dim(turns):
            return D * math.log(c["native"] / (turns * 2 * math.pi)) / (2 * math.log(c["base"]))
        lo, hi = max(math.floor(dim(32)), 0), min(math.ceil(dim(1)), D - 1)
        t = ((torch.arange(D // 2, dtype=torch.float64, device="cuda") - lo) / (hi - lo if hi != lo else 0.001)).clamp(0, 1)
        return t * inv / f + (1 - t) * inv, 0.1 * math.log(f) + 1 if f > 1 else 1.0
    return inv, 1.0


def _token_places(s):
    """Sequence and position of every packed token."""
    T, cu = s["c"]["T"], s["cu_d"]
    seq = torch.arange(s["c"]["B"], device="cuda").repeat_interleave(cu[1:] - cu[:-1], output_size=T)
    return seq, torch.arange(T, device="cuda") - cu[seq] + s["start_d"][seq]


def _plain_rope(s):
    c = s["c"]
    pos = _token_places(s)[1]
    inv, m = _frequencies(c)
    ang = pos[:, None].double() * inv                # float32 angles of far positions lose the turn's fraction
    cos, sin = (ang.cos() * m).float(), (ang.sin() * m).float()
    x0, x1 = s["src"].float().chunk(2, -1)
    return torch.cat([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).to(s["src"].dtype)


def _plain_prompt(s):
    c = s["c"]
    G, D = c["Hq"] // c["Hkv"], c["D"]
    out = torch.empty(c["T"], c["Hq"], D, dtype=s["q"].dtype, device="cuda")
    for a, b in zip(s["cu"], s["cu"][1:]):
        for g in range(c["Hkv"]):
            k, v = s["k"][g, a:b].float().t().contiguous(), s["v"][g, a:b].float()
            q = s["q"][g * G:(g + 1) * G, a:b].float() * D ** -0.5
            step = max(1, (1 << 29) // (G * (b - a)))               # 2 GB of scores at a time
            for i in range(0, b - a, step):
                n = min(step, b - a - i)
                keys = i + n if c["causal"] else b - a
                x = q[:, i:i + n].reshape(G * n, D) @ k[:, :keys]
                if c["causal"]:
                    late = torch.arange(keys, device="cuda") > torch.arange(i, i + n, device="cuda")[:, None]
                    x.view(G, n, keys).masked_fill_(late, -math.inf)
                x -= x.amax(1, keepdim=True)
                x.exp_()
                o = x @ v[:keys] / x.sum(1, keepdim=True)
                out[a + i:a + i + n, g * G:(g + 1) * G] = o.view(G, n, D).transpose(0, 1).to(out.dtype)
    return out.view(c["T"], -1)


def _quantise(x):
    """Codes [.., D / 2] and scale bytes [.., D / 32] of float32 values: the scale 2^e of 32 dimensions is the least with
    no magnitude above 7 times it, e in [-124, 125]; a magnitude goes to the nearest of E2M1, halfway to the even code, and
    above 6 to 6.  The low half of a byte is the even dimension."""
    b = x.unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))           # m 2^e, m in [0.5, 1)
    e = torch.where(m > 7 / 8, e - 2, e - 3).clamp(-124, 125)    # 7 2^(e - 3) = (7 / 8) 2^e
    e = torch.where(m == 0, -124, e)
    a = torch.ldexp(b.abs(), -e)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(b)).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (e + 127).squeeze(-1).to(torch.uint8)


def _values(codes, scales):
    """float32 values of codes [.., D / 2] and scale bytes [.., D / 32]."""
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device="cuda")
    x = torch.stack([lut[(codes & 15).int()], lut[(codes >> 4).int()]], -1).flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, BLOCK)), scales.int().unsqueeze(-1) - 127).flatten(-2)


def _attended(c, t, anchor):
    """Which of the keys [0, t] a step at position t attends to."""
    keep = torch.zeros(t + 1, dtype=torch.bool, device="cuda")
    keep[anchor.long().clamp(max=t)] = True           # the anchors end before t
    keep[max(0, t - c["window"] + 1):] = c["window"] > 0
    keep[:c["sink"]] = True
    return keep


def _plain_decode(s):
    c = s["c"]
    Hkv, G, D = c["Hkv"], c["Hq"] // c["Hkv"], c["D"]
    out = torch.empty_like(s["Q"])
    ptr = s["ptr"].view(c["B"], Hkv + 1).tolist() if s["stride"] else [[0] * (Hkv + 1)] * c["B"]
    for b, t in enumerate(s["pos"]):
        for g in range(Hkv):
            k = _values(s["K4"][b, g, :t + 1], s["S"][b, g, :t + 1, 0])
            v = _values(s["V4"][b, g, :t + 1], s["S"][b, g, :t + 1, 1])
            x = s["Q"][b, g * G:(g + 1) * G].float() @ k.t() * D ** -0.5
            row = s["idx"][b * s["stride"] + ptr[b][g]:b * s["stride"] + ptr[b][g + 1]]
            keep = _attended(c, t, row)
            x = torch.where(keep, x, -math.inf)
            p = torch.where(keep, (x - x.amax(1, keepdim=True)).exp(), 0.0)
            den = p.sum(1, keepdim=True)
            out[b, g * G:(g + 1) * G] = torch.where(den > 0, p @ v / den, 0.0).to(out.dtype)      # no key: zeros
    return out


def _order(x):
    """int32 that orders float32 values as they compare."""
    i = (x + 0.0).view(torch.int32)                  # -0.0 is 0.0
    return torch.where(i < 0, i ^ 0x7FFFFFFF, i)


def _top(x, k):
    """Ids of the k largest of each row, ties to the lowest id; -1 where a row has fewer tokens above -inf."""
    V = x.shape[1]
    key = _order(x).long() * (1 << 31) + torch.arange(V - 1, -1, -1, device="cuda")
    ids = V - 1 - (key.topk(k, 1).values & ((1 << 31) - 1))
    return torch.where(x.gather(1, ids) > -math.inf, ids, -1)


def _plain_score(s):
    c = s["c"]
    parts = []
    for r in range(0, c["rows"], 512):
        x = s["logits"][r:r + 512].float()
        d = x - x.amax(1, keepdim=True)
        p = d.exp()
        z = p.sum(1, keepdim=True)
        log_z = z.log()
        y = d - log_z
        ent = log_z[:, 0] - torch.where(p > 0, p * d, 0.0).sum(1) / z[:, 0]
        ids = _top(x, c["top"]) if c["top"] else s["targets"][r:r + 512, :0]
        top = torch.where(ids >= 0, y.gather(1, ids.clamp(min=0)), -math.inf)
        parts.append((y.gather(1, s["targets"][r:r + 512]), ent, ids, top))
    return dict(zip(("logprob", "entropy", "ids", "top"), (torch.cat(t) for t in zip(*parts))))


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "rope":
        n = (c["Hq"] + c["Hkv"]) * c["T"] * c["D"]
        return dict(bytes=2.0 * e * n, flops=3.0 * n)
    if c["kind"] == "prompt":
        pairs = sum(n * (n + 1) / 2 if c["causal"] else n * n for n in _lens(c))
        return dict(bytes=2.0 * e * (c["Hq"] + c["Hkv"]) * c["T"] * c["D"], flops=4.0 * c["Hq"] * c["D"] * pairs)
    if c["kind"] == "cache":
        n = 2 * c["Hkv"] * c["T"] * c["D"]
        return dict(bytes=2.0 * n * e + 2.0 * n * (0.5 + 1 / BLOCK), flops=6.0 * n)
    if c["kind"] == "decode":
        keys = nnz = 0.0
        for t in _positions(c):
            near = min(t + 1, c["window"]) + min(c["sink"], max(0, t + 1 - c["window"]))
            keys += near + c["anchor"] * max(0, t + 1 - near)
            nnz += c["anchor"] * max(1, t - 5)
        keys, nnz = keys * c["Hkv"], nnz * c["Hkv"]
        return dict(bytes=2.0 * keys * c["D"] * (0.5 + 1 / BLOCK) + 4 * nnz + 4.0 * c["B"] * c["Hq"] * c["D"],
                    flops=4.0 * c["D"] * (c["Hq"] // c["Hkv"]) * keys)
    return dict(bytes=c["rows"] * (1.0 * e * c["vocab"] + 12 * c["targets"] + 12 * c["top"] + 4), flops=4.0 * c["rows"] * c["vocab"])


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "rope":
        D, f, out = c["D"], c["factor"], []
        freq, m = [], 1.0
        for i in range(D // 2):
            w = c["base"] ** (-2.0 * i / D)
            if c["rope"] == "linear":
                w /= f
            if c["rope"] == "yarn":
                m = 1.0 + 0.1 * math.log(f)
                edge = [D * math.log(c["native"] / (2 * math.pi * turns)) / (2 * math.log(c["base"])) for turns in (32, 1)]
                lo, hi = max(0, math.floor(edge[0])), min(D - 1, math.ceil(edge[1]))
                ramp = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001)))
                w = w * (1 - ramp) + w / f * ramp
            freq.append(w)
        freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
        for a, b, p in zip(s["cu"], s["cu"][1:], s["start"]):
            turn = torch.polar(torch.full((), m, dtype=torch.float64, device="cuda"),
                               torch.arange(p, p + b - a, dtype=torch.float64, device="cuda")[:, None] * freq)
            x = s["src"][:, a:b].double()
            y = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn
            out.append(torch.cat([y.real, y.imag], -1))
        return torch.cat(out, 1)
    if c["kind"] == "prompt":
        out = torch.zeros(c["T"], c["Hq"] * c["D"], dtype=torch.float64, device="cuda")
        for a, b in zip(s["cu"], s["cu"][1:]):
            for h in range(c["Hq"]):
                k, v = (s[x][h * c["Hkv"] // c["Hq"], a:b].double() for x in "kv")
                for i in range(a, b, 4096):
                    e = min(b, i + 4096)
                    w = s["q"][h, i:e].double() @ k.t().contiguous() / math.sqrt(c["D"])
                    if c["causal"]:
                        w += torch.full_like(w, -math.inf).triu(1 + i - a)
                    out[i:e, h * c["D"]:(h + 1) * c["D"]] = w.softmax(1) @ v
        return out
    if c["kind"] == "cache":
        out = {}
        for x in "kv":
            y = s[x].double().reshape(c["Hkv"], c["T"], -1, BLOCK)
            top = y.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(top / 7)).clamp(-124, 125)
            e = torch.where(7 * 2.0 ** (e - 1) >= top, e - 1, torch.where(7 * 2.0 ** e < top, e + 1, e)).clamp(-124, 125)
            grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
            a = (y.abs() / 2.0 ** e).clamp(max=6.0)
            up = torch.searchsorted(grid, a.contiguous()).clamp(min=1)
            lo, hi = grid[up - 1], grid[up]
            odd = (up - 1) % 2 == 1
            near = torch.where((a - lo < hi - a) | ((a - lo == hi - a) & ~odd), lo, hi)
            out[x] = (near * 2.0 ** e * torch.sign(y)).reshape(s[x].shape)
        return out
    if c["kind"] == "decode":
        lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64, device="cuda")
        out = torch.zeros(c["B"], c["Hq"], c["D"], dtype=torch.float64, device="cuda")
        G = c["Hq"] // c["Hkv"]
        for b, t in enumerate(s["pos"]):
            for g in range(c["Hkv"]):
                near = torch.arange(max(0, t + 1 - c["window"]), t + 1, device="cuda") if c["window"] else _ids([])
                sets = [near, torch.arange(min(c["sink"], t + 1), device="cuda")]
                if s["stride"]:
                    lo, hi = (int(v) for v in s["ptr"][b * (c["Hkv"] + 1) + g:b * (c["Hkv"] + 1) + g + 2])
                    row = s["idx"][b * s["stride"] + lo:b * s["stride"] + hi].long()
                    sets.append(row[row <= t])
                keys = torch.cat(sets).unique()
                if keys.numel() == 0:
                    continue
                kv = []
                for i, codes in enumerate((s["K4"], s["V4"])):
                    by = codes[b, g, keys].long()
                    sc = 2.0 ** (s["S"][b, g, keys, i].double() - 127)
                    kv.append(torch.stack([lut[by % 16], lut[by // 16]], 2).reshape(len(keys), c["D"])
                              * sc.repeat_interleave(BLOCK, 1))
                w = s["Q"][b, g * G:(g + 1) * G].double() @ kv[0].t().contiguous() / math.sqrt(c["D"])
                out[b, g * G:(g + 1) * G] = w.softmax(1) @ kv[1]
        return out
    out = dict(logprob=[], entropy=[], ids=[], top=[])
    for r in range(0, c["rows"], 128):
        x = s["logits"][r:r + 128].double()
        y = x - x.logsumexp(1, keepdim=True)
        out["logprob"].append(y.gather(1, s["targets"][r:r + 128]))
        out["entropy"].append(-torch.xlogy(y.exp(), y.exp()).sum(1))
        v, ids = x.sort(dim=1, descending=True, stable=True)
        v, ids = v[:, :c["top"]], ids[:, :c["top"]]
        out["ids"].append(torch.where(v == -math.inf, -1, ids))
        out["top"].append(y.gather(1, ids))
    return {k: torch.cat(v) for k, v in out.items()}
