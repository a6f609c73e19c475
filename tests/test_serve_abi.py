"""The serving operators' C ABI (``include/ris_serve.h``) and binding refuse bad
arguments on the host (no GPU needed: every call fails validation before
anything is launched)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def serve():
    from paper_2607_21927_amd import _build, ris, serve as s
    if not os.path.exists(ris.LIB_PATH):
        _build.build()
    s.lib()
    return s


def test_header_binding_and_library_agree(serve):
    from paper_2607_21927_amd import ris
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ris_serve.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(ris_[a-z_0-9]+)\s*\(", text))
    assert declared == set(serve.EXPORTS)
    out = subprocess.run(["nm", "-D", "--defined-only", ris.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert declared <= set(re.findall(r"\sT\s(ris_\w+)", out))
    assert f"#define RIS_MAX_TOP {serve.MAX_TOP}" in text
    assert ris.version() & 0xFFFF >= 5


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "c.c"
    src.write_text('#include "ris_serve.h"\nint main(void) { return sizeof(ris_prompt_desc) == 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-I",
                    os.path.join(ROOT, "include"), str(src)], check=True)


def prompt(serve, **kw):
    d = dict(dtype_in=1, dtype_out=1, Hq=12, Hkv=2, D=128, batch=3, T=1000, causal=1, scale=0.0, q_head=128000,
             q_token=128, k_head=128000, k_token=128, v_head=128, v_token=2048, o_head=128, o_token=1536)
    d.update(kw)
    return serve.PromptDesc(**d)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype_in=4), -3), (dict(dtype_out=-1), -3), (dict(Hq=13), -2), (dict(Hq=0), -1), (dict(Hkv=0), -1),
    (dict(D=96), -5), (dict(D=256), -5), (dict(batch=0), -1), (dict(T=0), -1), (dict(T=2**31), -5), (dict(causal=2), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(q_head=-128), -1),
    (dict(k_token=132), -1), (dict(v_head=4), -1), (dict(o_token=1537), -1),
    (dict(dtype_out=0, o_token=1538), -1), (dict(T=2**31 - 1, Hq=12800, Hkv=100), -5), (dict(o_head=0), -1), (dict(o_token=0), -1),
    (dict(k_token=2**24), -5), (dict(v_token=2**24), -5),
])
def test_prompt_refusals(serve, bad, code):
    assert serve.lib().ris_prompt_attn(P, P, P, P, P, ctypes.byref(prompt(serve, **bad)), None) == code


def test_scales_beyond_the_range_are_refused(serve):
    """scale * log2 e has to be a float32 number."""
    L = serve.lib()
    assert L.ris_prompt_attn(P, P, P, P, P, ctypes.byref(prompt(serve, scale=3e38)), None) == -1
    assert L.ris_kv4_decode_workspace_bytes(ctypes.byref(decode(scale=3e38))) == -1


def test_prompt_null_and_unaligned(serve):
    L, d = serve.lib(), prompt(serve)
    assert L.ris_prompt_attn(P, P, P, P, P, None, None) == -1
    for i in range(5):
        args = [P] * 5
        args[i] = None
        assert L.ris_prompt_attn(*args, ctypes.byref(d), None) == -1
        if i != 3:
            args[i] = ctypes.c_void_p(0x1008)
            assert L.ris_prompt_attn(*args, ctypes.byref(d), None) == -1


def test_rope_packed_refusals(serve):
    from paper_2607_21927_amd import ris
    L, good = serve.lib(), ris.rope_desc(ris.ROPE_YARN, 1e6, orig_max_pos=32768, factor=2.0)

    def call(src=P, hs=512, ts=64, x=P, dtype=1, heads=2, T=8, D=64, cu=P, batch=1, desc=good):
        return L.ris_rope_packed(src, hs, ts, x, dtype, heads, T, D, cu, None, batch,
                                 ctypes.byref(desc) if desc is not None else None, None)
    for kw, code in [(dict(src=None), -1), (dict(x=None), -1), (dict(cu=None), -1), (dict(desc=None), -1),
                     (dict(hs=-1), -1), (dict(ts=-1), -1), (dict(dtype=3), -3), (dict(heads=0), -1), (dict(T=0), -1),
                     (dict(T=2**31), -5), (dict(D=63), -2), (dict(D=1024), -2), (dict(batch=0), -1),
                     (dict(T=2**31 - 1, D=512), -5),
                     (dict(desc=ris.rope_desc(ris.ROPE_YARN, 1e6, orig_max_pos=32768)), -1),       # factor not given
                     (dict(desc=ris.rope_desc(ris.ROPE_LINEAR, 1e6, orig_max_pos=0, factor=2.0)), -1),
                     (dict(desc=ris.rope_desc(7, 1e6, factor=1.0)), -1), (dict(desc=ris.rope_desc(0, 0.5)), -1)]:
        assert call(**kw) == code, kw


def kv4(serve, **kw):
    d = dict(dtype=1, Hkv=2, D=128, batch=3, T=100, max_len=4096, k_head=12800, k_token=128, v_head=128, v_token=2048)
    d.update(kw)
    return serve.Kv4Desc(**d)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -3), (dict(Hkv=0), -1), (dict(D=32), -5), (dict(batch=0), -1), (dict(T=0), -1), (dict(T=2**31), -5),
    (dict(max_len=0), -1), (dict(max_len=2**31 + 1), -1), (dict(k_token=4), -1), (dict(v_head=-8), -1),
    (dict(Hkv=65536), -5),
])
def test_kv4_refusals(serve, bad, code):
    d = kv4(serve, **bad)
    assert serve.lib().ris_kv4_store(P, P, P, None, P, P, P, ctypes.byref(d), None) == code
    assert serve.lib().ris_kv4_load(P, P, P, P, None, P, P, ctypes.byref(d), None) == code


def test_kv4_load_refuses_rows_in_one_place(serve):
    for bad in (dict(k_token=0), dict(v_token=0), dict(k_head=0), dict(v_head=0)):
        assert serve.lib().ris_kv4_load(P, P, P, P, None, P, P, ctypes.byref(kv4(serve, **bad)), None) == -1


def test_kv4_null_and_unaligned(serve):
    L, d = serve.lib(), kv4(serve)
    for i in (0, 1, 2, 4, 5, 6):            # all but start
        args = [P] * 7
        args[i] = None
        assert L.ris_kv4_store(*args, ctypes.byref(d), None) == -1
        if i != 2:
            args[i] = ctypes.c_void_p(0x1004)
            assert L.ris_kv4_store(*args, ctypes.byref(d), None) == -1
    assert L.ris_kv4_store(*[P] * 7, None, None) == -1
    assert L.ris_kv4_load(P, P, P, P, None, P, None, ctypes.byref(d), None) == -1


def decode(**kw):
    from paper_2607_21927_amd import ris
    d = dict(dtype_in=1, dtype_out=0, batch=2, Hq=12, Hkv=2, D=128, max_len=4096, anchor_stride=1000, window=1024, sink=4,
             scale=0.0)
    d.update(kw)
    return ris.DecodeDesc(**d)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype_in=0), -5), (dict(dtype_in=3), -3), (dict(dtype_out=7), -3), (dict(D=96), -5), (dict(Hq=13), -2),
    (dict(Hq=18), -5), (dict(batch=0), -1), (dict(Hkv=0), -1), (dict(max_len=0), -1), (dict(anchor_stride=-1), -1),
    (dict(window=-1), -1), (dict(sink=-2), -1), (dict(scale=-1.0), -1), (dict(batch=40000), -5),
])
def test_kv4_decode_refusals(serve, bad, code):
    d = decode(**bad)
    assert serve.lib().ris_kv4_decode_workspace_bytes(ctypes.byref(d)) == code
    assert serve.lib().ris_kv4_decode_attn(*[P] * 9, 1 << 40, ctypes.byref(d), None) == code


def test_kv4_decode_null_unaligned_and_capacity(serve):
    L, d = serve.lib(), decode()
    need = serve.kv4_decode_workspace_bytes(d)
    assert need > 0 and L.ris_kv4_decode_attn(*[P] * 9, need - 1, ctypes.byref(d), None) == -4
    for i in range(9):
        args = [P] * 9
        args[i] = None
        assert L.ris_kv4_decode_attn(*args, need, ctypes.byref(d), None) == -1
    for i in (0, 1, 2, 3, 8):
        args = [P] * 9
        args[i] = ctypes.c_void_p(0x1004)
        assert L.ris_kv4_decode_attn(*args, need, ctypes.byref(d), None) == -1
    # without an anchor its pointers may be missing: the next check is reached
    args = [P, P, P, P, P, None, None, P, P]
    assert L.ris_kv4_decode_attn(*args, 0, ctypes.byref(decode(anchor_stride=0)), None) == -4


def logprob(serve, **kw):
    d = dict(dtype=1, n_targets=1, top_k=5, rows=4, vocab=1000, row_stride=1000)
    d.update(kw)
    return serve.LogprobDesc(**d)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=5), -3), (dict(n_targets=-1), -1), (dict(n_targets=65537), -1), (dict(top_k=-1), -1), (dict(top_k=65), -1),
    (dict(rows=0), -1), (dict(vocab=0), -1), (dict(vocab=2**31, row_stride=2**31), -1), (dict(row_stride=999), -1),
    (dict(rows=2**32), -5),
])
def test_logprob_refusals(serve, bad, code):
    d = logprob(serve, **bad)
    assert serve.lib().ris_logprobs_workspace_bytes(ctypes.byref(d)) == code
    assert serve.lib().ris_logprobs(*[P] * 7, 1 << 40, ctypes.byref(d), None) == code


def test_logprob_null_unaligned_and_capacity(serve):
    L, d = serve.lib(), logprob(serve, vocab=151936, row_stride=151936)
    need = serve.logprobs_workspace_bytes(d)
    assert need > 0 and L.ris_logprobs(*[P] * 7, need - 1, ctypes.byref(d), None) == -4
    for i in (0, 1, 2, 4, 5, 6):            # all but the entropy
        args = [P] * 7
        args[i] = None
        assert L.ris_logprobs(*args, need, ctypes.byref(d), None) == -1
    for i, at in ((0, 0x1001), (6, 0x1008)):
        args = [P] * 7
        args[i] = ctypes.c_void_p(at)
        assert L.ris_logprobs(*args, need, ctypes.byref(d), None) == -1


def test_binding_refuses_before_any_call(serve):
    """CPU tensors, and shapes, strides and dtypes that do not fit, raise."""
    from paper_2607_21927_amd import ris
    cu = torch.tensor([0, 4])
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    rd = ris.rope_desc(ris.ROPE_PLAIN, 1e4)
    with pytest.raises(ValueError, match="on one GPU"):
        serve.rope_packed(x, torch.empty_like(x), cu, rd)
    with pytest.raises(ValueError, match="on one GPU"):
        serve.prompt_attn(x, x, x, cu, torch.empty_like(x), serve.prompt_desc(x, x, x, x, cu))
    with pytest.raises(ValueError, match="on one GPU"):
        serve.kv4_store(x, x, cu, *serve.kv4_cache(1, 2, 8, 64, "cpu"))
    with pytest.raises(TypeError):
        serve._bounds(cu.int())
    with pytest.raises(ValueError):
        serve._bounds(cu, torch.tensor([0, 0]))
    with pytest.raises(ValueError):
        serve._bounds(torch.tensor([0]))
    with pytest.raises(ValueError, match="16 bytes"):
        serve._rows(torch.zeros(2, 4, 65, dtype=torch.bfloat16)[..., 1:], (2, 4, 64))
    with pytest.raises(ValueError, match="16 bytes"):
        serve._rows(torch.zeros(2, 4, 64)[..., ::2], (2, 4, 32))
    with pytest.raises(ValueError, match="view"):
        serve._rows(x, (2, 5, 64))
    K4, V4, S = serve.kv4_cache(1, 2, 8, 64, "cpu")
    assert serve._need_cache(K4, V4, S, 1, 2, 64) == 8
    for bad in ((K4, V4[:, :, :4], S), (K4, V4, S[..., :1]), (K4[:, :1], V4[:, :1], S)):
        with pytest.raises(ValueError):
            serve._need_cache(*bad, 1, 2, 64)
    with pytest.raises(TypeError):
        serve._need_cache(K4.int(), V4, S, 1, 2, 64)
    with pytest.raises(TypeError):
        serve.logprob_desc(torch.zeros(2, 8, dtype=torch.float16))
    with pytest.raises(ris.RisError):
        serve.logprobs_workspace_bytes(serve.logprob_desc(torch.zeros(2, 8), top_k=65))
    with pytest.raises(ris.RisError):
        serve.kv4_decode_workspace_bytes(decode(D=96))


def test_binding_holds_views_against_the_descriptor(serve):
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    one = torch.zeros(1, 1, 64)                 # any stride of a dimension of one
    assert serve._placed(x, (2, 4, 64), (256, 64, 1)) == x.data_ptr() and serve._placed(one, (1, 1, 64), (0, 0, 1))
    for bad, shape, strides in ((x, (2, 5, 64), (256, 64, 1)), (x, (2, 4, 64), (256, 128, 1)), (one, (1, 1, 64), (64, 64, 0))):
        with pytest.raises(ValueError, match="match the descriptor"):
            serve._placed(bad, shape, strides)
    with pytest.raises(ValueError, match="16 bytes"):
        serve._placed(torch.zeros(2, 4, 65)[..., 1:], (2, 4, 64), (260, 65, 1))
