"""The paged cache's and the 4-bit weights' entry points and bindings refuse bad arguments on
the host (no GPU needed: every call fails validation before anything is launched)."""
import ctypes
import os

import pytest
import torch

P = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
MAP = dict(page=64, max_pages=100, pages=500, page_stride=2 * 64 * 128, table_stride=100)


@pytest.fixture(scope="module")
def serve():
    from paper_2607_21927_amd import _build, ris, serve as s
    if not os.path.exists(ris.LIB_PATH):
        _build.build()
    s.lib()
    assert ris.version() & 0xFFFF >= 6
    return s


def the_map(serve, kw):
    return serve.PageMap(**{k: kw.pop(k, v) for k, v in MAP.items()})


def store(serve, **kw):
    m = the_map(serve, kw)
    d = dict(dtype=1, Hq=12, Hkv=2, D=128, batch=3, T=100, map=m, q_head=128, q_token=2048, qo_head=128, qo_token=1536,
             k_head=128, k_token=2048, v_head=128, v_token=2048)
    return serve.PageStoreDesc(**{**d, **kw})


def attn(serve, **kw):
    m = the_map(serve, kw)
    d = dict(dtype_in=1, dtype_out=1, Hq=12, Hkv=2, D=128, batch=3, T=100, map=m, window=1000, sink=4, scale=0.0,
             q_head=128, q_token=2048, o_head=128, o_token=1536)
    return serve.PageAttnDesc(**{**d, **kw})


BAD_MAPS = [
    (dict(page=0), -1), (dict(page=48), -1), (dict(page=-64), -1), (dict(page=131072), -1), (dict(max_pages=0), -1),
    (dict(pages=0), -1), (dict(pages=2**31), -1), (dict(table_stride=99), -1), (dict(page_stride=2 * 64 * 128 - 128), -1),
    (dict(page_stride=2 * 64 * 128 + 64), -1), (dict(max_pages=2**25, table_stride=2**25), -5),
    (dict(pages=2**31 - 1), -5), (dict(page_stride=2**62), -5), (dict(table_stride=2**33), -5),
]


@pytest.mark.parametrize("bad,code", BAD_MAPS + [
    (dict(dtype=0), -5), (dict(dtype=2), -3), (dict(Hq=-1), -1), (dict(Hkv=0), -1), (dict(D=96), -5), (dict(batch=0), -1),
    (dict(T=0), -1), (dict(T=2**31), -5), (dict(Hkv=65536), -5), (dict(Hq=65536), -5), (dict(batch=2**25), -5),
    (dict(q_head=4), -1), (dict(q_token=-8), -1), (dict(k_token=132), -1), (dict(v_head=4), -1), (dict(qo_head=0), -1),
    (dict(qo_token=0), -1), (dict(qo_token=1540), -1),
])
def test_store_refusals(serve, bad, code):
    assert serve.lib().ris_page_store(*[P] * 9, ctypes.byref(store(serve, **bad)), None, None) == code


def test_store_null_unaligned_and_rope(serve):
    from paper_2607_21927_amd import ris
    L, d = serve.lib(), store(serve)
    assert L.ris_page_store(*[P] * 9, None, None, None) == -1
    for i in (0, 1, 2, 3, 4, 6, 7, 8):           # all but start
        args = [P] * 9
        args[i] = None
        assert L.ris_page_store(*args, ctypes.byref(d), None, None) == -1
        if i not in (4, 6):
            args[i] = ctypes.c_void_p(0x1008)
            assert L.ris_page_store(*args, ctypes.byref(d), None, None) == -1
    for rd in (ris.rope_desc(ris.ROPE_YARN, 1e6, orig_max_pos=32768), ris.rope_desc(9, 1e6, factor=1.0), ris.rope_desc(0, 0.5)):
        assert L.ris_page_store(*[P] * 9, ctypes.byref(d), ctypes.byref(rd), None) == -1


@pytest.mark.parametrize("bad,code", BAD_MAPS + [
    (dict(dtype_in=0), -5), (dict(dtype_in=7), -3), (dict(dtype_out=2), -3), (dict(Hq=13), -2), (dict(Hq=0), -1),
    (dict(Hkv=0), -1), (dict(Hq=2 * 129), -5), (dict(D=32), -5), (dict(batch=0), -1), (dict(T=0), -1), (dict(T=2**31), -5),
    (dict(window=-1), -1), (dict(sink=-1), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=3e38), -1),
])
def test_attn_refusals(serve, bad, code):
    d = attn(serve, **bad)
    assert serve.lib().ris_page_attn_workspace_bytes(ctypes.byref(d)) == code
    assert serve.lib().ris_page_attn(*[P] * 8, 1 << 40, ctypes.byref(d), None) == code


def test_attn_null_unaligned_and_capacity(serve):
    L, d = serve.lib(), attn(serve)
    need = serve.page_attn_workspace_bytes(d)
    for i in (0, 1, 2, 3, 4, 6):                 # all but start and the workspace
        args = [P] * 8
        args[i] = None
        assert L.ris_page_attn(*args, need, ctypes.byref(d), None) == -1
        if i not in (3, 4):
            args[i] = ctypes.c_void_p(0x1008)
            assert L.ris_page_attn(*args, need, ctypes.byref(d), None) == -1
    assert L.ris_page_attn(*[P] * 8, need, None, None) == -1
    if need:
        assert L.ris_page_attn(*[P] * 8, need - 1, ctypes.byref(d), None) == -4
        assert L.ris_page_attn(*[P] * 7, None, need, ctypes.byref(d), None) == -1
        assert L.ris_page_attn(*[P] * 7, ctypes.c_void_p(0x1008), need, ctypes.byref(d), None) == -1
    for bad in (dict(q_head=4), dict(q_token=-8), dict(o_head=0), dict(o_token=0), dict(o_token=1540)):
        assert L.ris_page_attn(*[P] * 8, 1 << 40, ctypes.byref(attn(serve, **bad)), None) == -1


def linear(serve, **kw):
    d = dict(dtype=1, gated=0, rows=4, N=100, K=256, x_stride=256, out_stride=100)
    return serve.W4Desc(**{**d, **kw})


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), -3), (dict(gated=2), -1), (dict(gated=1), -2), (dict(rows=0), -1), (dict(rows=2**31), -1), (dict(N=0), -1),
    (dict(K=0), -1), (dict(N=2**28 + 1, out_stride=2**29), -5), (dict(K=2**24 + 1, x_stride=2**25), -5), (dict(x_stride=248), -1),
    (dict(x_stride=260), -1), (dict(dtype=0, x_stride=258), -1), (dict(out_stride=99), -1), (dict(out_stride=2**41), -1),
    (dict(rows=2**31 - 1, N=2**20, out_stride=2**20), -5), (dict(N=2**27 + 16, out_stride=2**28), -5),
])
def test_linear_refusals(serve, bad, code):
    assert serve.lib().ris_w4_linear(P, P, P, None, P, ctypes.byref(linear(serve, **bad)), None) == code


def test_linear_null_and_unaligned(serve):
    L, d = serve.lib(), linear(serve)
    assert L.ris_w4_linear(P, P, P, P, P, None, None) == -1
    for i, at in ((0, 0x1008), (1, 0x1008), (2, None), (3, 0x1001), (4, 0x1001)):
        args = [P] * 5
        if i != 3:
            args[i] = None
            assert L.ris_w4_linear(*args, ctypes.byref(d), None) == -1
        if at:
            args[i] = ctypes.c_void_p(at)
            assert L.ris_w4_linear(*args, ctypes.byref(d), None) == -1


@pytest.mark.parametrize("dtype,N,K,stride,code", [(2, 16, 128, 128, -3), (1, 0, 128, 128, -1), (1, 16, 0, 128, -1),
                                                   (1, 16, 128, 127, -1), (1, 2**28 + 1, 128, 128, -5),
                                                   (1, 16, 2**24 + 1, 2**25, -5), (1, 16, 128, 2**41, -1)])
def test_pack_and_load_refusals(serve, dtype, N, K, stride, code):
    L = serve.lib()
    assert L.ris_w4_pack(P, dtype, N, K, stride, P, P, None) == code
    assert L.ris_w4_load(P, P, P, dtype, N, K, stride, None) == code


def test_pack_and_load_null_and_unaligned(serve):
    L = serve.lib()
    for W, C, S in ((None, P, P), (P, None, P), (P, P, None), (ctypes.c_void_p(0x1001), P, P), (P, ctypes.c_void_p(0x1008), P)):
        assert L.ris_w4_pack(W, 1, 16, 128, 128, C, S, None) == -1
        assert L.ris_w4_load(C, S, W, 1, 16, 128, 128, None) == -1


def test_bindings_refuse(serve):
    """CPU tensors, and shapes, strides and dtypes that do not fit, raise."""
    from paper_2607_21927_amd import ris
    cu, q, k = torch.tensor([0, 4]), torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    Kp, Vp = serve.page_cache(3, 2, 16, 64, "cpu")
    table = torch.zeros(1, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="on one GPU"):
        serve.page_store(k, k, cu, table, Kp, Vp)
    desc = serve.page_attn_desc(q, Kp, table, cu, q)
    assert desc.window == 48 and (desc.Hq, desc.Hkv, desc.T, desc.D) == (4, 2, 4, 64)
    with pytest.raises(ValueError, match="on one GPU"):
        serve.page_attn(q, Kp, Vp, table, cu, torch.empty_like(q), None, desc)
    with pytest.raises(TypeError, match="int32"):
        serve._page_map(Kp, table.long())
    with pytest.raises(ValueError, match="unit stride"):
        serve._page_map(Kp, torch.zeros(1, 6, dtype=torch.int32)[:, ::2])
    with pytest.raises(ValueError, match="contiguous"):
        serve._page_map(Kp.transpose(1, 2), table)
    assert serve._page_map(torch.zeros(3, 2, 2, 16, 64)[:, 0], table).page_stride == 2 * 2 * 16 * 64
    # a dimension of one element may have any stride; windows and sinks beyond 32 bits are all of it
    odd = torch.zeros(3, 1, 16, 64).as_strided((3, 1, 16, 64), (1024, 7, 64, 1))
    assert serve._page_map(odd, table).page_stride == 1024
    far = serve.page_attn_desc(q, Kp, table, cu, q, window=2**40, sink=2**40)
    assert far.window == far.sink == 2**31 - 1
    for bad in ((Kp, Vp[:, :1]), (Kp, Vp[:2]), (Kp[0], Vp[0])):
        with pytest.raises(ValueError):
            serve._need_pages(*bad)
    with pytest.raises(TypeError):
        serve._need_pages(Kp.float(), Vp.float())
    with pytest.raises(ris.RisError):
        serve.page_attn_workspace_bytes(serve.page_attn_desc(q, Kp, table, cu, q, sink=-1))
    C, S = serve.w4_weight(40, 300, "cpu")
    assert C.shape == (3, 3, 4, 16, 16) and S.shape == (3, 1, 4, 16, 4)
    x = torch.zeros(2, 300, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on one GPU"):
        serve.w4_linear(x, C, S, torch.zeros(2, 40, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="on one GPU"):
        serve.w4_pack(torch.zeros(40, 300), C, S)
    for bad in ((C, S, 50, 300), (C, S, 40, 400), (C, S, 40, 600), (C[:2], S, 40, 300)):
        with pytest.raises(ValueError):
            serve._need_w4(*bad)
    with pytest.raises(TypeError):
        serve._need_w4(C.int(), S, 40, 300)
    with pytest.raises(ValueError, match="unit stride"):
        serve._matrix(x[:, ::2], 2, 150)
    assert serve._matrix(x[:1, :7], 1, 7) == 7 and serve._matrix(x[:, :7], 2, 7) == 300


def test_model_refuses_weights_without_whole_pieces():
    from paper_2607_21927_amd.model import W4Weight
    for w in (torch.zeros(16, 36, dtype=torch.bfloat16), torch.zeros(16, 34)):
        with pytest.raises(ValueError, match="multiples of 16 bytes"):
            W4Weight(w)
