"""Python binding of the serving operators of libris.so (``include/ris_serve.h``).

Argument checks and marshalling only, as in ``ris``: every step runs in the HIP
library, the caller owns every tensor, and the work goes to torch's current HIP
stream of the tensors' device unless a stream is given.
"""
import ctypes

import torch

from . import ris

MAX_TOP = 64
KV4_BLOCK = 32          # dimensions that share a scale in the 4-bit cache


class PromptDesc(ctypes.Structure):
    _fields_ = [("dtype_in", ctypes.c_int32), ("dtype_out", ctypes.c_int32),
                ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("T", ctypes.c_int64), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float),
                ("q_head", ctypes.c_int64), ("q_token", ctypes.c_int64),
                ("k_head", ctypes.c_int64), ("k_token", ctypes.c_int64),
                ("v_head", ctypes.c_int64), ("v_token", ctypes.c_int64),
                ("o_head", ctypes.c_int64), ("o_token", ctypes.c_int64)]


class Kv4Desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("T", ctypes.c_int64), ("max_len", ctypes.c_int64),
                ("k_head", ctypes.c_int64), ("k_token", ctypes.c_int64),
                ("v_head", ctypes.c_int64), ("v_token", ctypes.c_int64)]


class LogprobDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_targets", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class PageMap(ctypes.Structure):
    _fields_ = [("page", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("pages", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("table_stride", ctypes.c_int64)]


class PageStoreDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("T", ctypes.c_int64), ("map", PageMap),
                ("q_head", ctypes.c_int64), ("q_token", ctypes.c_int64),
                ("qo_head", ctypes.c_int64), ("qo_token", ctypes.c_int64),
                ("k_head", ctypes.c_int64), ("k_token", ctypes.c_int64),
                ("v_head", ctypes.c_int64), ("v_token", ctypes.c_int64)]


class PageAttnDesc(ctypes.Structure):
    _fields_ = [("dtype_in", ctypes.c_int32), ("dtype_out", ctypes.c_int32),
                ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("T", ctypes.c_int64), ("map", PageMap),
                ("window", ctypes.c_int32), ("sink", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q_head", ctypes.c_int64), ("q_token", ctypes.c_int64),
                ("o_head", ctypes.c_int64), ("o_token", ctypes.c_int64)]


class W4Desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("gated", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("x_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64)]


EXPORTS = ("ris_rope_packed", "ris_prompt_attn", "ris_kv4_store", "ris_kv4_load",
           "ris_kv4_decode_workspace_bytes", "ris_kv4_decode_attn", "ris_logprobs_workspace_bytes",
           "ris_logprobs", "ris_page_store", "ris_page_attn_workspace_bytes", "ris_page_attn", "ris_w4_pack", "ris_w4_load",
           "ris_w4_linear")

_lib = None


def lib():
    """``ris.lib()`` with the prototypes of this module's entry points."""
    global _lib
    if _lib is None:
        L = ris.lib()
        vp, i32, i64, ptr = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.POINTER
        L.ris_rope_packed.argtypes = [vp, i64, i64, vp, i32, i32, i64, i32, vp, vp, i32, ptr(ris.RopeDesc), vp]
        L.ris_prompt_attn.argtypes = [vp, vp, vp, vp, vp, ptr(PromptDesc), vp]
        L.ris_kv4_store.argtypes = [vp] * 7 + [ptr(Kv4Desc), vp]
        L.ris_kv4_load.argtypes = [vp] * 7 + [ptr(Kv4Desc), vp]
        L.ris_kv4_decode_workspace_bytes.argtypes = [ptr(ris.DecodeDesc)]
        L.ris_kv4_decode_attn.argtypes = [vp] * 9 + [i64, ptr(ris.DecodeDesc), vp]
        L.ris_logprobs_workspace_bytes.argtypes = [ptr(LogprobDesc)]
        L.ris_logprobs.argtypes = [vp] * 7 + [i64, ptr(LogprobDesc), vp]
        L.ris_page_store.argtypes = [vp] * 9 + [ptr(PageStoreDesc), ptr(ris.RopeDesc), vp]
        L.ris_page_attn_workspace_bytes.argtypes = [ptr(PageAttnDesc)]
        L.ris_page_attn.argtypes = [vp] * 8 + [i64, ptr(PageAttnDesc), vp]
        L.ris_w4_pack.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
        L.ris_w4_load.argtypes = [vp, vp, vp, i32, i64, i64, i64, vp]
        L.ris_w4_linear.argtypes = [vp] * 5 + [ptr(W4Desc), vp]
        for name in EXPORTS:
            getattr(L, name).restype = i64 if name.endswith("_bytes") else ctypes.c_int
        _lib = L
    return _lib


_CODES = {torch.float32: ris.F32, torch.bfloat16: ris.BF16}


def _code(t):
    code = _CODES.get(t.dtype)
    return ris._dtype_code(t) if code is None else code         # raises


def _one_gpu(t, *others):
    """Index of the GPU that holds all of the tensors."""
    index = t.get_device()
    for o in others:
        if o is not None and o.get_device() != index:
            index = -1
    if index < 0:
        raise ValueError("tensors must be on one GPU")
    return index


def _need_dense(*ts):
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


def _rows(t, shape):
    """Address, head and token stride of a [heads, T, D] view whose rows 16-byte
    accesses can walk; a dimension of one element counts with stride 0."""
    if t.shape != shape:
        raise ValueError(f"expected a {shape} view, got {tuple(t.shape)}")
    head, token, one = t.stride()
    if shape[0] == 1:
        head = 0
    if shape[1] == 1:
        token = 0
    at = t.data_ptr()
    if one != 1 or (at | (head | token) * t.element_size()) & 15:
        raise ValueError("rows must be contiguous, bases and strides multiples of 16 bytes")
    return at, head, token


def _placed(t, shape, strides):
    """Address of a view that a descriptor has the shape and (head, token, 1) strides of."""
    if t.shape != shape or t.stride() != strides and _rows(t, shape)[1:] != strides[:2]:
        raise ValueError(f"shape and strides must match the descriptor, got {tuple(t.shape)}, {t.stride()}")
    at = t.data_ptr()
    if at & 15:
        raise ValueError("bases must be multiples of 16 bytes")
    return at


def _bounds(cu_seqlens, start=None):
    batch = cu_seqlens.numel() - 1
    if cu_seqlens.dtype != torch.int64 or not cu_seqlens.is_contiguous():
        raise TypeError("cu_seqlens must be a contiguous int64 vector")
    if batch < 1:
        raise ValueError("cu_seqlens must hold batch + 1 offsets")
    if start is not None:
        if start.dtype != torch.int64 or not start.is_contiguous():
            raise TypeError("start must be a contiguous int64 vector")
        if start.numel() != batch:
            raise ValueError("start must hold one position a sequence")
    return batch


def _at(t):
    return 0 if t is None else t.data_ptr()


# torch.cuda.current_stream without the Stream object around the handle (1 us of a 9 us call)
_current_stream = torch._C._cuda_getCurrentRawStream if torch.version.hip else None
_entry = {}


def _call(index, stream, name, *args):
    """Launch on `stream` (torch's current one of GPU `index`) with that GPU current."""
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return _call(index, stream, name, *args)
    if stream is None:
        stream = _current_stream(index)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    entry = _entry.get(name)
    if entry is None:
        entry = _entry[name] = getattr(lib(), name)
    status = entry(*args, stream)
    if status != ris.OK:
        raise ris.RisError(status, name)


def rope_packed(src, out, cu_seqlens, desc, start=None, stream=None):
    """ris_rope_packed: src is a [heads, T, D] view (unit stride along D), out
    [heads, T, D] contiguous; token i of sequence b is rotated to position
    start[b] + i (start None: i)."""
    index = _one_gpu(out, src, cu_seqlens, start)
    _need_dense(out)
    H, T, D = out.shape
    head, token, one = src.stride()
    if src.shape != out.shape or one != 1 or src.dtype != out.dtype:
        raise ValueError("src must be a [heads, T, D] view of out's dtype with unit stride along D")
    batch = _bounds(cu_seqlens, start)
    _call(index, stream, "ris_rope_packed", src.data_ptr(), head, token, out.data_ptr(), _code(out), H, T, D,
          cu_seqlens.data_ptr(), _at(start), batch, desc)
    return out


def prompt_desc(Q, K, V, out, cu_seqlens, causal=1, scale=0.0):
    """Descriptor from views Q, out [Hq, T, D] and K, V [Hkv, T, D]."""
    Hq, T, D = Q.shape
    return PromptDesc(_code(Q), _code(out), Hq, K.shape[0], D, cu_seqlens.numel() - 1, T, causal, scale,
                      *_rows(Q, Q.shape)[1:], *_rows(K, K.shape)[1:], *_rows(V, V.shape)[1:], *_rows(out, out.shape)[1:])


def prompt_attn(Q, K, V, cu_seqlens, out, desc, stream=None):
    """ris_prompt_attn: dense attention of packed prompts.  Q, out [Hq, T, D] and
    K, V [Hkv, T, D] are views of any head and token strides that are multiples of
    16 bytes (head columns of a token-major projection output, for instance)."""
    index = _one_gpu(out, Q, K, V, cu_seqlens)
    if not (Q.dtype == K.dtype == V.dtype):
        raise TypeError("Q, K, V must share a dtype")
    if _code(Q) != desc.dtype_in or _code(out) != desc.dtype_out:
        raise TypeError("Q and out dtypes must match the descriptor")
    q, kv = (desc.Hq, desc.T, desc.D), (desc.Hkv, desc.T, desc.D)
    q_at, k_at = _placed(Q, q, (desc.q_head, desc.q_token, 1)), _placed(K, kv, (desc.k_head, desc.k_token, 1))
    v_at, o_at = _placed(V, kv, (desc.v_head, desc.v_token, 1)), _placed(out, q, (desc.o_head, desc.o_token, 1))
    if _bounds(cu_seqlens) != desc.batch:
        raise ValueError("cu_seqlens must hold the descriptor's batch + 1 offsets")
    _call(index, stream, "ris_prompt_attn", q_at, k_at, v_at, cu_seqlens.data_ptr(), o_at, desc)
    return out


def kv4_cache(batch, Hkv, max_len, D, device="cuda"):
    """Empty 4-bit cache: codes K4, V4 [batch, Hkv, max_len, D / 2] and scales S
    [batch, Hkv, max_len, 2, D / 32], uint8."""
    codes = [torch.zeros(batch, Hkv, max_len, D // 2, dtype=torch.uint8, device=device) for _ in range(2)]
    return codes[0], codes[1], torch.zeros(batch, Hkv, max_len, 2, D // KV4_BLOCK, dtype=torch.uint8, device=device)


def _need_cache(K4, V4, S, batch, Hkv, D):
    if not (K4.dtype == V4.dtype == S.dtype == torch.uint8):
        raise TypeError("K4, V4 and S must be uint8")
    _need_dense(K4, V4, S)
    max_len = K4.shape[2] if K4.dim() == 4 else 0
    if (K4.shape != (batch, Hkv, max_len, D // 2) or V4.shape != K4.shape
            or S.shape != (batch, Hkv, max_len, 2, D // KV4_BLOCK)):
        raise ValueError("K4 and V4 must be [batch, Hkv, max_len, D / 2] and S [batch, Hkv, max_len, 2, D / 32]")
    return max_len


def _kv4(K, V, cu_seqlens, K4, V4, S, start):
    index = _one_gpu(K4, K, V, cu_seqlens, V4, S, start)
    if K.dtype != V.dtype:
        raise TypeError("K and V must share a dtype")
    Hkv, T, D = shape = tuple(K.shape)
    batch = _bounds(cu_seqlens, start)
    max_len = _need_cache(K4, V4, S, batch, Hkv, D)
    k_at, *k_strides = _rows(K, shape)
    v_at, *v_strides = _rows(V, shape)
    return index, k_at, v_at, Kv4Desc(_code(K), Hkv, D, batch, T, max_len, *k_strides, *v_strides)


def kv4_store(K, V, cu_seqlens, K4, V4, S, start=None, stream=None):
    """ris_kv4_store: rows K, V [Hkv, T, D] (views as in ``prompt_attn``) quantised
    into the cache, token i of sequence b at position start[b] + i (start None: i)."""
    index, k_at, v_at, desc = _kv4(K, V, cu_seqlens, K4, V4, S, start)
    _call(index, stream, "ris_kv4_store", k_at, v_at, cu_seqlens.data_ptr(), _at(start), K4.data_ptr(),
          V4.data_ptr(), S.data_ptr(), desc)


def kv4_load(K4, V4, S, cu_seqlens, K, V, start=None, stream=None):
    """ris_kv4_load: the cache's values at those positions into K, V [Hkv, T, D]."""
    index, k_at, v_at, desc = _kv4(K, V, cu_seqlens, K4, V4, S, start)
    _call(index, stream, "ris_kv4_load", K4.data_ptr(), V4.data_ptr(), S.data_ptr(), cu_seqlens.data_ptr(), _at(start),
          k_at, v_at, desc)


def kv4_decode_desc(Q, K4, out, anchor_stride=0, window=0, sink=0, scale=0.0):
    """Descriptor from Q [B, Hq, D], the codes K4 [B, Hkv, max_len, D / 2] and out."""
    B, Hq, D = Q.shape
    return ris.DecodeDesc(_code(Q), _code(out), B, Hq, K4.shape[1], D, K4.shape[2], anchor_stride, window,
                          sink, scale)


def kv4_decode_workspace_bytes(desc):
    v = lib().ris_kv4_decode_workspace_bytes(ctypes.byref(desc))
    if v < 0:
        raise ris.RisError(int(v), "ris_kv4_decode_workspace_bytes")
    return int(v)


def kv4_decode_attn(Q, K4, V4, S, pos, anchor_ptr, anchor_idx, out, workspace, desc, stream=None):
    """ris_kv4_decode_attn; workspace is a device uint8 tensor of at least
    kv4_decode_workspace_bytes(desc) bytes.  anchor_ptr and anchor_idx may be None
    where the descriptor's anchor_stride is 0."""
    index = _one_gpu(out, Q, K4, V4, S, pos, anchor_ptr, anchor_idx, workspace)
    _need_dense(Q, pos, anchor_ptr, anchor_idx, out, workspace)
    if pos.dtype != torch.int64 or pos.numel() != desc.batch:
        raise ValueError("pos must be int64 and hold B entries")
    if desc.anchor_stride > 0:
        if anchor_ptr is None or anchor_idx is None:
            raise ValueError("anchor_ptr and anchor_idx are needed where anchor_stride > 0")
        if anchor_ptr.dtype != torch.int64 or anchor_idx.dtype != torch.int32:
            raise TypeError("anchor_ptr must be int64, anchor_idx int32")
        if anchor_ptr.numel() != desc.batch * (desc.Hkv + 1) or anchor_idx.numel() < desc.batch * desc.anchor_stride:
            raise ValueError("anchor_ptr must hold B * (Hkv + 1) entries and anchor_idx B * anchor_stride")
    if _code(Q) != desc.dtype_in or _code(out) != desc.dtype_out:
        raise TypeError("Q and out dtypes must match the descriptor")
    if Q.shape != (desc.batch, desc.Hq, desc.D) or out.shape != Q.shape:
        raise ValueError("Q and out must be [B, Hq, D] as in the descriptor")
    if _need_cache(K4, V4, S, desc.batch, desc.Hkv, desc.D) != desc.max_len:
        raise ValueError("the cache's max_len must match the descriptor")
    nbytes = workspace.numel() * workspace.element_size()
    _call(index, stream, "ris_kv4_decode_attn", Q.data_ptr(), K4.data_ptr(), V4.data_ptr(), S.data_ptr(), pos.data_ptr(),
          _at(anchor_ptr), _at(anchor_idx), out.data_ptr(), workspace.data_ptr(), nbytes, desc)
    return out


def logprob_desc(logits, n_targets=1, top_k=0):
    """Descriptor from logits [rows, vocab] (unit stride along vocab)."""
    rows, vocab = logits.shape
    return LogprobDesc(_code(logits), n_targets, top_k, rows, vocab, max(logits.stride(0), vocab) if rows > 1 else vocab)


def logprobs_workspace_bytes(desc):
    v = lib().ris_logprobs_workspace_bytes(ctypes.byref(desc))
    if v < 0:
        raise ris.RisError(int(v), "ris_logprobs_workspace_bytes")
    return int(v)


def logprobs(logits, targets, logprob, entropy, top_ids, top_logprob, workspace, desc, stream=None):
    """ris_logprobs: rows of logits [rows, vocab] scored.  targets int64 and
    logprob float32 [rows, n_targets], entropy float32 [rows] or None, top_ids
    int64 and top_logprob float32 [rows, top_k]; what the descriptor counts 0 of
    may be None.  workspace: at least logprobs_workspace_bytes(desc) bytes."""
    index = _one_gpu(logits, targets, logprob, entropy, top_ids, top_logprob, workspace)
    rows, n, k = desc.rows, desc.n_targets, desc.top_k
    if logits.shape != (rows, desc.vocab) or logits.stride(1) != 1 and desc.vocab > 1:
        raise ValueError("logits must be [rows, vocab] as in the descriptor, unit stride along vocab")
    if rows > 1 and logits.stride(0) != desc.row_stride or _code(logits) != desc.dtype:
        raise ValueError("the logits' row stride and dtype must match the descriptor")
    _need_dense(targets, logprob, entropy, top_ids, top_logprob, workspace)
    for t, count, dtype in ((targets, n, torch.int64), (logprob, n, torch.float32), (top_ids, k, torch.int64),
                            (top_logprob, k, torch.float32)):
        if t is None and count or t is not None and (t.shape != (rows, count) or t.dtype != dtype):
            raise ValueError("targets and logprob must be [rows, n_targets], top_ids and top_logprob [rows, top_k] "
                             "(ids int64, the others float32)")
    if entropy is not None and (entropy.shape != (rows,) or entropy.dtype != torch.float32):
        raise ValueError("entropy must be float32 [rows]")
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _call(index, stream, "ris_logprobs", logits.data_ptr(), _at(targets), _at(logprob), _at(entropy), _at(top_ids),
          _at(top_logprob), _at(workspace), nbytes, desc)
    return logprob


# ---- cache in pages

def page_cache(pages, Hkv, page, D, device="cuda"):
    """Empty pages Kp, Vp [pages, Hkv, page, D], bf16."""
    return [torch.zeros(pages, Hkv, page, D, dtype=torch.bfloat16, device=device) for _ in range(2)]


def _page_map(Kp, table):
    """Map of pages [pages, Hkv, page, D], whose pages may lie apart, under a block table
    [batch, max_pages] int32, whose rows may."""
    pages, Hkv, page, D = Kp.shape
    stride, *within = Kp.stride()
    if within != [page * D, D, 1] and not Kp[0].is_contiguous():
        raise ValueError("pages must be [Hkv, page, D] contiguous")
    if table.dtype != torch.int32:
        raise TypeError("the block table must be int32")
    rows, row = table.shape, table.stride()
    if len(rows) != 2 or row[1] != 1 and rows[1] > 1:
        raise ValueError("the block table must be [batch, max_pages] with unit stride along a row")
    return PageMap(page, rows[1], pages, Hkv * page * D if pages == 1 else stride, rows[1] if rows[0] == 1 else row[0])


def _need_pages(Kp, Vp):
    if Kp.dtype != torch.bfloat16 or Vp.dtype != torch.bfloat16:
        raise TypeError("pages must be bfloat16")
    shape, k, v = Kp.shape, Kp.stride(), Vp.stride()
    if len(shape) != 4 or Vp.shape != shape or v != k and any(n > 1 and a != b for n, a, b in zip(shape, k, v)):
        raise ValueError("Kp and Vp must be [pages, Hkv, page, D], of one shape and strides")
    return shape


def page_store(K, V, cu_seqlens, table, Kp, Vp, start=None, q=None, q_out=None, rope=None, stream=None):
    """ris_page_store: rows K, V [Hkv, T, D] (views as in ``prompt_attn``) into the pages
    that ``table`` names, token i of sequence b at position start[b] + i (start None: i).
    rope: a ``ris.rope_desc`` that K, and q [Hq, T, D] into q_out, are rotated by (None: K and q
    are copied)."""
    index = _one_gpu(Kp, K, V, cu_seqlens, table, Vp, start, q, q_out)
    pages = _need_pages(Kp, Vp)
    dtype, shape = K.dtype, K.shape
    if V.dtype != dtype:
        raise TypeError("K and V must share a dtype")
    k_at, k_head, k_token = _rows(K, shape)
    v_at, v_head, v_token = _rows(V, shape)
    Hkv, T, D = shape
    if pages[1] != Hkv or pages[3] != D:
        raise ValueError("Kp and Vp must be [pages, Hkv, page, D] with the rows' Hkv and D")
    batch = _bounds(cu_seqlens, start)
    where = _page_map(Kp, table)
    if table.shape[0] != batch:
        raise ValueError("the block table must hold one row a sequence")
    Hq = q_at = q_head = q_token = o_at = o_head = o_token = 0
    if q is not None and q_out is not None:
        if q.dtype != dtype or q_out.dtype != dtype:
            raise TypeError("q and q_out must have the dtype of K and V")
        Hq = q.shape[0]
        of = (Hq, T, D)
        q_at, q_head, q_token = _rows(q, of)
        o_at, o_head, o_token = _rows(q_out, of)
    elif q is not q_out:
        raise ValueError("q and q_out go together")
    desc = PageStoreDesc(_code(K), Hq, Hkv, D, batch, T, where, q_head, q_token, o_head, o_token, k_head, k_token, v_head,
                         v_token)
    _call(index, stream, "ris_page_store", q_at, o_at, k_at, v_at, cu_seqlens.data_ptr(), _at(start), table.data_ptr(),
          Kp.data_ptr(), Vp.data_ptr(), desc, rope)


def page_attn_desc(Q, Kp, table, cu_seqlens, out, window=None, sink=0, scale=0.0):
    """Descriptor from views Q, out [Hq, T, D], pages Kp [pages, Hkv, page, D] and the block
    table [batch, max_pages].  window None: every key up to a token."""
    Hq, T, D = Q.shape
    return PageAttnDesc(_code(Q), _code(out), Hq, Kp.shape[1], D, cu_seqlens.numel() - 1, T, _page_map(Kp, table),
                        min(0x7FFFFFFF, table.shape[1] * Kp.shape[2] if window is None else window), min(0x7FFFFFFF, sink), scale,
                        *_rows(Q, Q.shape)[1:], *_rows(out, Q.shape)[1:])


def page_attn_workspace_bytes(desc):
    v = lib().ris_page_attn_workspace_bytes(ctypes.byref(desc))
    if v < 0:
        raise ris.RisError(int(v), "ris_page_attn_workspace_bytes")
    return int(v)


def page_attn(Q, Kp, Vp, table, cu_seqlens, out, workspace, desc, start=None, stream=None):
    """ris_page_attn: attention of the new tokens Q [Hq, T, D] over the pages that hold
    them already, token i of sequence b at position start[b] + i (start None: i).
    workspace: at least page_attn_workspace_bytes(desc) bytes, None where that is 0."""
    index = _one_gpu(out, Q, Kp, Vp, table, cu_seqlens, workspace, start)
    shape = _need_pages(Kp, Vp)
    _need_dense(workspace)
    if _code(Q) != desc.dtype_in or _code(out) != desc.dtype_out:
        raise TypeError("Q and out dtypes must match the descriptor")
    m, q, batch, D = desc.map, (desc.Hq, desc.T, desc.D), desc.batch, desc.D
    pages, page, stride = m.pages, m.page, Kp.stride()
    if shape != (pages, desc.Hkv, page, D) or stride != (m.page_stride, page * D, D, 1) and (
            pages > 1 and stride[0] != m.page_stride or stride[1:] != (page * D, D, 1) and not Kp[0].is_contiguous()):
        raise ValueError("Kp and Vp must be [pages, Hkv, page, D] as in the descriptor")
    most, row = m.max_pages, table.stride()
    if table.dtype != torch.int32 or table.shape != (batch, most) or row != (m.table_stride, 1) and (
            row[1] != 1 and most > 1 or row[0] != m.table_stride and batch > 1):
        raise ValueError("the block table must be int32 [batch, max_pages] as in the descriptor")
    q_at, o_at = _placed(Q, q, (desc.q_head, desc.q_token, 1)), _placed(out, q, (desc.o_head, desc.o_token, 1))
    if _bounds(cu_seqlens, start) != batch:
        raise ValueError("cu_seqlens must hold the descriptor's batch + 1 offsets")
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _call(index, stream, "ris_page_attn", q_at, Kp.data_ptr(), Vp.data_ptr(), table.data_ptr(), cu_seqlens.data_ptr(),
          _at(start), o_at, _at(workspace), nbytes, desc)
    return out


# ---- weights in 4 bits

def w4_weight(N, K, device="cuda"):
    """Empty 4-bit weights of N outputs and K inputs: codes C [tiles of 16 outputs, tiles of
    128 inputs, 4, 16, 16] and scales S [tiles, ceil(K / 512), 4, 16, 4], uint8."""
    n = -(-N // 16)
    return (torch.zeros(n, -(-K // 128), 4, 16, 16, dtype=torch.uint8, device=device),
            torch.zeros(n, -(-K // 512), 4, 16, 4, dtype=torch.uint8, device=device))


def _need_w4(C, S, N, K):
    if C.dtype != torch.uint8 or S.dtype != torch.uint8:
        raise TypeError("C and S must be uint8")
    n = -(-N // 16)
    if C.shape != (n, -(-K // 128), 4, 16, 16) or S.shape != (n, -(-K // 512), 4, 16, 4):
        raise ValueError(f"C and S must be those of {N} outputs and {K} inputs")
    _need_dense(C, S)


def _matrix(t, rows, cols):
    """Row stride of a [rows, cols] matrix with unit stride along a row."""
    if t.shape != (rows, cols) or t.stride(1) != 1 and cols > 1:
        raise ValueError(f"expected a [{rows}, {cols}] matrix with unit stride along its rows, got {tuple(t.shape)}")
    return t.stride(0) if rows > 1 else cols


def w4_pack(W, C, S, stream=None):
    """ris_w4_pack: rows of W [N, K] quantised into the weights C, S."""
    index = _one_gpu(W, C, S)
    N, K = W.shape
    _need_w4(C, S, N, K)
    _call(index, stream, "ris_w4_pack", W.data_ptr(), _code(W), N, K, _matrix(W, N, K), C.data_ptr(), S.data_ptr())


def w4_load(C, S, W, stream=None):
    """ris_w4_load: the values that the weights C, S stand for into W [N, K]."""
    index = _one_gpu(W, C, S)
    N, K = W.shape
    _need_w4(C, S, N, K)
    _call(index, stream, "ris_w4_load", C.data_ptr(), S.data_ptr(), W.data_ptr(), _code(W), N, K, _matrix(W, N, K))
    return W


def w4_linear(x, C, S, out, bias=None, gated=False, stream=None):
    """ris_w4_linear: out [rows, N] = x [rows, K] W^T + bias for the weights C, S; gated:
    out [rows, N / 2] = silu(first half) * second half.  Rows of x lie multiples of 16
    bytes apart."""
    index = _one_gpu(out, x, C, S, bias)
    (rows, K), cols = x.shape, out.shape[1]
    N = 2 * cols if gated else cols
    _need_w4(C, S, N, K)
    if out.dtype != x.dtype or bias is not None and (bias.dtype != x.dtype or bias.shape != (N,)):
        raise ValueError("out and bias [N] must have the dtype of x")
    _need_dense(bias)
    x_stride = _matrix(x, rows, K)
    if rows == 1:
        x_stride = -(-K // 8) * 8                       # whatever the stride of one row
    desc = W4Desc(_code(x), int(gated), rows, N, K, x_stride, _matrix(out, rows, cols))
    _call(index, stream, "ris_w4_linear", x.data_ptr(), C.data_ptr(), S.data_ptr(), _at(bias), out.data_ptr(), desc)
    return out
