"""Shared by the GPU tests of the serving operators: inputs, 64-bit references and
the error bars of the attention kernels.

A rounding is off by at most half a step, 2^-8 of a bf16 value and u = 2^-24 of a
float32 one.  A score is a float32 sum of D exact products (of D rounded ones for
float32 inputs): off by at most (D + 1) u sum |q k|, and u of itself for the scale
and for the exponent's argument each, all at most (D + 4) u |q| |k| scale =: e.  A
weight is then off by a factor within exp(e) and 3 u (exp2 within an ulp, the rescale
of the running sum); the sum of n of them by n u more.  Numerator and denominator each
carry that, and the numerator's weights are rounded to bf16 for bf16 inputs; the
division and the merge of partial results are a few u.  An output, an average of values
of at most |V|, is off by
    |V| (2 e + (2 n + 64) u + 2^-8 [bf16 weights]) + its own rounding.
"""
import numpy as np

from gpu_common import torch

U = 2.0**-24


def need_serve():
    from gpu_common import need_gpu
    need_gpu()
    from paper_2607_21927_amd import serve
    return serve


def attn_bar(Q, K, V, n, scale, want, in_dtype, out_dtype):
    """Per-element bar; Q, K, V and want as float64 tensors or arrays."""
    D = Q.shape[-1]
    def norm(x):
        x = torch.as_tensor(x).double().nan_to_num(0, 0, 0)
        return float(x.norm(dim=-1).max()) if x.numel() else 0.0
    v = torch.as_tensor(V).double().nan_to_num(0, 0, 0).abs().max().item()
    e = (D + 4) * U * norm(Q) * norm(K) * scale
    bar = v * (2 * e + (2 * n + 64) * U + (2.0**-8 if in_dtype == torch.bfloat16 else 0))
    return bar + abs(want) * (2.0**-8 if out_dtype == torch.bfloat16 else U)


def bounds(lens):
    return torch.tensor(np.cumsum([0] + list(lens)), dtype=torch.int64, device="cuda")


def head_view(buf, first, heads, D):
    """[heads, T, D] view of head columns of a token-major [T, heads * D] buffer."""
    return buf[:, first * D:(first + heads) * D].unflatten(1, (heads, D)).transpose(0, 1)


def replay_checked(eager, graph_out, change, times=3):
    """Capture ``eager()`` into a HIP graph; replay it after every ``change(i)`` of
    its inputs and hold the outputs to an eager run's, bit for bit."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eager()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eager()
    for i in range(times):
        change(i)
        for t in graph_out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in graph_out]
        for t in graph_out:
            t.zero_()
        eager()
        torch.cuda.synchronize()
        for a, b in zip(got, graph_out):
            assert torch.equal(a, b), i
