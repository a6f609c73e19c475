"""Log probabilities where the row's maximum, or all that a part of the row holds, is
far from 0: tokens banned by a large negative number instead of -inf.  Bars as in
``test_gpu_logprobs``."""
import pytest

from gpu_common import say, torch
from serve_common import need_serve
from test_gpu_logprobs import check, score

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("far", [1e4, 1e6, 1e9, 1e10, 3e12, 1e20, 1e30, 1e37, 1e38, 2e38])
@pytest.mark.parametrize("rows,vocab", [(8, 700), (8, 40_001), (1030, 9000)])
def test_far_values(dtype, far, rows, vocab):
    """Whole rows, whole stretches and single tokens at -far; single tokens at far."""
    serve = need_serve()
    say(f"logprobs at {far} {dtype} {rows} x {vocab}")
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(8, vocab, generator=g) * 4
    x[0] = -far                                        # a uniform row
    x[1, :-3] = -far                                   # allowed tokens at the end
    x[2, 3:] = -far                                    # and at the start
    x[3, vocab // 3:vocab // 2] = -far
    x[4, ::2] = -far
    x[5, vocab // 2] = far
    x[6, ::3] = far                                    # a uniform third
    x[7] = -far
    x[7, 5] = -far / 2
    x = x.to(dtype).repeat(rows // 8 + 1, 1)[:rows].cuda()
    targets = torch.tensor([[0, 1, vocab // 2, vocab - 1]], device="cuda").repeat(rows, 1)
    out = score(serve, x, targets, 6)
    check(x[:8], targets[:8], 6, [t[:8] for t in out])
    for t in out:                                      # the other rows are the same eight
        assert torch.equal(t.nan_to_num(7.0), t[:8].repeat(rows // 8 + 1, *[1] * (t.dim() - 1))[:rows].nan_to_num(7.0))
