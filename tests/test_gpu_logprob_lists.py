"""Top alternatives where few logits are 0 and the rest lie below: the bound that the
lists start above is then 0 itself, which -0 equals and which has no number just
below it but a subnormal one.  Ids exactly, against the oracle."""
import pytest

from gpu_common import say, torch
from serve_common import need_serve
from test_gpu_logprobs import check, score

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rows_of_zeros(rows, vocab, kind):
    """Rows of -1 with sparse zeros, as a mask of allowed tokens used as logits."""
    g = torch.Generator().manual_seed(vocab + rows)
    x = torch.full((rows, vocab), -1.0)
    if kind == "every 200th":
        x[:, ::200] = 0.0
    else:
        share = 0.002 * (1 + torch.arange(rows) % 5)[:, None]
        x[torch.rand(rows, vocab, generator=g) < share] = 0.0
    if kind == "signed":
        zero = x == 0
        x[zero & (torch.rand(rows, vocab, generator=g) < 0.5)] = -0.0
        x[zero & (torch.rand(rows, vocab, generator=g) < 0.03)] = 0.5
        x[torch.rand(rows, vocab, generator=g) < 0.01] = -1e-40       # just below; 0 in a bf16 row's last bits
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["every 200th", "random", "signed"])
@pytest.mark.parametrize("rows", [1, 7, 1024])
def test_sparse_zeros_are_listed(dtype, kind, rows):
    serve = need_serve()
    vocab = 32_000
    say(f"logprob lists {dtype} {kind} {rows} rows")
    x = rows_of_zeros(rows, vocab, kind).to(dtype).cuda()
    targets = torch.zeros(rows, 1, dtype=torch.int64, device="cuda")
    some = list(range(0, rows, max(1, rows // 5)))
    for k in (5, 20, 40, 64):
        out = score(serve, x, targets, k)
        check(x[some], targets[some], k, [t[some] for t in out])
