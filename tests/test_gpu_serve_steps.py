"""Token steps over the 4-bit cache: what they refuse."""
import pytest

from gpu_common import torch
from serve_common import bounds, need_serve
from test_gpu_serve_model import setup

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
