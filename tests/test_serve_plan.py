"""What the serving path plans on the host: workspaces (no GPU needed)."""
import os
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture(scope="module")
def serve():
    from paper_2607_21927_amd import _build, ris, serve as s
    if not os.path.exists(ris.LIB_PATH):
        _build.build()
    s.lib()
    return s


def test_calls_that_overlap_have_scratch_of_their_own(serve):
    """Two steps over one cache, on two streams or in two captured graphs, must not write
    their partial results to one place."""
    from paper_2607_21927_amd.model import PrefillModel
    cfg = SimpleNamespace(kv_heads=2, head_dim=128)
    cache = PrefillModel.kv4_cache(SimpleNamespace(cfg=cfg, device="cpu", layers=[0]), 2, 4096)
    Q = torch.zeros(2, 12, 128, dtype=torch.bfloat16)
    desc = serve.kv4_decode_desc(Q, cache.layers[0][0], Q, window=4096)
    a, b = cache.workspace(desc), cache.workspace(desc)
    need = serve.kv4_decode_workspace_bytes(desc)
    assert need > 0 and a.numel() >= need and b.numel() >= need
    assert a.data_ptr() + a.numel() <= b.data_ptr() or b.data_ptr() + b.numel() <= a.data_ptr()
    assert a.data_ptr() % 16 == 0


def test_steps_of_another_batch_are_refused(serve):
    """Before the cache takes anything."""
    from paper_2607_21927_amd.model import PrefillModel
    cfg = SimpleNamespace(kv_heads=2, head_dim=128, heads=12)
    model = SimpleNamespace(cfg=cfg, device="cpu", layers=[0])
    cache = PrefillModel.kv4_cache(model, 2, 64)
    for ids, pos in (([1, 2, 3], [0, 0, 0]), ([1], [0]), ([1, 2], [0, 0, 0])):
        with pytest.raises(ValueError, match="2 sequences"):
            PrefillModel.decode_step(model, torch.tensor(ids), torch.tensor(pos), cache)


@pytest.mark.parametrize("rows", [1, 1000, 1024, 4096, 100_000])
@pytest.mark.parametrize("bits", [24, 25, 26, 28, 31])
def test_wide_rows_are_cut_into_parts(serve, rows, bits):
    """A float32 sum of a row has some 2^17 terms at most: 2^25 logits to a workgroup's
    256 threads.  A part's state is 16 bytes of the workspace, 0 where there is one part."""
    vocab = 2**bits - 1
    d = serve.LogprobDesc(1, 1, 0, rows, vocab, vocab)
    parts = max(1, serve.logprobs_workspace_bytes(d) // (16 * rows))
    assert parts <= 64 and -(-vocab // parts) <= 2**25


def test_parts_count_in_the_launch(serve):
    """64 parts a row of 2^31 - 1 logits: what their work-items exceed is refused."""
    for rows, ok in ((2**18 - 1, True), (2**18, False), (2**40, False)):
        v = serve.lib().ris_logprobs_workspace_bytes(serve.LogprobDesc(1, 1, 0, rows, 2**31 - 1, 2**31 - 1))
        assert v > 0 if ok else v == -5
