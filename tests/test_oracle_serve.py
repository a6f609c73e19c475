"""The serving oracle (``oracle/serve.py``) pinned against independent definitions."""
import numpy as np
import pytest
import torch

from oracle import attention as o_att
from oracle import serve as o_srv


@pytest.mark.parametrize("causal", [True, False])
def test_packed_attention_is_each_sequence_alone(causal):
    rng = np.random.default_rng(0)
    cu = [0, 5, 5, 6, 19]
    Q, K, V = (rng.standard_normal((h, 19, 8)) for h in (4, 2, 2))
    got = o_srv.packed_attention(Q, K, V, cu, 0.3, causal)
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        want = torch.nn.functional.scaled_dot_product_attention(
            torch.tensor(Q[:, a:b]), torch.tensor(K[:, a:b]).repeat_interleave(2, 0),
            torch.tensor(V[:, a:b]).repeat_interleave(2, 0), is_causal=causal, scale=0.3)
        np.testing.assert_allclose(got[:, a:b], want.numpy(), atol=1e-12)
    if causal:
        np.testing.assert_allclose(got[:, 6:], o_att.dense_causal(Q[:, 6:], K[:, 6:], V[:, 6:], 0.3), atol=1e-12)


def test_codes_are_the_nearest_values_of_the_least_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((300, 64)) * 10.0 ** rng.integers(-30, 30, (300, 1))
    codes, scales = o_srv.quantise(x)
    v = o_srv.values(codes, scales)
    step = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    assert (np.abs(v - x) <= step * (1 + 1e-12)).all()
    top = np.abs(x.reshape(300, 2, 32)).max(-1)
    s = 2.0 ** (scales.astype(float) - 127)
    assert (top <= 7 * s).all() and (top > 3.5 * s).all()
    # exactly representable values come back, whatever the scale
    e = np.concatenate([o_srv.E2M1, -o_srv.E2M1, o_srv.E2M1, -o_srv.E2M1]) * 2.0**9
    assert np.array_equal(o_srv.values(*o_srv.quantise(e)), e)


def test_ties_go_to_even_codes_and_the_ends_saturate():
    x = np.zeros((1, 32))
    x[0, :9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    codes, scales = o_srv.quantise(x)
    assert scales[0, 0] == 127
    assert list(o_srv.values(codes, scales)[0, :9]) == [6, 0, 1, 1, 2, 2, 4, 4, -4]
    x[0, 0] = 7.0
    assert o_srv.quantise(x)[1][0, 0] == 127 and o_srv.values(*o_srv.quantise(x))[0, 0] == 6
    x[0, 0] = 7.0000001
    assert o_srv.quantise(x)[1][0, 0] == 128
    assert o_srv.quantise(np.zeros((1, 32)))[1][0, 0] == 3
    big = np.full((1, 32), 3.3e38)
    assert o_srv.quantise(big)[1][0, 0] == 252 and np.isfinite(o_srv.values(*o_srv.quantise(big))).all()
    for odd in (np.nan, np.inf, -np.inf):
        x[0, 3] = odd
        assert o_srv.quantise(x)[1][0, 0] == 255 and np.isnan(o_srv.values(*o_srv.quantise(x))).all()


def test_packing_round_trip():
    codes = np.random.default_rng(2).integers(0, 16, (3, 64)).astype(np.uint8)
    assert o_srv.pack(codes)[0, 0] == codes[0, 0] + 16 * codes[0, 1]
    assert np.array_equal(o_srv.unpack(o_srv.pack(codes)), codes)


def test_logprobs_against_log_softmax():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(1000) * 5
    x[10:20] = -np.inf
    x[500] = x[7] = 30.0
    lp, ent, ids, top = o_srv.logprobs(x, [3, 15, -1, 1000], 12)
    y = torch.log_softmax(torch.tensor(x), 0)
    assert lp[0] == pytest.approx(y[3].item(), abs=1e-12) and lp[1] == -np.inf and lp[2] == 0 and np.isnan(lp[3])
    assert ent == pytest.approx(torch.distributions.Categorical(logits=torch.tensor(x)).entropy().item(), abs=1e-9)
    assert list(ids[:2]) == [7, 500]
    assert np.array_equal(np.sort(ids), np.sort(torch.tensor(x).topk(12).indices.numpy()))
    np.testing.assert_allclose(top, y[torch.tensor(ids)].numpy(), atol=1e-12)
    # nothing but -inf; fewer tokens than places; NaN first, then +inf
    lp, ent, ids, top = o_srv.logprobs(np.full(5, -np.inf), [1], 2)
    assert lp[0] == -np.inf and ent == 0 and list(ids) == [-1, -1] and (top == -np.inf).all()
    lp, ent, ids, top = o_srv.logprobs(np.array([-np.inf, 2.0, -np.inf]), [1], 2)
    assert lp[0] == 0 and ent == 0 and list(ids) == [1, -1] and list(top) == [0, -np.inf]
    lp, ent, ids, top = o_srv.logprobs(np.array([1.0, np.inf, np.nan]), [0], 3)
    assert np.isnan(lp[0]) and np.isnan(ent) and list(ids) == [2, 1, 0] and np.isnan(top).all()
