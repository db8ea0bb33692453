"""The oracle of the attention over sequences against differences, against torch's own softmax, and by hand."""
import numpy as np
import pytest
import torch

from oracle import seq_oracle as O


def _inputs(seed, B=2, heads=4, kv=2, Lq=7, Lk=9, D=5):
    g = np.random.default_rng(seed)
    return [g.standard_normal(s) for s in ((B, heads, Lq, D), (B, kv, Lk, D), (B, kv, Lk, D), (B, heads, Lq, D))]


MASKS = [dict(), dict(causal=True), dict(causal=True, window=3), dict(window=2), dict(causal=True, softcap=1.5), dict(slopes=np.array([0.1, 0.5, -0.2, 0.0])),
         dict(causal=True, documents=np.array([[0, 0, 0, 1, 1, 1, 2, 2, -1], [5, 5, -1, 5, 5, 7, 7, 7, 7]])),
         dict(causal=True, window=2, prefix=np.array([[1, 1, 0, 0, 0, 0, 0, 0, 1], [0] * 9]), softcap=2.0, slopes=np.array([0.3, 0.2, 0.1, 0.05]))]


@pytest.mark.parametrize("mask", MASKS)
def test_gradients_against_differences(mask):
    q, k, v, dout = _inputs(1)
    res, _ = O.attention(q, k, v, dout, **mask)
    g = np.random.default_rng(2)
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        step = g.standard_normal((q, k, v)[at].shape)
        sides = []
        for sign in (1, -1):
            x = [q, k, v]
            x[at] = x[at] + sign * 1e-5 * step
            sides.append((O.attention(*x, **mask)[0]["out"] * dout).sum())
        assert abs((sides[0] - sides[1]) / 2e-5 - (res[name] * step).sum()) < 1e-7, name


@pytest.mark.parametrize("mask", MASKS[:4])
def test_forward_against_torch(mask):
    q, k, v, _ = _inputs(3)
    see = torch.from_numpy(O.visible(7, 9, **mask))
    kk, vv = (torch.from_numpy(x).repeat_interleave(2, 1) for x in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q), kk, vv, attn_mask=see)
    assert np.abs(O.attention(q, k, v, **mask)[0]["out"] - want.numpy()).max() < 1e-12


def test_visible_by_hand():
    see = O.visible(2, 5, causal=True, window=2, prefix=np.array([1, 0, 0, 0, 0]), documents=np.array([3, 3, 3, 3, 4]))
    assert see.tolist() == [[True, False, True, True, False], [False, False, False, False, True]]
    assert not O.visible(3, 2, causal=True)[0].any()


def test_append_by_hand():
    cells, scales = np.zeros((2, 1, 2, 2), np.int8), np.zeros((2, 1), np.float32)
    x = np.array([[[[1.27, 0.0], [0.0, -2.54], [5.0, 5.0]]]], np.float32)
    table = np.array([[1, 0]])
    cells, scales = O.append(cells, scales, x, table, [0])
    assert cells[1, 0].tolist() == [[64, 0], [0, -127]] and cells[0, 0, 0].tolist() == [127, 127] and abs(scales[1, 0] - 0.02) < 1e-8
    # a larger token behind it: what the page held is rounded again on the new scale
    cells, scales = O.append(cells, scales, np.full((1, 1, 1, 2), 10.0, np.float32), table, [3])
    assert cells[0, 0].tolist() == [[64, 64], [127, 127]]
    assert O.gather(cells, scales, table, [4], [3], 2)[0, 0, 1].tolist() == [0.0, 0.0]
