"""The plain forms that the output head's cases are timed against: distillation in elementary operations gives the oracle's loss and
gradient, at the lists and rows where its formula has a case of its own."""
import numpy as np
import pytest
import torch

from oracle import heads
from perf import operators

U = 2.0 ** -24


def lists(rng, B, V, k):
    raw = rng.standard_normal((B, k))
    value = raw - np.log(np.exp(raw).sum(-1, keepdims=True)) + np.log(rng.uniform(0.3, 0.9, (B, 1)))
    index = np.argsort(rng.random((B, V)), -1)[:, :k] if k <= V else rng.integers(0, V, (B, k))
    return value.astype(np.float32), index.astype(np.int32)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,k", [(1, 1), (10, 10), (64, 64), (100, 64), (20, 16), (7, 30), (300, 5)])
def test_plain_distillation_is_the_oracle_s(V, k, tail):
    """Lists of the whole vocabulary, in which every token that has a probability is listed, of tokens listed twice, short ones; rows of
    weight 0.  The plain form rounds z, its exponentials and their sums to fp32: SUM covers V roundings and 32 |z| of 2^-24."""
    B, temperature = 9, 2.0
    rng = np.random.default_rng(V + k)
    x = rng.standard_normal((B, V)) * 3
    value, index = lists(rng, B, V, k)
    others = np.setdiff1d(np.arange(V), index[1])
    x[1, others] = -np.inf                                     # nothing outside the list
    index[2, k // 2:] = index[2, :k - k // 2]                  # the same tokens again
    index[3, (k + 1) // 2:] = -1
    weight = rng.uniform(0.5, 1.5, B).astype(np.float32)
    weight[4] = 0
    x = x.astype(np.float32)
    st = dict(op="distill", logits=torch.from_numpy(x), temperature=temperature, teacher_index=torch.from_numpy(index),
              teacher_logprob=torch.from_numpy(value), tail=tail, row_weight=torch.from_numpy(weight), B=B, nodes=1)
    out = operators._plain(st)
    loss, row_loss, grad = heads.distill_topk(x[None], value[None], index[None], tail, temperature, weight[None])
    SUM = (V + 32 * 16 + 64) * U
    near = lambda got, want, tol: (np.abs(got.double().numpy() - want) <= tol).all()
    assert near(out["row_loss"], row_loss[0], SUM * (2 + np.abs(row_loss[0])))
    assert near(out["loss"], loss, SUM * (2 + np.abs(loss)) * 1.5)
    assert near(out["dlogits"], grad[0], 4 * SUM * 1.5 / (B * temperature))


@pytest.mark.parametrize("masked", [False, True])
def test_gradient_where_nothing_lies_outside_the_list(masked):
    """A list of 0.6 of the teacher's mass over every token that has a probability: the loss has no class for the rest, and neither has the
    gradient, p sum t - t (central differences of the oracle's own loss, and the formula)."""
    x = np.array([[[0.3, -1.0, 0.8, 0.1]]])
    p = np.exp(x[0, 0]) / np.exp(x[0, 0]).sum()
    if masked:
        x = np.concatenate([x, np.full((1, 1, 3), -np.inf)], -1)
    t = np.array([0.3, 0.1, 0.15, 0.05])
    value, index = np.log(t)[None, None], np.arange(4)[None, None]
    loss, _, grad = heads.distill_topk(x, value, index, True)
    assert np.allclose(loss, (t * np.log(t / p)).sum())
    assert np.allclose(grad[0, 0, :4], p * t.sum() - t) and not grad[0, 0, 4:].any()
    for v in range(4):
        up, down = x.copy(), x.copy()
        up[0, 0, v] += 1e-5
        down[0, 0, v] -= 1e-5
        f = lambda x: heads.distill_topk(x, value, index, True)[0][0]
        assert abs((f(up) - f(down)) / 2e-5 - grad[0, 0, v]) < 1e-8


@pytest.mark.parametrize("mask", [-np.inf, float(np.finfo(np.float32).min)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_row_with_nan_beside_masks_answers_nan(mask, bad):
    """In the oracle: loss and gradient, with the token on the list, beside it, and without a list; not with a weight of 0."""
    x = np.full((1, 4, 6), mask)
    x[0, 0, 2] = x[0, 1, 5] = x[0, 2, 5] = x[0, 3, 2] = bad
    index = np.array([[[2, 4], [2, 4], [-1, -1], [2, 4]]])
    value = np.log(np.full((1, 4, 2), 0.3))
    weight = np.array([[1.0, 1.0, 1.0, 0.0]])
    for tail in (True, False):
        _, row_loss, grad = heads.distill_topk(x, value, index, tail, 1.0, weight)
        assert np.isnan(row_loss[0, :3]).all() and np.isnan(grad[0, :3]).all()
        assert row_loss[0, 3] == 0 and not grad[0, 3].any()


def test_the_others_class_far_below_the_list():
    """ln p_R = -1000 has a loss and a gradient though p_R itself is no number in 64 bits; mask values, -inf or finite, have neither."""
    x = np.array([[[0.0, 0.0, -1000.0, -1000.0]]])
    value, index = np.log(np.array([[[0.3, 0.3]]])), np.array([[[0, 1]]])
    loss, _, grad = heads.distill_topk(x, value, index, True)
    assert np.allclose(loss, 0.6 * np.log(0.6) + 0.4 * (np.log(0.4) + 1000 - np.log(2) + np.log(2)) - 0.6 * np.log(0.5) - 0.6 * np.log(2))
    assert np.allclose(grad[0, 0], [0.2, 0.2, -0.2, -0.2])
    for mask in (-np.inf, float(np.finfo(np.float32).min), -2e30):
        x[0, 0, 2:] = mask
        loss, _, grad = heads.distill_topk(x, value, index, True)
        assert np.allclose(loss, 0.6 * (np.log(0.3) + np.log(2))) and np.allclose(grad[0, 0], [0, 0, 0, 0])
