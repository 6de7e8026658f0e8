"""Pins for the oracle's gradient norm and clipping -- no GPU: hand examples, the library's own norm and clipping, range, masks."""
import numpy as np
import pytest
import torch

import oracle


def test_hand_examples():
    norm, factor, each = oracle.grad_norm([[[3.0], [9.0]], [[4.0, 0.0]]], [[1, 0], None], 2.5)
    assert (norm, factor, each) == (5.0, 0.5, [3.0, 4.0])
    assert oracle.grad_norm([[[3.0]]], [None], 3.0) == (3.0, 1.0, [3.0])
    assert oracle.grad_norm([], [], 0.0) == (0.0, 1.0, [])
    assert oracle.grad_norm([np.zeros((0, 3)), np.ones((2, 2))], [None, [0, 0]], 0.0) == (0.0, 1.0, [0.0, 0.0])


def test_the_library_s_norm_and_clipping():
    rng = np.random.default_rng(3)
    ts = [torch.tensor(rng.normal(size=s), requires_grad=True) for s in ((7, 3), (5,), (4, 2, 3))]
    for t in ts:
        t.grad = torch.tensor(rng.normal(size=t.shape))
    raw = [t.grad.numpy().copy() for t in ts]
    norm, factor, each = oracle.grad_norm(raw, [None] * 3, 1.5)
    got = torch.nn.utils.clip_grad_norm_(ts, 1.5)
    assert norm == pytest.approx(float(got), rel=1e-14)
    for t, g, e in zip(ts, raw, each):
        assert e == pytest.approx(np.linalg.norm(g), rel=1e-14)
        np.testing.assert_allclose(oracle.grad_clip(g, None, factor, None), t.grad.numpy(), rtol=1e-6)      # theirs adds 1e-6 to the norm
    clipped = [oracle.grad_clip(g, None, factor, None) for g in raw]
    assert oracle.grad_norm(clipped, [None] * 3, 9.0)[0] == pytest.approx(1.5, rel=1e-14)


def test_range_masks_and_values_that_are_not_finite():
    for size in (1e-200, 1e-30, 1e30, 1e200):
        assert oracle.grad_norm([np.array([3.0, 4.0]) * size], [None], np.inf)[0] == pytest.approx(5.0 * size, rel=1e-14)
    bad = np.array([[1.0, 2.0], [np.inf, 0.0], [2.0, np.nan]])
    assert oracle.grad_norm([bad], [[1, 0, 0]], 10.0)[:2] == (pytest.approx(np.sqrt(5.0)), 1.0)
    assert oracle.grad_norm([bad], [[1, 1, 0]], 10.0)[:2] == (float("inf"), 0.0)
    assert np.isnan(oracle.grad_norm([bad], [None], 10.0)[0])
    before = np.full((3, 2), 7.0)
    assert np.array_equal(oracle.grad_clip(bad, [1, 1, 0], 0.0, before), [[0, 0], [0, 0], [7, 7]])
    assert np.array_equal(oracle.grad_clip(bad, [1, 0, 0], 0.5, before), [[0.5, 1], [7, 7], [7, 7]])
