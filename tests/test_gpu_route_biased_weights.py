"""Weights of the gate with a balance bias where the chosen experts' scores are small, in both of its kernels."""
import numpy as np
import pytest
import torch

from harness import f64
from oracle import revive_oracle as orc
from test_gpu_route_biased import Gate

pytestmark = pytest.mark.gpu


def score64(logits, score_fn):
    with np.errstate(over="ignore", invalid="ignore"):
        return orc.scores(logits, score_fn)


def weights(E, T, k, score_fn, logits, lost, renormalise, seed=0):
    """Experts chosen by the bias alone: (their weights, logits and scores)."""
    g = Gate(E, 1, 1, k, score_fn, T, seed=seed, lost=False)
    g.L.update_map(np.zeros(1, dtype=np.uint8), expert_failed=lost)
    bias = np.random.default_rng(seed).permutation(E) * 4.0
    d = torch.from_numpy(logits).float().cuda()
    top, w, _ = g.run(d, torch.from_numpy(bias).float().cuda(), renormalise)
    z = np.take_along_axis(f64(d), top, axis=1)
    ref = np.argsort(-np.where(lost != 0, -1, bias), kind="stable")[:k]
    assert (top == ref[None, :]).all()
    g.L.close()
    return w, z, np.take_along_axis(score64(f64(d), score_fn), top, axis=1)


KERNELS = [(64, 5), (256, 40), (500, 6), (64, 3001), (320, 3002), (500, 8195)]


@pytest.mark.parametrize("E,T", KERNELS)
def test_softmax_weights_far_below_an_expert_that_is_not_chosen(E, T):
    """The largest logit is a lost expert's, or one that the bias keeps back: the others' scores underflow, their shares do not."""
    rng = np.random.default_rng(E)
    lost = np.zeros(E, dtype=np.uint8)
    lost[3] = 1
    for gap in (80.0, 95.0, 120.0, 1e4):
        logits = rng.standard_normal((T, E))
        logits[:, 3] += gap
        w, z, _ = weights(E, T, 6, "softmax", logits, lost, True, seed=E)
        e = np.exp(z - z.max(axis=1, keepdims=True))
        want = e / e.sum(axis=1, keepdims=True)
        assert (np.abs(w - want) <= 16 * 2.0 ** -24 * want).all(), gap
        w, z, s = weights(E, T, 6, "softmax", logits, lost, False, seed=E)
        assert (np.abs(w - s) <= 16 * 2.0 ** -24 * s + 2.0 ** -126).all(), gap


@pytest.mark.parametrize("E,T", KERNELS)
def test_sigmoid_weights_of_very_negative_logits(E, T):
    """Scores below the least normal number: their shares are those of exp(z), and by themselves they are zero."""
    rng = np.random.default_rng(E)
    lost = np.zeros(E, dtype=np.uint8)
    for at in (-20.0, -40.0, -86.0, -95.0, -110.0, -1e4):
        logits = rng.standard_normal((T, E)) + at
        logits[:, 7] = -np.inf
        w, z, s = weights(E, T, 6, "sigmoid", logits, lost, True, seed=E)
        e = np.exp(z - z.max(axis=1, keepdims=True)) / (1 + np.exp(z))
        want = e / e.sum(axis=1, keepdims=True)
        assert (np.abs(w - want) <= 16 * 2.0 ** -24 * want).all(), at
        w, z, s = weights(E, T, 6, "sigmoid", logits, lost, False, seed=E)
        assert (np.abs(w - s) <= 16 * 2.0 ** -24 * s + 2.0 ** -126).all(), at


@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
def test_weights_of_nothing_but_minus_infinity(score_fn):
    """0 / 0 renormalised, as in the gate without a bias; zero otherwise."""
    for T in (4, 3001):
        logits = np.zeros((T, 64))
        lost = np.zeros(64, dtype=np.uint8)
        bias = np.random.default_rng(0).permutation(64)
        logits[:, np.argsort(-bias)[:6]] = -np.inf  # the chosen ones
        w, _, _ = weights(64, T, 6, score_fn, logits, lost, True)
        assert np.isnan(w).all()
        w, _, _ = weights(64, T, 6, score_fn, logits, lost, False)
        assert (w == 0).all()
