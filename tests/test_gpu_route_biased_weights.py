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
