"""The gate with a balance bias where keys are huge, infinite or no numbers, in both of its kernels.

The reference is the definition, keys and sums of groups in 64 bits and rounded to the 24 of fp32: a live expert whose key is a number
comes before one whose key is NaN or -inf, that one before a lost expert; groups in the same manner, by the sum of their two best
numbers."""
import numpy as np
import pytest
import torch

from harness import f64
from oracle import revive_oracle as orc
from test_gpu_route_biased import Gate
from test_gpu_route_biased_weights import score64

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)
# experts, groups, groups kept, choices; tokens: a wavefront per token, and a row of lanes per token (later where E is no multiple of 64)
SHAPES = [(64, 1, 1, 8, 5), (64, 8, 4, 6, 5), (256, 8, 4, 8, 7), (500, 1, 1, 8, 6), (192, 4, 2, 5, 9), (320, 20, 5, 8, 3),
          (64, 1, 1, 8, 3001), (64, 8, 4, 6, 3001), (256, 8, 4, 8, 3002), (192, 4, 2, 5, 3003), (256, 2, 1, 12, 3001),
          (500, 1, 1, 8, 8195), (176, 8, 4, 8, 8195), (48, 4, 2, 3, 8193), (208, 2, 1, 8, 8194)]


def rounded(v):
    """To fp32's 24 bits, beyond its range as well."""
    return np.float32(0.5 * v).astype(np.float64) * 2


def reference(s, bias, live, n_group, topk_group, k):
    """(chosen experts [T, k], rows whose order hangs on no less than fp32 resolves)."""
    T, E = s.shape
    with np.errstate(invalid="ignore"):
        key = s + bias[None, :]
    level = np.where(live[None, :], np.where(key > -np.inf, 2, 1), 0)
    key = rounded(np.where(level == 2, key, 0.0))

    def rank(level, value):  # best first, ties to the lower index
        return np.lexsort((np.arange(len(level)), -value, -level))

    def close(a, b):  # unequal, and closer than 32 units of 2^-24 of either or of the largest score
        return a != b and np.isfinite(a) and np.isfinite(b) and abs(a - b) < 64 * 2.0 ** -24 * max(1.0, abs(a), abs(b))

    out, ok = np.zeros((T, k), dtype=np.int32), np.ones(T, dtype=bool)
    gsz = E // n_group
    for t in range(T):
        kept = np.ones(E, dtype=bool)
        if n_group > 1:
            glevel, gvalue = np.zeros(n_group, dtype=int), np.zeros(n_group)
            for g in range(n_group):
                part = slice(g * gsz, (g + 1) * gsz)
                glevel[g] = level[t, part].max()
                numbers = np.sort(key[t, part][level[t, part] == 2])[::-1]
                gvalue[g] = rounded(numbers[:2].sum()) if len(numbers) else 0.0
            order = rank(glevel, gvalue)
            if topk_group < n_group:  # fp32 may make equal what is not, and equal ones go by their ids: all against the two at the line
                for a in order[topk_group - 1:topk_group + 1]:
                    ok[t] &= not any(glevel[a] == glevel[b] and close(gvalue[a], gvalue[b]) for b in range(n_group))
            kept = np.isin(np.arange(E) // gsz, order[:topk_group])
        order = rank(np.where(kept, level[t], -1), key[t])
        out[t] = order[:k]
        for a in order[:k + 1]:
            ok[t] &= not any(level[t, a] == level[t, b] and close(key[t, a], key[t, b]) for b in order)
    return out, ok


def check(g, logits, bias):
    c = g.cfg
    d_logits, d_bias = torch.from_numpy(logits).float().cuda(), torch.from_numpy(bias).float().cuda()
    s = score64(f64(d_logits), c.score_fn)
    live = g.map.l2p_count > 0
    # the rows are copies of a few, in another order in every four
    n = min(len(logits), 24)
    ref, ok = reference(s[:n], f64(d_bias), live, c.n_group, c.topk_group, c.k)
    assert ok.mean() > 0.25  # of the reference alone
    which = (np.arange(len(logits)) * 11) % n
    d_logits, s, ref, ok = d_logits[torch.from_numpy(which).cuda()].contiguous(), s[which], ref[which], ok[which]
    for renormalise in (True, False):
        top, w, phys = g.run(d_logits, d_bias, renormalise)
        assert np.array_equal(top[ok], ref[ok])
        assert np.array_equal(phys[ok], orc.remap(ref, g.map)[ok])
        want = np.take_along_axis(s, ref, axis=1)
        with np.errstate(invalid="ignore"):
            if renormalise:
                want = want / want.sum(axis=1, keepdims=True)
            assert np.array_equal(np.isnan(w[ok]), np.isnan(want[ok]))
            # a score, the sum and the quotient: 16 units of 2^-24 at most; below the least normal number scores are zero
            assert not (np.abs(w - want)[ok] > 16 * 2.0 ** -24 * want[ok] + 2.0 ** -126).any()


def spread(rng, T, E):
    """Logits whose scores lie far apart, every row in another order."""
    return np.stack([rng.permutation(np.linspace(-4, 4, E)) for _ in range(T)])


@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,n_group,topk_group,k,T", SHAPES)
def test_a_mask_of_the_lowest_number(E, n_group, topk_group, k, T, score_fn):
    """Experts masked by the type's lowest value are the last of the numbers, and count in their group's score."""
    g = Gate(E, n_group, topk_group, k, score_fn, T, seed=E, lost=False)
    rng = np.random.default_rng(E + 1)
    bias = np.zeros(E)
    gsz = E // n_group
    bias[1:gsz] = LOWEST                      # the first group is masked down to one expert
    bias[rng.permutation(E)[:E // 8]] = LOWEST
    bias[0] = 0.0
    logits = spread(rng, T, E)
    best = logits.argmax(axis=1)
    for t in range(0, T, 2):                  # whose score is the best of all in every other row
        logits[t, best[t]], logits[t, 0] = logits[t, 0], logits[t, best[t]]
    check(g, logits, bias)
    g.L.close()


@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,n_group,topk_group,k,T", SHAPES)
def test_huge_biases_keep_their_order(E, n_group, topk_group, k, T, score_fn):
    g = Gate(E, n_group, topk_group, k, score_fn, T, seed=E)
    rng = np.random.default_rng(E + 2)
    bias = rng.choice([LOWEST, -3.3e38, -2e38, -1.4e38, -1.1e38, -6.5e37, -4.2e37, -1e30, 0.0], E)
    check(g, spread(rng, T, E), bias)
    bias = rng.choice([LOWEST, -3.3e38, -2e38, -1e38, 1e30, 1e38, 1.5e38], E)
    check(g, spread(rng, T, E), bias)
    bias = rng.choice([-3.3e38, -2.9e38, -2.3e38, -1.6e38, -1.1e38], E)
    check(g, spread(rng, T, E), bias)
    g.L.close()


@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,n_group,topk_group,k,T", SHAPES)
def test_keys_that_are_no_numbers(E, n_group, topk_group, k, T, score_fn):
    """NaN and infinities among logits and biases: a key that is no number comes after all that are, in ascending id, also where the
    score is NaN and the bias +inf or -inf."""
    g = Gate(E, n_group, topk_group, k, score_fn, T, seed=E)
    rng = np.random.default_rng(E + 3)
    bias = np.where(rng.random(E) < 0.3, rng.choice([np.nan, -np.inf, np.inf, 3e38, LOWEST, 1e30], E), rng.choice([0.0, -0.0], E))
    bias[2], bias[5] = -np.inf, np.nan        # among the ids that a row of nothing but NaN chooses
    logits = spread(rng, T, E)
    n = min(T, 24)
    for t in range(1, n):
        kind = t % 6
        if kind == 1:
            logits[t] = np.nan
        elif kind == 2:
            logits[t, rng.random(E) < 0.5] = np.nan
        elif kind == 3:
            logits[t, rng.integers(E)] = np.inf
        elif kind == 4:
            logits[t, rng.random(E) < 0.7] = -np.inf
        elif kind == 5:
            logits[t, np.isinf(bias) & (bias > 0)] = np.nan
    check(g, logits, bias)
    g.L.close()


def test_a_live_group_comes_before_a_lost_one_whatever_its_mask():
    for T in (4, 3001):
        for value in (LOWEST, -np.inf, np.nan):
            g = Gate(64, 4, 3, 16, "sigmoid", T, lost=False)
            lost = np.zeros(64, dtype=np.uint8)
            lost[:16] = 1                     # the first group is lost, the last one masked
            lost[[17, 18, 19, 20, 21, 22, 23, 24, 25, 26, 27, 33, 34, 35, 36, 37, 38, 39, 40, 41, 42, 43]] = 1
            g.L.update_map(np.zeros(1, dtype=np.uint8), expert_failed=lost)
            g.map = orc.build_map(g.p2l, np.zeros(1, dtype=np.uint8), g.cfg.slots_per_rank, 64, 2, expert_failed=lost)
            bias = np.zeros(64)
            bias[48:] = value
            check(g, spread(np.random.default_rng(1), T, 64), bias)  # ten experts of the other two groups, then six masked ones
            g.L.close()
