"""The gate with a balance bias against the oracle in 64 bits."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx_oracle as mx
from oracle import revive_oracle as orc
from paper_2602_21140_amd import ReviveLayer

pytestmark = pytest.mark.gpu


class Gate:
    def __init__(self, E, n_group, topk_group, k, score_fn, T, seed=0, lost=True, route_scale=1.0):
        rng = np.random.default_rng(seed)
        slots = -(-E * 5 // 4)
        self.p2l = np.concatenate([np.arange(E), rng.permutation(E)[:slots - E]]).astype(np.int32)  # some experts twice
        self.cfg = SimpleNamespace(T=T, H=64, E=E, k=k, I=64, I_shared=0, n_ranks=1, slots_per_rank=slots, max_replicas=2,
                                   score_fn=score_fn, n_group=n_group, topk_group=topk_group, dtype="bf16")
        self.L = ReviveLayer(self.cfg, route_scale=route_scale)
        self.L.set_placement(self.p2l)
        self.lost = np.zeros(E, dtype=np.uint8)
        if lost:
            self.lost[rng.permutation(E)[:E // 16]] = 1
        self.L.update_map(np.zeros(1, dtype=np.uint8), expert_failed=self.lost)
        self.map = orc.build_map(self.p2l, np.zeros(1, dtype=np.uint8), slots, E, 2, expert_failed=self.lost)

    def run(self, logits, bias, renormalise=True, **kw):
        _, top, w, phys = self.L.route_biased(None, None, bias, len(logits), renormalise=renormalise, logits=logits, logits_given=True, **kw)
        return top.cpu().numpy(), f64(w), phys.cpu().numpy()


def resolved(s, key, n_group, topk_group, k):
    """Tokens whose choices are in an order that fp32 resolves.  A score is off by up to 8 units of 2^-24 of its size (exp,
    division) and a key by a rounding more: two keys that are not equal keep their order if they are 32 units of the row's
    largest apart.  Groups: twice that between the last that is kept and the first that is not, whose sums may be equal ones of
    unlike keys."""
    unit = 32 * 2.0 ** -24 * np.maximum(np.where(np.isfinite(key), np.abs(key), 0).max(axis=1), s.max(axis=1))
    ok = np.ones(len(key), dtype=bool)
    if topk_group < n_group:
        groups = np.stack([orc.group_scores(row, n_group) for row in key])
        g = -np.sort(-groups, axis=1)
        ok = g[:, topk_group - 1] - g[:, topk_group] >= 2 * unit
        dropped = (groups < g[:, topk_group - 1:topk_group]).repeat(key.shape[1] // n_group, axis=1)
        key = np.where(dropped, -np.inf, key)
    order = -np.sort(-key, axis=1)[:, :k + 1]
    with np.errstate(invalid="ignore"):
        d = order[:, :-1] - order[:, 1:]
    return ok & ~((d > 0) & (d < unit[:, None])).any(axis=1)


SHAPES = [(64, 8, 3, 6), (256, 8, 4, 8), (512, 8, 4, 8), (192, 4, 2, 5), (200, 8, 2, 16), (256, 2, 1, 8), (32, 8, 8, 16), (512, 32, 8, 32),
          (320, 20, 3, 8), (61, 1, 1, 1), (384, 1, 1, 8), (500, 1, 1, 32), (16, 1, 1, 2), (2, 1, 1, 1), (130, 1, 1, 4), (48, 4, 2, 3),
          (400, 2, 1, 8), (96, 2, 1, 12), (128, 1, 1, 16)]


@pytest.mark.parametrize("T", [1, 17, 300, 4100])
@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,n_group,topk_group,k", SHAPES)
def test_against_the_oracle(E, n_group, topk_group, k, score_fn, T):
    g = Gate(E, n_group, topk_group, k, score_fn, T, seed=E + k, route_scale=2.5)
    rng = np.random.default_rng(E)
    logits = torch.from_numpy(np.round(rng.standard_normal((T, E)) * 8) / 8).float().cuda()  # eighths: many ties
    bias = torch.from_numpy(np.round(rng.standard_normal(E) * 2) / (16 if score_fn == "sigmoid" else 8 * E)).float().cuda()
    s = orc.scores(f64(logits), score_fn)
    key = mx.biased_keys(s, f64(bias), g.map.l2p_count)
    ok = resolved(s, key, n_group, topk_group, k)
    assert ok.mean() > 0.5 or T < 50
    ref = orc.select_topk(key, k, n_group, topk_group)
    for renormalise in (True, False):
        top, w, phys = g.run(logits, bias, renormalise)
        assert np.array_equal(top[ok], ref[ok])
        assert np.array_equal(phys[ok], orc.remap(ref, g.map)[ok])
        want = mx.biased_weights(s, ref, renormalise, 2.5)
        # a score is within 8 units of 2^-24, their sum and the quotient add fewer than as many again
        assert (np.abs(w - want)[ok] <= 16 * 2.0 ** -24 * want[ok] + 1e-38).all()
    g.L.close()


# many tokens: experts that are no multiple of 64, or of 16, or one more than a form of the kernel holds
@pytest.mark.parametrize("E,n_group,topk_group,k", [(16, 1, 1, 2), (61, 1, 1, 1), (65, 1, 1, 16), (100, 1, 1, 4), (48, 4, 2, 3), (200, 8, 2, 16),
                                                    (208, 2, 1, 8), (400, 2, 1, 8), (500, 1, 1, 16), (320, 4, 3, 7), (511, 1, 1, 5)])
def test_many_tokens(E, n_group, topk_group, k):
    test_against_the_oracle(E, n_group, topk_group, k, "sigmoid" if k % 2 else "softmax", 6147)


@pytest.mark.parametrize("E,n_group,topk_group,k", [(16, 1, 1, 2), (61, 1, 1, 1), (65, 1, 1, 16), (48, 4, 2, 3), (208, 2, 1, 8), (400, 2, 1, 8),
                                                    (500, 1, 1, 16), (511, 1, 1, 5)])
def test_a_row_of_lanes_per_token(E, n_group, topk_group, k):
    test_against_the_oracle(E, n_group, topk_group, k, "softmax" if k % 2 else "sigmoid", 8195)


@pytest.mark.parametrize("T", [2999, 3000])
@pytest.mark.parametrize("E,n_group,topk_group,k", [(256, 8, 4, 8), (320, 1, 1, 16), (512, 2, 1, 12)])
def test_both_sides_of_the_kernels_line(E, n_group, topk_group, k, T):
    test_against_the_oracle(E, n_group, topk_group, k, "softmax", T)


def test_more_tokens_than_the_workgroups_take_at_once():
    test_against_the_oracle(64, 1, 1, 4, "softmax", 33001)


def test_logits_and_bias_at_any_address():
    T, E = 2100, 128
    g = Gate(E, 4, 2, 6, "sigmoid", T, seed=3)
    logits, bias = torch.randn(T, E, generator=torch.Generator().manual_seed(1)).cuda(), torch.randn(E, generator=torch.Generator().manual_seed(2)).cuda() / 16
    want = g.run(logits, bias)
    for offset in (1, 2, 3):
        a, b = torch.empty(T * E + 4, device="cuda")[offset:offset + T * E].view(T, E), torch.empty(E + 4, device="cuda")[4 - offset:4 - offset + E]
        a.copy_(logits), b.copy_(bias)
        for x, y in ((a, bias), (logits, b), (a, b)):
            got = g.run(x, y)
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[2], want[2]) and np.abs(got[1] - want[1]).max() < 1e-6
    g.L.close()


@pytest.mark.parametrize("score_fn", ["softmax", "sigmoid"])
def test_no_bias_chooses_as_the_gate_without(score_fn):
    g = Gate(256, 8, 4, 8, score_fn, 2000, seed=5)
    logits = torch.randn(2000, 256, generator=torch.Generator().manual_seed(1)).cuda()
    s = orc.scores(f64(logits), score_fn)
    key = mx.biased_keys(s, np.zeros(256), g.map.l2p_count)
    ok = resolved(s, key, 8, 4, 8)
    _, top, w, phys = g.L.route(None, None, 2000, logits=logits, logits_given=True)
    mine = g.run(logits, torch.zeros(256, device="cuda"))
    assert ok.mean() > 0.9
    for a, b in ((top, mine[0]), (phys, mine[2])):
        assert np.array_equal(a.cpu().numpy()[ok], b[ok])
    assert np.abs(f64(w) - mine[1])[ok].max() < 1e-6
    g.L.close()


def test_equal_keys_go_to_the_lowest_expert():
    for E, n_group in ((64, 1), (256, 8), (500, 1)):
        g = Gate(E, n_group, max(1, n_group // 2), 8, "sigmoid", 40, lost=False)
        top, w, _ = g.run(torch.zeros(40, E, device="cuda"), torch.zeros(E, device="cuda"))
        assert (top == np.arange(8)).all() and (w == 0.125).all()
        g.L.close()


def test_the_router_product_and_the_token_offset():
    g = Gate(64, 1, 1, 4, "sigmoid", 50, seed=2)
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    w = (torch.randn(64, 64, generator=torch.Generator().manual_seed(4)) / 8).to(torch.bfloat16).cuda()
    bias = torch.randn(64, generator=torch.Generator().manual_seed(5)).cuda() * 0.1
    logits, top, wt, phys = g.L.route_biased(x, w, bias, 50)
    want = g.L.route(x, w, 50)[0]
    assert torch.equal(logits, want)
    again = g.run(logits, bias)
    assert np.array_equal(top.cpu().numpy(), again[0]) and np.array_equal(phys.cpu().numpy(), again[2])
    g.L.set_token_offset(7)
    shifted = g.run(logits, bias)
    m = g.map
    for t in range(50):
        for j, e in enumerate(shifted[0][t]):
            assert shifted[2][t, j] == m.l2p_table[e, (t + 7) % m.l2p_count[e]]
    g.L.close()


@pytest.mark.parametrize("E,n_group", [(64, 1), (256, 8), (500, 1)])
def test_keys_that_are_no_numbers_come_last(E, n_group):
    k = 8
    g = Gate(E, n_group, max(1, n_group // 2), k, "sigmoid", 6, lost=False, seed=8)
    logits = torch.randn(6, E, generator=torch.Generator().manual_seed(3)).cuda()
    logits[1] = float("nan")
    logits[2, ::2] = float("nan")
    logits[3, 5] = float("inf")
    logits[4] = float("-inf")
    bias = torch.zeros(E, device="cuda")
    bias[9] = float("-inf")
    top, w, phys = g.run(logits, bias)
    for t in range(6):
        assert len(set(top[t])) == k and (top[t] >= 0).all() and (top[t] < E).all() and (phys[t] >= 0).all()
    assert (top[1] == np.arange(k)).all() and np.isnan(w[1]).all()   # nothing but NaN: ascending ids
    assert (top[2] % 2 == 1).all() and np.isfinite(w[2]).all()
    assert top[3, 0] == 5
    assert 9 not in top[0] and 9 not in top[4]
    g.L.close()


def test_a_lost_expert_is_never_chosen_and_comes_back():
    g = Gate(64, 1, 1, 4, "softmax", 500, lost=False)
    logits = torch.randn(500, 64, generator=torch.Generator().manual_seed(1)).cuda()
    bias = torch.zeros(64, device="cuda")
    bias[3] = 10.0
    assert (g.run(logits, bias)[0][:, 0] == 3).all()
    failed = np.zeros(64, dtype=np.uint8)
    failed[3] = 1
    g.L.update_map(np.zeros(1, dtype=np.uint8), expert_failed=failed)
    assert not (g.run(logits, bias)[0] == 3).any()
    g.L.update_map(np.zeros(1, dtype=np.uint8))
    assert (g.run(logits, bias)[0][:, 0] == 3).all()
    g.L.close()


def test_refusals():
    g = Gate(16, 1, 1, 2, "sigmoid", 4)
    logits, bias = torch.zeros(4, 16, device="cuda"), torch.zeros(16, device="cuda")
    out = [torch.zeros(4, 2, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32)]
    good = [None, None, logits.data_ptr(), 1, bias.data_ptr(), 1, 4, *(t.data_ptr() for t in out), None]
    call = lambda a: g.L.L.revive_route_biased(g.L._ctx, *a)  # noqa: E731
    assert call(good) == 0
    for i in (2, 4, 7, 8, 9):
        assert call(good[:i] + [None] + good[i + 1:]) == -1
    assert call(good[:3] + [0] + good[4:]) == -1       # no logits and nothing to make them of
    for T in (-1, 5):
        assert call(good[:6] + [T] + good[7:]) == -1
    fresh = ReviveLayer(g.cfg)
    assert fresh.L.revive_route_biased(fresh._ctx, *good) == -3   # no map yet
    torch.cuda.synchronize()
    fresh.close()
    g.L.close()
