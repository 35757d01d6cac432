"""The gate with a balance bias, its kernel for many tokens: loads of four and of 16 bytes, equal keys, groups of two lanes."""
import numpy as np
import pytest
import torch

from test_gpu_route_biased import Gate, test_against_the_oracle as against_the_oracle

pytestmark = pytest.mark.gpu


# a wavefront per token at any address; a row of lanes per token where the loads are aligned; and at any address
@pytest.mark.parametrize("T", [2100, 3001, 8195])
@pytest.mark.parametrize("E,n_group,topk_group,k", [(128, 4, 2, 6), (256, 8, 4, 8), (384, 1, 1, 8)])
def test_logits_and_bias_at_any_address(E, n_group, topk_group, k, T):
    g = Gate(E, n_group, topk_group, k, "sigmoid", T, seed=3)
    logits, bias = torch.randn(T, E, generator=torch.Generator().manual_seed(1)).cuda(), torch.randn(E, generator=torch.Generator().manual_seed(2)).cuda() / 16
    want = g.run(logits, bias)
    for offset in (1, 2, 3):
        a, b = torch.empty(T * E + 4, device="cuda")[offset:offset + T * E].view(T, E), torch.empty(E + 4, device="cuda")[4 - offset:4 - offset + E]
        a.copy_(logits), b.copy_(bias)
        for x, y in ((a, bias), (logits, b), (a, b)):
            got = g.run(x, y)
            # sigmoid scores do not depend on the order of the lanes: the same choices, and weights whose sums are in another order
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[2], want[2]) and np.abs(got[1] - want[1]).max() < 1e-6
    g.L.close()


@pytest.mark.parametrize("E,n_group,T", [(64, 1, 3001), (256, 8, 3001), (384, 1, 3001), (500, 1, 8195), (176, 8, 8195), (48, 4, 8195)])
def test_equal_keys_go_to_the_lowest_expert(E, n_group, T):
    g = Gate(E, n_group, max(1, n_group // 2), 8, "sigmoid", T, lost=False)
    top, w, _ = g.run(torch.zeros(T, E, device="cuda"), torch.zeros(E, device="cuda"))
    assert (top == np.arange(8)).all() and (w == 0.125).all()
    g.L.close()


# groups of two lanes with loads of four bytes
@pytest.mark.parametrize("E,k", [(16, 3), (48, 5), (176, 8), (240, 16), (464, 6)])
def test_eight_groups_of_experts_that_are_no_multiple_of_64(E, k):
    against_the_oracle(E, 8, 4, k, "sigmoid" if k % 2 else "softmax", 8195)
