"""Microbatches over a layer that has no bf16 weights are refused before anything is multiplied."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from synth.resident import MicrobatchPipeline


def base(gu, dn):
    return SimpleNamespace(cfg=SimpleNamespace(T=4, P=4), p2l=np.array([0, 1, -1, 0], dtype=np.int32), gu=gu, dn=dn, device="cpu")


@pytest.mark.parametrize("gu,dn", [([None] * 4, [None] * 4), ([1, 1, None, 1], [1, None, None, 1]), ([1, 1, None, None], [1, 1, None, 1])])
def test_a_slot_with_an_expert_and_no_weights(gu, dn):
    weights = [[None if w is None else torch.zeros(1) for w in ws] for ws in (gu, dn)]
    with pytest.raises(ValueError, match="weights"):
        MicrobatchPipeline(base(*weights), 2)
