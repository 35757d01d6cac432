"""Options of the resident layer with the balanced gate and 4-bit experts."""
import pytest
import torch

import synth
from synth.resident_mx import ResidentMxLayer
from test_gpu_mx_layer import GROUPED, SOFTMAX

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [5, 301])
def test_resident_layer_without_the_shared_expert(T):
    g = ResidentMxLayer(synth.scaled(GROUPED, T=T))
    with_shared = g.forward()["out"].clone()
    y_perm, y_shared = g.buf["y_perm"].clone(), g.buf["y_shared"].clone()
    g.buf["y_shared"].fill_(3.0)
    alone = g.forward(shared=False)["out"].clone()
    assert torch.equal(g.buf["y_perm"], y_perm) and bool((g.buf["y_shared"] == 3.0).all())
    want = g.layer.combine(y_perm, g.buf["dst_row"], g.buf["topk_weight"], None, T)
    assert torch.equal(alone, want) and not torch.equal(alone, with_shared)
    for overlap in (True, False):
        assert torch.equal(g.forward(overlap_shared=overlap)["out"], with_shared)
    assert torch.equal(g.buf["y_shared"], y_shared)
    g.close()


@pytest.mark.parametrize("cfg", [GROUPED, SOFTMAX], ids=["grouped", "softmax"])
def test_resident_layer_marks_its_stages(cfg):
    g = ResidentMxLayer(synth.scaled(cfg, T=64))
    marks = []
    g.forward(stage_marks=marks)
    torch.cuda.synchronize()
    assert len(marks) == 5 and all(a.elapsed_time(b) >= 0 for a, b in zip(marks, marks[1:]))
    with pytest.raises(TypeError):
        g.forward(no_such_option=True)
    g.close()
