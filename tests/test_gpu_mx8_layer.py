"""The block in 8-bit form (projection with residual, norm, balanced gate, 8-bit experts, norm with residual), stage by stage against
the oracle from what the stage before left on the device: eager, and one captured graph across map changes."""
import numpy as np
import pytest
import torch

import synth
from harness import f64, rel_err
from oracle import mx8_oracle as mx
from oracle import mx_oracle
from oracle import revive_oracle as orc
from paper_2602_21140_amd import mx8_quantize
from synth.resident_mx8 import ResidentMx8Block
from test_gpu_mx8 import check_ffn, sum_error
from test_gpu_mx_layer import GROUPED, SOFTMAX, g_map
from test_gpu_norm import check as check_norm
from test_gpu_route_biased import resolved

pytestmark = pytest.mark.gpu


def check(g):
    c, b = g.cfg, {n: t.clone() if isinstance(t, torch.Tensor) else t if t is None else tuple(v.clone() for v in t) for n, t in g.buf.items()}
    # the projection: the sums' error, two additions, one rounding
    x, w = mx.rounded(f64(g.x)), mx.rounded(f64(g.w_attention))
    z = x @ w.T + f64(g.attention_bias)
    want = z + f64(g.residual)
    off = np.abs(f64(b["stream"]) - want)
    assert (off <= sum_error(x, w.T) * 1.01 + 2.0 ** -22 * (np.abs(z) + np.abs(want)) + 2.0 ** -8 * np.abs(want)).all()
    check_norm(b["stream"], None, g.norms[0], g.EPS, None, b["x"], *b["x_form"])
    s = orc.scores(f64(b["logits"]), c.score_fn)
    m = g_map(g)
    key = mx_oracle.biased_keys(s, f64(g.bias), m.l2p_count)
    top, phys = b["topk_logical"].cpu().numpy(), b["topk_phys"].cpu().numpy()
    ok = resolved(s, key, c.n_group, c.topk_group, c.k)
    ref = orc.select_topk(key, c.k, c.n_group, c.topk_group)
    assert ok.mean() > 0.9 or c.T < 50
    assert np.array_equal(top[ok], ref[ok]) and np.array_equal(phys, orc.remap(top, m))
    weights = mx_oracle.biased_weights(s, top, True)
    assert (np.abs(f64(b["topk_weight"]) - weights) <= 16 * 2.0 ** -24 * weights).all()
    offsets, dst, src = orc.dispatch_indices(phys, c.P)
    n = int(offsets[-1])
    assert np.array_equal(b["slot_offsets"].cpu().numpy(), offsets) and np.array_equal(b["dst_row"].cpu().numpy().reshape(dst.shape), dst)
    x, y = mx.values(*(t.cpu().numpy() for t in b["x_form"])), f64(b["y_perm"])
    for p in np.nonzero(np.diff(offsets))[0]:
        a, e = offsets[p], offsets[p + 1]
        v = mx.expert_values({name: f64(t) for name, t in synth.draw_expert(c, int(g.p2l[p]), g.device).items()})
        check_ffn(y[a:e], x[np.asarray(src)[a:e] // c.k], v, ("slot", p))
    shared = None
    if c.I_shared:
        shared = f64(b["y_shared"])
        check_ffn(shared, x, mx.expert_values({name: f64(t) for name, t in synth.draw_shared(c, g.device).items()}), "shared")
    out = orc.combine(y, dst, f64(b["topk_weight"]), shared)
    assert n == c.N and rel_err(f64(b["out"]), out) < 2.0 ** -8  # fp32 sums of k + 1 terms, one rounding to bf16
    check_norm(b["out"], b["stream"], g.norms[1], g.EPS, b["next_stream"], b["next_x"], *b["next_form"])
    return b


@pytest.mark.parametrize("T", [1, 16, 17, 301, 700])
@pytest.mark.parametrize("cfg", [GROUPED, SOFTMAX], ids=["grouped", "softmax"])
def test_block(cfg, T):
    g = ResidentMx8Block(synth.scaled(cfg, T=T))
    g.forward()
    b = check(g)
    # what the norm gives the experts is what quantising its bf16 output gives
    assert all(torch.equal(a, c) for a, c in zip(b["x_form"], mx8_quantize(b["x"])))
    marks = []
    g.forward(stage_marks=marks)
    alone = g.forward(shared=False)["out"].clone()
    assert len(marks) == 7
    want = g.layer.combine(b["y_perm"], b["dst_row"], b["topk_weight"], None, T)
    assert torch.equal(alone, want)
    with pytest.raises(TypeError):
        g.forward(no_such_option=True)
    g.close()


@pytest.mark.parametrize("T", [7, 96, 1024])
def test_one_graph_serves_every_map(T):
    g = ResidentMx8Block(synth.scaled(GROUPED, T=T), failed=[])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    g.capture(stream)
    for failed in ([], [5], [2, 5], [5]):
        g.set_failed(failed, stream=stream)
        g.buf["next_x"].fill_(7.0)
        torch.cuda.synchronize()
        g.replay(stream)
        stream.synchronize()
        replayed = check(g)
        g.buf["next_x"].zero_()
        g.forward()
        torch.cuda.synchronize()
        for name in ("topk_logical", "topk_weight", "topk_phys", "out", "next_stream", "next_x"):
            assert torch.equal(g.buf[name], replayed[name]), name
    g.close()
