"""The layer with the balanced gate and 4-bit experts, stage by stage against the oracle: eager, and one captured graph across
map changes."""
import numpy as np
import pytest
import torch

import synth
from harness import f64, rel_err
from oracle import mx_oracle as mx
from oracle import revive_oracle as orc
from synth.resident_mx import ResidentMxLayer
from test_gpu_mx import check_ffn
from test_gpu_route_biased import resolved

pytestmark = pytest.mark.gpu

GROUPED = synth.scaled(synth.get_config("c3"), H=576, E=32, k=4, I=192, I_shared=320, n_ranks=8, slots_per_rank=5, max_replicas=3, n_group=4, topk_group=2)
SOFTMAX = synth.scaled(synth.get_config("c2"), H=320, E=24, k=3, I=64, I_shared=0, n_ranks=8, slots_per_rank=4, max_replicas=3)


def check(g):
    """Every stage from what the stage before left on the device."""
    c, b = g.cfg, {n: None if t is None else t.clone() for n, t in g.buf.items()}
    s = orc.scores(f64(b["logits"]), c.score_fn)
    m = g_map(g)
    key = mx.biased_keys(s, f64(g.bias), m.l2p_count)
    top, phys = b["topk_logical"].cpu().numpy(), b["topk_phys"].cpu().numpy()
    ok = resolved(s, key, c.n_group, c.topk_group, c.k)
    ref = orc.select_topk(key, c.k, c.n_group, c.topk_group)
    assert ok.mean() > 0.9 or c.T < 50
    assert np.array_equal(top[ok], ref[ok]) and np.array_equal(phys, orc.remap(top, m))
    want = mx.biased_weights(s, top, True)
    assert (np.abs(f64(b["topk_weight"]) - want) <= 16 * 2.0 ** -24 * want).all()
    offsets, dst, src = orc.dispatch_indices(phys, c.P)
    n = int(offsets[-1])
    assert np.array_equal(b["slot_offsets"].cpu().numpy(), offsets) and np.array_equal(b["dst_row"].cpu().numpy().reshape(dst.shape), dst)
    assert np.array_equal(b["src_of"].cpu().numpy()[:n], np.asarray(src)[:n])
    x, y = mx.rounded(f64(g.x)), f64(b["y_perm"])
    for p in np.nonzero(np.diff(offsets))[0]:
        a, e = offsets[p], offsets[p + 1]
        w = mx.expert_values({name: f64(t) for name, t in synth.draw_expert(c, int(g.p2l[p]), g.device).items()})
        check_ffn(y[a:e], x[np.asarray(src)[a:e] // c.k], w, ("slot", p))
    shared = None
    if c.I_shared:
        shared = f64(b["y_shared"])
        check_ffn(shared, x, mx.expert_values({name: f64(t) for name, t in synth.draw_shared(c, g.device).items()}), "shared")
    out = orc.combine(y, dst, f64(b["topk_weight"]), shared)
    # fp32 sums of k + 1 terms, one rounding to bf16 (2^-9)
    assert rel_err(f64(b["out"]), out) < 2.0 ** -8
    return b


def g_map(g):
    c = g.cfg
    return orc.build_map(g.p2l, g.failed, c.slots_per_rank, c.E, c.max_replicas, expert_failed=g.expert_failed)


@pytest.mark.parametrize("T", [1, 16, 17, 301, 700])
@pytest.mark.parametrize("cfg", [GROUPED, SOFTMAX], ids=["grouped", "softmax"])
def test_layer(cfg, T):
    g = ResidentMxLayer(synth.scaled(cfg, T=T))
    g.forward()
    check(g)
    g.close()


@pytest.mark.parametrize("T", [7, 96, 1024])
def test_one_graph_serves_every_map(T):
    g = ResidentMxLayer(synth.scaled(GROUPED, T=T), failed=[])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    g.capture(stream)
    for failed in ([], [5], [2, 5], [5]):
        g.set_failed(failed, stream=stream)
        g.buf["out"].fill_(7.0)
        torch.cuda.synchronize()
        g.replay(stream)
        stream.synchronize()
        replayed = check(g)
        g.buf["out"].zero_()
        g.forward()
        torch.cuda.synchronize()
        for name in ("topk_logical", "topk_weight", "topk_phys", "out"):
            assert torch.equal(g.buf[name], replayed[name]), name
    g.close()
