"""The layer with a balanced gate and 4-bit experts, resident in HBM, and how it compares with the bf16 one.

route_biased -> dispatch_index -> mx_expert_ffn -> combine: the experts are chosen with a bias per expert, the rows are never
permuted (the FFN finds them through src_of), and weights and activations are microscaled 4-bit floats.  The workloads, the
map updates and the graph are those of `resident.py`.

Usage: python -m synth.resident_mx [--workload c2] [--tokens T] [--steps K]
"""
from __future__ import annotations

import argparse
import json
from typing import Dict, List, Optional

import numpy as np
import torch

import synth
from paper_2602_21140_amd.binding import mx_pack_expert
from synth.resident import ResidentLayer


class ResidentMxLayer(ResidentLayer):
    def __init__(self, cfg: synth.LayerConfig, device="cuda:0", **kw):
        super().__init__(cfg, device=device, with_weights=False, **kw)
        L, T, P = self.layer, cfg.T, cfg.P
        # what balancing leaves: offsets of about the distance between neighbouring scores
        z = torch.randn(cfg.E, generator=torch.Generator().manual_seed(cfg.seed)) / (16 if cfg.score_fn == "sigmoid" else 4 * cfg.E)
        self.bias = z.to(device)
        self.mx_gu: List[Optional[torch.Tensor]] = [None] * P
        self.mx_dn: List[Optional[torch.Tensor]] = [None] * P
        for e in range(cfg.E):
            slots = np.nonzero(self.p2l == e)[0]
            if slots.size:
                w = synth.draw_expert(cfg, e, device)
                g, d = mx_pack_expert(w["gate"], w["up"], w["down"])
                for i, p in enumerate(slots):  # each replica owns its own copy of the bits
                    self.mx_gu[p], self.mx_dn[p] = (g, d) if i == 0 else (g.clone(), d.clone())
        L.set_mx_expert_weights(self.mx_gu, self.mx_dn)
        sh = synth.draw_shared(cfg, device)
        self.mx_sh = (None, None) if sh is None else mx_pack_expert(sh["gate"], sh["up"], sh["down"])
        self.buf["x_perm"] = None
        if sh is not None:
            self.buf["y_shared"] = L.empty(T, cfg.H)

    def forward(self, logits: Optional[torch.Tensor] = None, shared=True, stream=None, overlap_shared=True,
                stage_marks: Optional[list] = None) -> Dict[str, Optional[torch.Tensor]]:
        """As ResidentLayer.forward, in 4-bit form.  The shared expert is served by the launches of the routed ones, so that
        overlap_shared, which would put it on a stream beside them, changes nothing here."""
        L, b, T = self.layer, self.buf, self.cfg.T
        main = torch.cuda.current_stream() if stream is None else stream
        given = logits is not None
        sh = self.mx_sh if shared else (None, None)
        y_shared = b["y_shared"] if sh[0] is not None else None

        def mark():
            if stage_marks is not None:
                ev = torch.cuda.Event(enable_timing=True)
                ev.record(main)
                stage_marks.append(ev)

        mark()
        if given:
            with torch.cuda.stream(main):
                b["logits"].copy_(logits)
        L.route_biased(None if given else self.x, None if given else self.w_router_packed, self.bias, T, logits=b["logits"],
                       logits_given=given, out=(b["topk_logical"], b["topk_weight"], b["topk_phys"]), stream=main)
        mark()
        L.dispatch_index(b["topk_phys"], T, out=(b["slot_offsets"], b["dst_row"], b["src_of"]), stream=main)
        mark()
        L.mx_expert_ffn(self.x, b["src_of"], b["slot_offsets"], T, *sh, out=(b["y_perm"], y_shared), stream=main)
        mark()
        L.combine(b["y_perm"], b["dst_row"], b["topk_weight"], y_shared, T, out=b["out"], stream=main)
        mark()
        return b


def _ms_per_step(layer, steps: int) -> float:
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    layer.forward(stream=stream)
    stream.synchronize()
    layer.capture(stream)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        layer.replay(stream)
    begin.record(stream)
    for _ in range(steps):
        layer.replay(stream)
    end.record(stream)
    end.synchronize()
    return begin.elapsed_time(end) / steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="c2", choices=[n for n, c in synth.CONFIGS.items() if c.dtype == "bf16"])
    ap.add_argument("--tokens", type=int, default=None)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    cfg = synth.get_config(args.workload)
    if args.tokens:
        cfg = synth.scaled(cfg, T=args.tokens)
    line, outs = {"workload": cfg.name, "tokens": cfg.T}, {}
    for name, kind in (("bf16", ResidentLayer), ("mx", ResidentMxLayer)):
        g = kind(cfg)
        gu, dn = (g.gu, g.dn) if name == "bf16" else (g.mx_gu, g.mx_dn)
        line[f"{name}_ms_per_step"] = round(_ms_per_step(g, args.steps), 4)
        line[f"{name}_weight_gib"] = round(sum(w.numel() * w.element_size() for w in gu + dn if w is not None) / 2 ** 30, 3)
        if name == "mx":
            g.bias.zero_()  # the bf16 layer's choices, to compare the outputs
            g.forward(logits=outs["logits"])
        outs.setdefault("logits", g.buf["logits"].clone())
        outs[name] = (g.buf["topk_logical"].sort(dim=1).values, g.buf["out"].float())
        g.close()
    same = (outs["bf16"][0] == outs["mx"][0]).all(dim=1)
    a, b = outs["bf16"][1][same], outs["mx"][1][same]
    line["tokens_with_the_same_experts"] = float(same.float().mean())
    line["relative_rms_difference"] = float((a - b).pow(2).mean().sqrt() / a.pow(2).mean().sqrt())
    print(json.dumps(line))


if __name__ == "__main__":
    main()
