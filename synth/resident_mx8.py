"""The layer in 8-bit form with what stands around it in a transformer block, resident in HBM.

attention's output -> mx8_quantize -> mx8_linear with the residual in its epilogue -> add_rms_norm -> route_biased ->
dispatch_index -> mx8_expert_ffn -> combine -> add_rms_norm with the residual: what the next block reads, in bf16 and in 8 bits,
and the residual stream that it adds to.  The norm's 8-bit output is what the experts take, its bf16 output what the gate takes.
The workloads, the map updates and the graph are those of `resident.py`; its x stands for attention's output.

Usage: python -m synth.resident_mx8 [--workload c2] [--tokens T] [--steps K]
"""
from __future__ import annotations

import argparse
import json
from typing import Dict, List, Optional

import numpy as np
import torch

import synth
from paper_2602_21140_amd import add_rms_norm, mx8_linear, mx8_pack, mx8_pack_expert, mx8_quantize
from synth.resident import ResidentLayer
from synth.resident_mx import _ms_per_step


class ResidentMx8Block(ResidentLayer):
    EPS = 1e-6

    def __init__(self, cfg: synth.LayerConfig, device="cuda:0", **kw):
        super().__init__(cfg, device=device, with_weights=False, **kw)
        L, T, H, P = self.layer, cfg.T, cfg.H, cfg.P
        gen = torch.Generator().manual_seed(cfg.seed + 101)
        # what balancing leaves: offsets of about the distance between neighbouring scores
        self.bias = (torch.randn(cfg.E, generator=gen) / (16 if cfg.score_fn == "sigmoid" else 4 * cfg.E)).to(device)
        self.residual = (2 * torch.randn(T, H, generator=gen)).to(torch.bfloat16).to(device)
        self.w_attention = (torch.randn(H, H, generator=gen) * H ** -0.5).to(torch.bfloat16).to(device)  # [out, in]
        self.attention_bias = (0.1 * torch.randn(H, generator=gen)).to(device)
        self.norms = [(1 + 0.1 * torch.randn(H, generator=gen)).to(torch.bfloat16).to(device) for _ in range(2)]
        self.w_attention_packed = mx8_pack(*mx8_quantize(self.w_attention))
        self.mx_gu: List[Optional[torch.Tensor]] = [None] * P
        self.mx_dn: List[Optional[torch.Tensor]] = [None] * P
        for e in range(cfg.E):
            slots = np.nonzero(self.p2l == e)[0]
            if slots.size:
                w = synth.draw_expert(cfg, e, device)
                g, d = mx8_pack_expert(w["gate"], w["up"], w["down"])
                for i, p in enumerate(slots):  # each replica owns its own copy of the bits
                    self.mx_gu[p], self.mx_dn[p] = (g, d) if i == 0 else (g.clone(), d.clone())
        L.set_mx8_expert_weights(self.mx_gu, self.mx_dn)
        sh = synth.draw_shared(cfg, device)
        self.mx_sh = (None, None) if sh is None else mx8_pack_expert(sh["gate"], sh["up"], sh["down"])
        b = self.buf
        b["x_perm"] = None
        b["y_shared"] = None if sh is None else L.empty(T, H)
        form = lambda: (L.empty(T, H, dtype=torch.uint8), L.empty(T, H // 32, dtype=torch.uint8))  # noqa: E731
        b.update(attention_form=form(), stream=L.empty(T, H), x=L.empty(T, H), x_form=form(), next_stream=L.empty(T, H), next_x=L.empty(T, H),
                 next_form=form())

    def forward(self, logits: Optional[torch.Tensor] = None, shared=True, stream=None, overlap_shared=True,
                stage_marks: Optional[list] = None) -> Dict[str, Optional[torch.Tensor]]:
        """The block into the preallocated buffers (returned).  The shared expert is served by the launches of the routed ones, so that
        overlap_shared changes nothing here.  stage_marks: seven timing events, before the projection and after it (with the first norm), the
        gate, dispatch, the experts, combine and the last norm."""
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
        mx8_quantize(self.x, out=b["attention_form"], stream=main)
        mx8_linear(*b["attention_form"], self.w_attention_packed, self.cfg.H, bias=self.attention_bias, residual=self.residual, out=b["stream"],
                   stream=main)
        add_rms_norm(b["stream"], self.norms[0], eps=self.EPS, quantize=True, out=(None, b["x"], *b["x_form"]), stream=main)
        mark()
        if given:
            with torch.cuda.stream(main):
                b["logits"].copy_(logits)
        L.route_biased(None if given else b["x"], None if given else self.w_router_packed, self.bias, T, logits=b["logits"],
                       logits_given=given, out=(b["topk_logical"], b["topk_weight"], b["topk_phys"]), stream=main)
        mark()
        L.dispatch_index(b["topk_phys"], T, out=(b["slot_offsets"], b["dst_row"], b["src_of"]), stream=main)
        mark()
        L.mx8_expert_ffn(*b["x_form"], b["src_of"], b["slot_offsets"], T, *sh, out=(b["y_perm"], y_shared), stream=main)
        mark()
        L.combine(b["y_perm"], b["dst_row"], b["topk_weight"], y_shared, T, out=b["out"], stream=main)
        mark()
        add_rms_norm(b["out"], self.norms[1], residual=b["stream"], eps=self.EPS, quantize=True,
                     out=(b["next_stream"], b["next_x"], *b["next_form"]), stream=main)
        mark()
        return b


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="c2", choices=[n for n, c in synth.CONFIGS.items() if c.dtype == "bf16"])
    ap.add_argument("--tokens", type=int, default=None)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    cfg = synth.get_config(args.workload)
    if args.tokens:
        cfg = synth.scaled(cfg, T=args.tokens)
    g = ResidentMx8Block(cfg)
    line = {"workload": cfg.name, "tokens": cfg.T, "ms_per_step": round(_ms_per_step(g, args.steps), 4),
            "weight_gib": round(sum(w.numel() for w in g.mx_gu + g.mx_dn if w is not None) / 2 ** 30, 3)}
    marks: list = []
    g.forward(stage_marks=marks)
    torch.cuda.synchronize()
    names = ("projection_and_norm", "gate", "dispatch", "experts", "combine", "norm")
    line["stage_ms"] = {n: round(a.elapsed_time(b), 4) for n, a, b in zip(names, marks, marks[1:])}
    print(json.dumps(line))
    g.close()


if __name__ == "__main__":
    main()
