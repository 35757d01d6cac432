"""The layer in 8-bit form and what stands in front of it, as cases that can be timed: the norm with the residual's addition
and an 8-bit output, microscaled 8-bit floats, the matrix product on them with bias, activation and residual, and the expert FFN.

own               False: run() computes the plain form in torch; True: it calls the library
listed()          the cases
draw(rng)         one more case of the same ranges
prepare(c, seed)  what a user's program holds before the call
run(state)        one pass; returns what it computed
work(c)           bytes and flops the pass cannot do without
exact(c, seed)    what run() returns for these inputs, in 64 bits

A microscaled row is cut into blocks of 32 numbers.  A block has one scale 2^e, e the smallest with largest magnitude <= 448 * 2^e
(at least -127), and its numbers are kept as x / 2^e rounded to the nearest 8-bit float with 4 bits of exponent and 3 of
mantissa (whose largest number is 448), ties to the even code.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

# Layer shapes of the workloads: experts over ranks, each rank with one spare slot.
_MID = dict(H=2048, I=1408, I_shared=2816, n_ranks=8, slots_per_rank=9)
_LARGE = dict(H=7168, I=2048, I_shared=2048, n_ranks=32, slots_per_rank=9)


def _norm(name, rows, H, dtype="bf16", residual=True, quantize=True):
    return dict(name=name, op="norm", rows=rows, H=H, dtype=dtype, residual=residual, quantize=quantize)


def _quantize(name, rows, K, dtype):
    return dict(name=name, op="quantize", rows=rows, K=K, dtype=dtype)


def _linear(name, rows, K, N, bias=False, activation="none", residual=False):
    return dict(name=name, op="linear", rows=rows, K=K, N=N, bias=bias, activation=activation, residual=residual)


def _ffn(name, shape, T, k, n_failed=1, skew=0.0, **changes):
    return dict(shape, name=name, op="ffn", T=T, k=k, n_failed=n_failed, skew=skew, **changes)


def listed():
    return [
        # the norm in front of the layer in a decode step: launch and latency are all of it
        _norm("norm_decode", 64, 7168),
        # rows of an odd length, fp32, nothing to add
        _norm("norm_odd", 1003, 2839, dtype="fp32", residual=False),
        # the norm of the largest prefill chunk
        _norm("norm_prefill", 32768, 7168),
        # fp32 rows of an odd length, as of a matrix that is no multiple of the block
        _quantize("quantize_odd", 1003, 2839, "fp32"),
        # activations of the largest prefill chunk that no norm of ours made
        _quantize("quantize_prefill", 32768, 7168, "bf16"),
        # attention's output projection into the residual stream, one token: 51 MB of weights are streamed
        _linear("linear_one_token", 1, 7168, 7168, residual=True),
        # the same of a decode batch
        _linear("linear_decode", 64, 7168, 7168, residual=True),
        # a ragged chunk, an odd number of columns, everything in the epilogue
        _linear("linear_odd", 1003, 2048, 1411, bias=True, activation="gelu", residual=True),
        # a prefill chunk
        _linear("linear_prefill", 8192, 7168, 7168, bias=True, residual=True),
        # a decode batch: two rows per expert, nearly every expert's weights are streamed once
        _ffn("ffn_decode", _LARGE, 64, 8),
        # a ragged chunk of the smaller layer under uneven load: slots with no rows beside slots with hundreds
        _ffn("ffn_uneven", _MID, 1003, 6, skew=1.0),
        # a large batch of the large layer
        _ffn("ffn_batch", _LARGE, 8192, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, without a name: 1 to 32 768 rows of 32 to 16 384 numbers for the norm and the rounding; products
    of 1 to 8192 rows, 32 to 16 384 deep, 1 to 16 384 wide; layers of 1 to 8192 tokens, hidden sizes 256 to 7168, 12 to 288 slots."""
    op = rng.choice(["norm", "quantize", "linear", "linear", "ffn", "ffn"])
    if op in ("norm", "quantize"):
        rows, K, dtype = _log_int(rng, 1, 32768), _log_int(rng, 32, 16384), rng.choice(["bf16", "bf16", "fp32"])
        rows = min(rows, 32768 * 7168 // (K * (2 if dtype == "fp32" else 1)))
        if op == "quantize":
            return dict(op=op, rows=rows, K=K, dtype=dtype)
        return dict(op=op, rows=rows, H=K, dtype=dtype, residual=rng.random() < 0.7, quantize=rng.random() < 0.7)
    if op == "linear":
        while True:
            c = dict(op=op, rows=_log_int(rng, 1, 8192), K=32 * _log_int(rng, 1, 512), N=_log_int(rng, 1, 16384),
                     bias=rng.random() < 0.5, activation=rng.choice(["none", "none", "relu", "silu", "gelu"]),
                     residual=rng.random() < 0.5)
            if c["rows"] * c["K"] * c["N"] <= 8192 * 7168 * 7168 and c["K"] * c["N"] <= 16384 * 7168:
                return c
    while True:
        per = rng.choice([2, 4, 8])
        c = dict(op=op, T=_log_int(rng, 1, 8192), H=64 * _log_int(rng, 4, 112), I=64 * _log_int(rng, 2, 32), k=rng.randint(1, 8),
                 n_ranks=_log_int(rng, 4, 32), slots_per_rank=per + 1, n_failed=rng.choice([0, 1]), skew=rng.choice([0.0, 0.0, 1.0]))
        c["I_shared"] = rng.choice([0, c["I"], 2 * c["I"]])
        slots = c["n_ranks"] * c["slots_per_rank"]
        fits = slots * c["H"] * c["I"] <= 288 * 7168 * 2048 and c["T"] * c["H"] * (c["k"] * c["I"] + c["I_shared"]) <= 8192 * 7168 * 9 * 2048
        if fits and c["T"] * c["k"] * c["H"] <= 65536 * 7168 and (not c["skew"] or c["T"] <= 2048):
            return c


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7919 + 31)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


# ---- inputs --------------------------------------------------------------------------------------


def _activations(gen, rows, K, dtype):
    """Rows of unlike size with a few columns far out, some rows of nothing but zeros."""
    x = _normal(gen, rows, K) * torch.exp(_normal(gen, rows, 1))
    x *= torch.where(torch.rand(K, generator=gen, device=DEVICE) < 0.01, 20.0, 1.0)
    x *= torch.rand(rows, 1, generator=gen, device=DEVICE) > 0.02
    return x.to(DTYPES[dtype])


def _norm_inputs(c, seed):
    gen = _generator(seed)
    x = _activations(gen, c.rows, c.H, c.dtype)
    residual = (3 * _normal(gen, c.rows, c.H)).to(x.dtype) if c.residual else None
    return x, residual, (1 + 0.2 * _normal(gen, c.H)).to(x.dtype)


def _linear_inputs(c, seed):
    gen = _generator(seed)
    x = _codes(_normal(gen, c.rows, c.K) * torch.exp(0.5 * _normal(gen, c.rows, 1)))
    w = _codes(_normal(gen, c.N, c.K) * c.K ** -0.5)
    bias = 0.5 * _normal(gen, c.N) if c.bias else None
    residual = (3 * _normal(gen, c.rows, c.N)).to(torch.bfloat16) if c.residual else None
    return x, w, bias, residual


def _ffn_routing(c, gen):
    """Rows of every slot in order, as dispatch gives them: slots of a failed rank have none, and with skew some have many."""
    P, N = c.n_ranks * c.slots_per_rank, c.T * c.k
    dead = np.zeros(c.n_ranks, dtype=bool)
    dead[[(2 * i + 1) * c.n_ranks // (2 * c.n_failed) for i in range(c.n_failed)]] = True
    dead = torch.from_numpy(np.repeat(dead, c.slots_per_rank)).to(DEVICE)
    liking = (c.skew * _normal(gen, 1, P)).masked_fill(dead, -math.inf)
    chosen = (liking - torch.rand(c.T, P, generator=gen, device=DEVICE).log().neg().log()).topk(c.k, dim=1).indices.reshape(N)
    by_slot = chosen.sort(stable=True)
    offsets = torch.searchsorted(by_slot.values, torch.arange(P + 1, device=DEVICE))
    return by_slot.indices.int(), offsets.int()


def _matrices(c, gen):
    """Codes and scales of every slot's gate, up and down matrix, and of the shared expert's, one expert after the other."""
    P = c.n_ranks * c.slots_per_rank
    for width in [c.I] * P + ([c.I_shared] if c.I_shared else []):
        yield [_codes(_normal(gen, rows, K) * c.H ** -0.5) for rows, K in ((width, c.H), (width, c.H), (c.H, width))]


def _ffn_inputs(c, seed):
    gen = _generator(seed)
    x = _codes(_normal(gen, c.T, c.H))
    src_of, offsets = _ffn_routing(c, gen)
    return x, src_of, offsets, _matrices(c, gen)


# ---- microscaled numbers in plain torch ----------------------------------------------------------


def _blocks(x):
    """x [rows, K] in fp32 blocks [rows, ceil(K / 32), 32], the last one filled up with zeros."""
    rows, K = x.shape
    return torch.nn.functional.pad(x.float(), (0, -K % 32)).view(rows, -1, 32)


def _steps(b):
    """The numbers of blocks in units of their scale, rounded, and the scales' exponents."""
    part, e = torch.frexp(b.abs().amax(dim=2, keepdim=True))
    e = torch.where(part > 0, e - 9 + (part > 0.875), -127).clamp(-127, 127)
    return torch.ldexp(b, -e).to(torch.float8_e4m3fn), e


def _codes(x):
    """x [rows, K] -> a code to a byte, and a scale's exponent + 127 to a byte."""
    q, e = _steps(_blocks(x))
    return q.view(torch.uint8).view(len(x), -1), (e + 127).byte().view(len(x), -1)


def _rounded(x):
    """x [rows, K] -> the values that its microscaled form stands for, fp32 [rows, K]."""
    q, e = _steps(_blocks(x))
    return torch.ldexp(q.float(), e).view(len(x), -1)[:, :x.shape[1]]


def _values(codes, scales):
    """Codes [..., K] and scales [..., K / 32] -> fp32 [..., K]."""
    v = codes.view(torch.float8_e4m3fn).float().view(*scales.shape, 32)
    return torch.ldexp(v, scales[..., None].int() - 127).view(codes.shape)


def _as_floats(codes, scales):
    """The bytes as the 8-bit floats that they are."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


# ---- the state a user's program holds ------------------------------------------------------------


def _empty_form(rows, K):
    blocks = -(-K // 32)
    return tuple(torch.empty(rows, n * blocks, dtype=torch.uint8, device=DEVICE) for n in (32, 1))


def _prepare_norm(c, seed):
    s = SimpleNamespace(c=c)
    s.x, s.residual, s.weight = _norm_inputs(c, seed)
    if own:
        from paper_2602_21140_amd import binding
        s.lib = binding
        s.out = (torch.empty_like(s.x) if c.residual else None, torch.empty_like(s.x), *(_empty_form(c.rows, c.H) if c.quantize else (None, None)))
    return s


def _prepare_quantize(c, seed):
    s = SimpleNamespace(c=c, x=_activations(_generator(seed), c.rows, c.K, c.dtype))
    if own:
        from paper_2602_21140_amd import binding
        s.lib = binding
        s.out = _empty_form(c.rows, c.K)
        s.values = torch.empty_like(s.x)
    return s


def _prepare_linear(c, seed):
    s = SimpleNamespace(c=c)
    s.x, s.w, s.bias, s.residual = _linear_inputs(c, seed)
    if own:
        from paper_2602_21140_amd import binding
        s.lib = binding
        s.w = binding.mx8_pack(*s.w)
        s.out = torch.empty(c.rows, c.N, dtype=torch.bfloat16, device=DEVICE)
    return s


def _prepare_ffn(c, seed):
    s = SimpleNamespace(c=c)
    s.x, s.src_of, s.offsets, matrices = _ffn_inputs(c, seed)
    P, N = c.n_ranks * c.slots_per_rank, c.T * c.k
    s.most = int((s.offsets[1:] - s.offsets[:-1]).max())
    if own:
        from paper_2602_21140_amd import ReviveLayer, binding
        packed = []
        for gate, up, down in matrices:
            packed.append((torch.cat([binding.mx8_pack(*gate), binding.mx8_pack(*up)]), binding.mx8_pack(*down)))
        s.shared = packed[P] if c.I_shared else (None, None)
        shape = dict(max_replicas=2, score_fn="softmax", n_group=1, topk_group=1, dtype="bf16", E=P)
        s.layer = ReviveLayer(SimpleNamespace(**{**shape, **{n: v for n, v in vars(c).items() if n not in ("name", "op")}}), device=DEVICE)
        s.layer.set_mx8_expert_weights([w for w, _ in packed[:P]], [w for _, w in packed[:P]])
        s.out = (s.layer.empty(N, c.H), s.layer.empty(c.T, c.H) if c.I_shared else None)
        return s
    empty = lambda rows, K: (torch.empty(P, rows, K, dtype=torch.uint8, device=DEVICE),  # noqa: E731
                             torch.empty(P, rows, K // 32, dtype=torch.uint8, device=DEVICE))
    s.gate_up, s.down, s.shared = empty(2 * c.I, c.H), empty(c.H, c.I), None
    for p, (gate, up, down) in enumerate(matrices):
        joined = [torch.cat(m) for m in zip(gate, up)]
        if p == P:
            s.shared = joined, down
            break
        for to, m in zip(s.gate_up + s.down, joined + list(down)):
            to[p] = m
    return s


def prepare(case, seed):
    c = SimpleNamespace(**case)
    return {"norm": _prepare_norm, "quantize": _prepare_quantize, "linear": _prepare_linear, "ffn": _prepare_ffn}[c.op](c, seed)


# ---- one pass ------------------------------------------------------------------------------------


def _plain_norm(s):
    c, dtype = s.c, s.x.dtype
    out, v = {}, s.x
    if c.residual:
        out["sum"] = v = (s.x.float() + s.residual.float()).to(dtype)
    size = v.double().square().mean(dim=1, keepdim=True)  # a number next to a border of the 8-bit grid hangs on its last bits
    out["y"] = (v.float() * (1 / torch.sqrt(size + EPS)).float() * s.weight.float()).to(dtype)
    if c.quantize:
        out.update(_as_floats(*_codes(out["y"])))
    return out


def _activated(z, activation):
    if activation == "relu":
        return z.clamp(min=0)
    if activation == "silu":
        return z / (1 + torch.exp(-z))
    return z * 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) if activation == "gelu" else z


def _plain_linear(s):
    z = torch.mm(_values(*s.x), _values(*s.w).T)
    if s.bias is not None:
        z = z + s.bias
    z = _activated(z, s.c.activation)
    if s.residual is not None:
        z = z + s.residual.float()
    return {"out": z.to(torch.bfloat16)}


def _plain_swiglu(x, gate_up, down):
    """x [n, rows, K] times n experts' matrices: the matrices come first, so that the smaller operand is turned over."""
    both = torch.bmm(_values(*gate_up), x.transpose(1, 2).contiguous())
    gate, up = both.chunk(2, dim=1)
    h = (gate / (1 + torch.exp(-gate)) * up).transpose(1, 2)
    h = _rounded(h.reshape(-1, h.shape[2])).view(h.shape)
    return torch.bmm(_values(*down), h.transpose(1, 2).contiguous()).transpose(1, 2)


def _plain_ffn(s):
    c = s.c
    P, N = len(s.offsets) - 1, c.T * c.k
    x = _values(*s.x)
    rows, first = torch.arange(N, device=DEVICE), s.offsets.long()
    slot = torch.bucketize(rows, first[1:], right=True)
    if N <= P:  # few rows: each with its own slot's matrices
        y = _plain_swiglu(x[s.src_of // c.k][:, None], [m[slot] for m in s.gate_up], [m[slot] for m in s.down])[:, 0]
    else:  # every slot's rows filled up to those of the fullest
        row = (first[:-1, None] + torch.arange(s.most, device=DEVICE)).clamp(max=N - 1)
        y = _plain_swiglu(x[s.src_of[row] // c.k], s.gate_up, s.down)[slot, rows - first[slot]]
    out = {"y": y.to(torch.bfloat16)}
    if c.I_shared:
        (gate_up, down) = s.shared
        out["shared"] = _plain_swiglu(x[None], [m[None] for m in gate_up], [m[None] for m in down])[0].to(torch.bfloat16)
    return out


def run(state):
    s, c = state, state.c
    if not own:
        if c.op == "quantize":
            return {"values": _rounded(s.x).to(s.x.dtype)}
        return {"norm": _plain_norm, "linear": _plain_linear, "ffn": _plain_ffn}[c.op](s)
    if c.op == "norm":
        total, y, codes, scales = s.lib.add_rms_norm(s.x, s.weight, residual=s.residual, eps=EPS, quantize=c.quantize, out=s.out)
        out = {"y": y, "sum": total} if c.residual else {"y": y}
        return {**out, **_as_floats(codes, scales)} if c.quantize else out
    if c.op == "quantize":
        s.lib.mx8_quantize(s.x, out=s.out)
        s.lib.mx8_dequantize(*s.out, out=s.values)
        return {"values": s.values}
    if c.op == "linear":
        return {"out": s.lib.mx8_linear(*s.x, s.w, c.N, bias=s.bias, activation=c.activation, residual=s.residual, out=s.out)}
    s.layer.mx8_expert_ffn(*s.x, s.src_of, s.offsets, c.T, w_sh_gate_up=s.shared[0], w_sh_down=s.shared[1], out=s.out)
    return {"y": s.out[0], "shared": s.out[1]} if c.I_shared else {"y": s.out[0]}


def work(case):
    """Inputs read once, outputs written once; of the experts' weights, those of the slots that the rows are expected to reach
    (even load).  The FFN's intermediate is the library's own and is not counted."""
    c = SimpleNamespace(**case)
    if c.op == "norm":
        b = 2 if c.dtype == "bf16" else 4
        return {"bytes": int(c.rows * c.H * (b * (4 if c.residual else 2) + (33 / 32 if c.quantize else 0))), "flops": 8 * c.rows * c.H}
    if c.op == "quantize":
        b = 2 if c.dtype == "bf16" else 4
        return {"bytes": int(c.rows * c.K * (2 * b + 33 / 32)), "flops": 4 * c.rows * c.K}
    if c.op == "linear":
        return {"bytes": int((c.rows + c.N) * c.K * 33 / 32 + c.rows * c.N * (4 if c.residual else 2)), "flops": 2 * c.rows * c.K * c.N}
    live, N = (c.n_ranks - c.n_failed) * c.slots_per_rank, c.T * c.k
    used = live * (1 - (1 - c.k / live) ** c.T)
    weights = 3 * c.H * (used * c.I + c.I_shared) * 33 / 32
    rows = c.H * (c.T * 33 / 32 + 2 * N + (2 * c.T if c.I_shared else 0)) + 4 * N
    return {"bytes": int(weights + rows), "flops": 6 * c.H * (N * c.I + c.T * c.I_shared)}


# ---- the same passes in 64 bits ------------------------------------------------------------------


def _form64(x):
    """x [rows, K] -> the 8-bit numbers [rows, 32 n] and the scales [rows, n] of its microscaled form, from the definition."""
    rows, K = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -K % 32)).view(rows, -1, 32)
    largest = x.abs().amax(dim=2, keepdim=True)
    scale = torch.exp2(torch.log2(largest / 448).ceil().clamp(-127, 127))
    scale = torch.where(scale * 448 < largest, scale * 2, scale)  # a logarithm that was rounded down, or up
    scale = torch.where((scale * 224 >= largest) & (scale > 2.0 ** -127), scale / 2, scale)
    a = x.abs() / scale
    low = torch.exp2(torch.log2(a).floor().clamp(min=-6.0))  # the power of two below: eight steps up to the next one
    low = torch.where(low > a, (low / 2).clamp(min=2.0 ** -6), torch.where(low * 2 <= a, low * 2, low))
    q = torch.round(a / (low / 8)) * (low / 8) * torch.sign(x)
    return q.view(rows, -1), scale.view(rows, -1)


def _rounded64(x):
    q, scale = _form64(x)
    return (q * scale.repeat_interleave(32, dim=1))[:, :x.shape[1]]


def _values64(codes, scales):
    """Sign, four bits of exponent, three of mantissa; exponent 0: in steps of 2^-9."""
    b = codes.int()
    exponent, mantissa = ((b >> 3) & 15).double(), (b & 7).double()
    v = torch.where(exponent > 0, torch.exp2(exponent - 7) * (1 + mantissa / 8), mantissa * 2.0 ** -9)
    return torch.where(b >= 128, -v, v) * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)


def _swiglu64(x, gate, up, down):
    h = torch.nn.functional.silu(x @ _values64(*gate).T) * (x @ _values64(*up).T)
    return _rounded64(h) @ _values64(*down).T


def exact(case, seed):
    c = SimpleNamespace(**case)
    if c.op == "quantize":
        return {"values": _rounded64(_activations(_generator(seed), c.rows, c.K, c.dtype))}
    if c.op == "norm":
        x, residual, weight = _norm_inputs(c, seed)
        res, v = {}, x.double()
        if residual is not None:
            res["sum"] = v + residual.double()
            v = res["sum"].to(x.dtype).double()  # the norm is that of the sum as it is stored
        res["y"] = v * torch.rsqrt((v * v).sum(dim=1, keepdim=True) / c.H + EPS) * weight.double()
        if c.quantize:  # the 8-bit form is that of y as it is stored
            res["codes"], res["scales"] = _form64(res["y"].to(x.dtype))
        return res
    if c.op == "linear":
        x, w, bias, residual = _linear_inputs(c, seed)
        z = torch.nn.functional.linear(_values64(*x), _values64(*w), None if bias is None else bias.double())
        z = {"relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}.get(c.activation, lambda v: v)(z)
        return {"out": z if residual is None else z + residual.double()}
    x, src_of, offsets, matrices = _ffn_inputs(c, seed)
    x = _values64(*x)
    y = torch.zeros(c.T * c.k, c.H, dtype=torch.float64, device=DEVICE)
    res, at, P = {"y": y}, offsets.tolist(), len(offsets) - 1
    for p, m in enumerate(matrices):
        if p == P:
            res["shared"] = _swiglu64(x, *m)
        elif at[p] < at[p + 1]:
            y[at[p]:at[p + 1]] = _swiglu64(x[(src_of[at[p]:at[p + 1]] // c.k).long()], *m)
    return res
