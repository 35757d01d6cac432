"""The operators of the layer in 4-bit form, as cases that can be timed: the gate with a balance bias, microscaled 4-bit
floats and back, and the expert FFN on them.

own               False: run() computes the plain form in torch; True: it calls the library
listed()          the cases
draw(rng)         one more case of the same ranges
prepare(c, seed)  what a user's program holds before the call
run(state)        one pass; returns what it computed
work(c)           bytes and flops the pass cannot do without
exact(c, seed)    what run() returns for these inputs, in 64 bits

A microscaled row is cut into blocks of 32 numbers.  A block has one scale 2^e, e = floor(log2(largest magnitude)) - 2, and
its numbers are kept as x / 2^e rounded to the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the even code.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEVICE = "cuda:0"

# Layer shapes of the workloads: experts over ranks, each rank with one spare slot.
_MID = dict(H=2048, I=1408, I_shared=2816, n_ranks=8, slots_per_rank=9)
_LARGE = dict(H=7168, I=2048, I_shared=2048, n_ranks=32, slots_per_rank=9)


def _route(name, T, E, k, score_fn, n_group, n_ranks, renormalise=True, n_failed=1):
    return dict(name=name, op="route", T=T, E=E, k=k, score_fn=score_fn, n_group=n_group, topk_group=max(1, n_group // 2),
                n_ranks=n_ranks, renormalise=renormalise, n_failed=n_failed)


def _quantize(name, rows, K, dtype):
    return dict(name=name, op="quantize", rows=rows, K=K, dtype=dtype)


def _ffn(name, shape, T, k, n_failed=1, skew=0.0, **changes):
    return dict(shape, name=name, op="ffn", T=T, k=k, n_failed=n_failed, skew=skew, **changes)


def listed():
    return [
        # the gate of a decode step: a few tokens, launch and latency are all of it
        _route("route_decode", 64, 256, 8, "sigmoid", 8, 32),
        # the gate of an odd chunk of a smaller layer whose weights are not renormalised
        _route("route_odd", 1003, 64, 6, "softmax", 1, 8, renormalise=False),
        # the gate of a batch that keeps four groups of eight, three ranks down
        _route("route_batch", 8192, 256, 8, "sigmoid", 8, 32, n_failed=3),
        # the gate of the largest prefill chunk, without groups
        _route("route_prefill", 32768, 384, 8, "softmax", 1, 48, n_failed=2),
        # activations of a decode step
        _quantize("quantize_decode", 64, 7168, "bf16"),
        # fp32 rows of an odd length, as of a matrix that is no multiple of the block
        _quantize("quantize_odd", 1003, 2839, "fp32"),
        # activations of the largest prefill chunk
        _quantize("quantize_prefill", 32768, 7168, "bf16"),
        # single-stream decode: eight experts' weights are read, every latency shows
        _ffn("ffn_one_token", _LARGE, 1, 8),
        # a decode batch: two rows per expert, nearly every expert's weights are streamed once
        _ffn("ffn_decode", _LARGE, 64, 8),
        # a ragged chunk of the smaller layer under uneven load: slots with no rows beside slots with hundreds
        _ffn("ffn_uneven", _MID, 1003, 6, skew=1.0),
        # a prefill step of the smaller layer
        _ffn("ffn_mid", _MID, 4096, 6),
        # a large batch of the large layer
        _ffn("ffn_batch", _LARGE, 8192, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, without a name: 1 to 32 768 tokens and 16 to 512 experts of a gate, rows of 32 to 16 384
    numbers, and layers of 1 to 8192 tokens, hidden sizes 256 to 7168, 16 to 288 slots."""
    op = rng.choice(["route", "quantize", "ffn", "ffn"])
    if op == "route":
        n_group = rng.choice([1, 1, 2, 4, 8])
        per = rng.choice([1, 2, 4])
        E = n_group * per * 2 * _log_int(rng, max(1, 16 // (2 * n_group * per)), 512 // (2 * n_group * per))
        n_ranks = E // per
        c = dict(op=op, T=_log_int(rng, 1, 32768), E=E, k=rng.randint(1, min(16, max(1, E // n_group - per))), n_group=n_group,
                 topk_group=max(1, n_group // 2), score_fn=rng.choice(["softmax", "sigmoid"]), n_ranks=n_ranks,
                 renormalise=rng.random() < 0.7, n_failed=rng.choice([0, 1]))
        return c if c["T"] * E <= 32768 * 384 else dict(c, T=32768 * 384 // E)
    if op == "quantize":
        rows, K = _log_int(rng, 1, 32768), _log_int(rng, 32, 16384)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        return dict(op=op, rows=min(rows, 32768 * 7168 // (K * (2 if dtype == "fp32" else 1))), K=K, dtype=dtype)
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
    gen.manual_seed(seed * 7919 + 29)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)


def _failed(c):
    m = np.zeros(c.n_ranks, dtype=np.uint8)
    for i in range(c.n_failed):
        m[(2 * i + 1) * c.n_ranks // (2 * c.n_failed)] = 1
    return m


# ---- inputs --------------------------------------------------------------------------------------


def _placement(c):
    """A rank's primaries, then one spare slot with a copy of the next rank's first."""
    per = c.E // c.n_ranks
    p2l = np.zeros((c.n_ranks, per + 1), dtype=np.int32)
    p2l[:, :per] = np.arange(c.E).reshape(c.n_ranks, per)
    p2l[:, per] = np.roll(p2l[:, 0], -1)
    return p2l.reshape(-1)


def _copies(c):
    """Live slots of every expert: their number, and a table padded with the last one."""
    p2l, dead = _placement(c), np.repeat(_failed(c), c.E // c.n_ranks + 1)
    lists = [np.nonzero((p2l == e) & (dead == 0))[0] for e in range(c.E)]
    count = np.array([len(v) for v in lists])
    table = np.array([[v[min(j, len(v) - 1)] if len(v) else -1 for j in range(2)] for v in lists])
    return torch.from_numpy(count).to(DEVICE), torch.from_numpy(table.astype(np.int32)).to(DEVICE)


def _keys64(c, logits, bias, count):
    z = logits.double()
    score = torch.sigmoid(z) if c.score_fn == "sigmoid" else torch.softmax(z, dim=1)
    return score, (score + bias.double()).masked_fill(count == 0, -math.inf)


def _kept64(c, key):
    """Keys with those of dropped groups at -inf, and the groups' scores in descending order."""
    if c.n_group == 1:
        return key, None
    group = key.view(len(key), c.n_group, -1)
    best = group.topk(2, dim=2).values
    best = torch.where(best[:, :, 1] > -math.inf, best.sum(dim=2), best[:, :, 0])
    order = best.sort(dim=1, descending=True)
    keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, order.indices[:, :c.topk_group], True)
    return group.masked_fill(~keep[:, :, None], -math.inf).reshape(key.shape), order.values


def _route_inputs(c, seed):
    """Logits and a bias of the size that evens out such scores.  A token whose order hangs on less than 32 bits resolve is
    drawn again: no definition in 32 bits orders it."""
    gen = _generator(seed)
    logits, bias = _normal(gen, c.T, c.E), _normal(gen, c.E) * (0.05 if c.score_fn == "sigmoid" else 0.5 / c.E)
    count, table = _copies(c)
    for _ in range(12):
        kept, groups = _kept64(c, _keys64(c, logits, bias, count)[1])
        top = kept.topk(min(c.k + 1, c.E), dim=1).values
        near = 2e-6 * top[:, :1].abs()
        tie = ((top[:, :-1] - top[:, 1:] < near) & (top[:, :-1] > -math.inf)).any(dim=1, keepdim=True)
        if groups is not None:
            tie |= groups[:, c.topk_group - 1:c.topk_group] - groups[:, c.topk_group:c.topk_group + 1] < near
        logits = torch.where(tie, _normal(gen, c.T, c.E), logits)
    return logits, bias, count, table


def _quantize_inputs(c, seed):
    """Activations: rows of unlike size, a few numbers far out, some blocks of nothing but zeros."""
    gen = _generator(seed)
    x = _normal(gen, c.rows, c.K) * torch.exp(_normal(gen, c.rows, 1))
    x *= torch.where(torch.rand(c.K, generator=gen, device=DEVICE) < 0.01, 20.0, 1.0)
    x *= torch.rand(c.rows, 1, generator=gen, device=DEVICE) > 0.02
    return x.to(torch.bfloat16 if c.dtype == "bf16" else torch.float32)


def _ffn_routing(c, gen):
    """Rows of every slot in order, as dispatch gives them: slots of a failed rank have none, and with skew some have many."""
    P, N = c.n_ranks * c.slots_per_rank, c.T * c.k
    dead = torch.from_numpy(np.repeat(_failed(c), c.slots_per_rank)).to(DEVICE) != 0
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
    x = _normal(gen, c.T, c.H).to(torch.bfloat16)
    src_of, offsets = _ffn_routing(c, gen)
    return x, src_of, offsets, _matrices(c, gen)


# ---- microscaled numbers in plain torch ----------------------------------------------------------


def _blocks(x):
    """x [rows, K] in fp32 blocks [rows, ceil(K / 32), 32], the last one filled up with zeros."""
    rows, K = x.shape
    return torch.nn.functional.pad(x.float(), (0, -K % 32)).view(rows, -1, 32)


def _steps(b):
    """The numbers of blocks in units of their scale, rounded, and the scales' exponents."""
    largest = b.abs().amax(dim=2, keepdim=True)
    e = torch.where(largest > 0, torch.frexp(largest).exponent - 3, -127).clamp(-127, 127)
    a = torch.ldexp(b.abs(), -e).clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, b), e


def _rounded(x):
    """x [rows, K] -> the values that its microscaled form stands for, fp32 [rows, K]."""
    q, e = _steps(_blocks(x))
    return torch.ldexp(q, e).view(len(x), -1)[:, :x.shape[1]]


def _codes(x):
    """x [rows, K] -> two 4-bit codes to a byte, the lower one first, and a scale's exponent + 127 to a byte."""
    q, e = _steps(_blocks(x))
    a = q.abs()
    code = torch.where(a <= 2, a * 2, torch.where(a <= 4, a + 2, 7.0)).byte() | (torch.signbit(q).byte() << 3)
    code = code.view(len(x), -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), (e + 127).byte().view(len(x), -1)


def _table():
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEVICE)
    return torch.stack([v.repeat(16), v.repeat_interleave(16)], dim=1)  # a byte's two values


def _values(codes, scales):
    """Codes [..., K / 2] and scales [..., K / 32] -> fp32 [..., K]."""
    v = _table().index_select(0, codes.reshape(-1).int()).view(*scales.shape, 32)
    return torch.ldexp(v, scales[..., None].int() - 127).view(*scales.shape[:-1], -1)


# ---- the state a user's program holds ------------------------------------------------------------


def _layer(c, **more):
    from paper_2602_21140_amd import ReviveLayer
    shape = dict(H=64, E=1, k=1, I=64, I_shared=0, slots_per_rank=1, max_replicas=2, score_fn="softmax", n_group=1, topk_group=1, dtype="bf16")
    return ReviveLayer(SimpleNamespace(**{**shape, **vars(c), **more}), device=DEVICE)


def _prepare_route(c, seed):
    s = SimpleNamespace(c=c)
    s.logits, s.bias, s.count, s.table = _route_inputs(c, seed)
    if own:
        s.layer = _layer(c, slots_per_rank=c.E // c.n_ranks + 1)
        s.layer.set_placement(_placement(c))
        s.layer.update_map(_failed(c))
        s.out = [torch.empty(c.T, c.k, dtype=d, device=DEVICE) for d in (torch.int32, torch.float32, torch.int32)]
    return s


def _prepare_quantize(c, seed):
    s = SimpleNamespace(c=c, x=_quantize_inputs(c, seed))
    if own:
        from paper_2602_21140_amd import binding
        s.lib = binding
        blocks = -(-c.K // 32)
        s.out = [torch.empty(c.rows, n * blocks, dtype=torch.uint8, device=DEVICE) for n in (16, 1)]
        s.values = torch.empty_like(s.x)
    return s


def _prepare_ffn(c, seed):
    s = SimpleNamespace(c=c)
    s.x, s.src_of, s.offsets, matrices = _ffn_inputs(c, seed)
    P, N = c.n_ranks * c.slots_per_rank, c.T * c.k
    s.most = int((s.offsets[1:] - s.offsets[:-1]).max())
    if own:
        from paper_2602_21140_amd import binding
        packed = []
        for gate, up, down in matrices:
            packed.append((torch.cat([binding.mx_pack(*gate), binding.mx_pack(*up)]), binding.mx_pack(*down)))
        s.shared = packed[P] if c.I_shared else (None, None)
        s.layer = _layer(c, E=P, n_ranks=c.n_ranks)
        s.layer.set_mx_expert_weights([w for w, _ in packed[:P]], [w for _, w in packed[:P]])
        s.out = (s.layer.empty(N, c.H), s.layer.empty(c.T, c.H) if c.I_shared else None)
        return s
    empty = lambda rows, K: (torch.empty(P, rows, K // 2, dtype=torch.uint8, device=DEVICE),  # noqa: E731
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
    return {"route": _prepare_route, "quantize": _prepare_quantize, "ffn": _prepare_ffn}[c.op](c, seed)


# ---- one pass ------------------------------------------------------------------------------------


def _plain_route(s):
    c = s.c
    score = 1 / (1 + torch.exp(-s.logits))
    if c.score_fn == "softmax":
        score = torch.exp(s.logits - s.logits.amax(dim=1, keepdim=True))
        score = score / score.sum(dim=1, keepdim=True)
    key = torch.where(s.count > 0, score + s.bias, -math.inf)
    if c.n_group > 1:
        group = key.view(c.T, c.n_group, -1)
        two = group.sort(dim=2, descending=True, stable=True).values[:, :, :2]
        best = torch.where(two[:, :, 1] > -math.inf, two.sum(dim=2), two[:, :, 0])
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :c.topk_group]
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, kept, True)
        key = torch.where(kept[:, :, None], group, -math.inf).view(c.T, c.E)
    experts = key.sort(dim=1, descending=True, stable=True).indices[:, :c.k]
    weights = score.gather(1, experts)
    if c.renormalise:
        weights = weights / weights.sum(dim=1, keepdim=True)
    token = torch.arange(c.T, device=DEVICE)[:, None]
    return {"experts": experts.int(), "weights": weights, "slots": s.table[experts, token % s.count[experts]]}


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
    x = _rounded(s.x)
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
        return _plain_route(s) if c.op == "route" else _plain_ffn(s)
    if c.op == "route":
        s.layer.route_biased(None, None, s.bias, c.T, renormalise=c.renormalise, logits=s.logits, logits_given=True, out=s.out)
        return {"experts": s.out[0], "weights": s.out[1], "slots": s.out[2]}
    if c.op == "quantize":
        s.lib.mx_quantize(s.x, out=s.out)
        s.lib.mx_dequantize(*s.out, out=s.values)
        return {"values": s.values}
    s.layer.mx_expert_ffn(s.x, s.src_of, s.offsets, c.T, w_sh_gate_up=s.shared[0], w_sh_down=s.shared[1], out=s.out)
    return {"y": s.out[0], "shared": s.out[1]} if c.I_shared else {"y": s.out[0]}


def work(case):
    """Inputs read once, outputs written once; of the experts' weights, those of the slots that the rows are expected to reach
    (even load).  The FFN's intermediate is the library's own and is not counted."""
    c = SimpleNamespace(**case)
    if c.op == "route":
        return {"bytes": 4 * c.T * c.E + 12 * c.T * c.k + 16 * c.E, "flops": 8 * c.T * c.E}
    if c.op == "quantize":
        b = 2 if c.dtype == "bf16" else 4
        return {"bytes": int(c.rows * c.K * (2 * b + 17 / 32)), "flops": 4 * c.rows * c.K}
    live, N = (c.n_ranks - c.n_failed) * c.slots_per_rank, c.T * c.k
    used = live * (1 - (1 - c.k / live) ** c.T)
    weights = 3 * c.H * (used * c.I + c.I_shared) * 17 / 32
    rows = 2 * c.H * (c.T + N + (c.T if c.I_shared else 0)) + 4 * N
    return {"bytes": int(weights + rows), "flops": 6 * c.H * (N * c.I + c.T * c.I_shared)}


# ---- the same passes in 64 bits ------------------------------------------------------------------


def _rounded64(x):
    """The nearest number of the grid by the midpoints between neighbours; on a midpoint the even code."""
    rows, K = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -K % 32)).view(rows, -1, 32)
    largest = x.abs().amax(dim=2, keepdim=True)
    scale = torch.exp2(torch.log2(largest).floor().clamp(-125, 127) - 2)
    scale = torch.where(scale * 4 > largest, scale / 2, scale)  # a logarithm that was rounded up
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEVICE)
    middle = (grid[1:] + grid[:-1]) / 2
    a = x.abs() / scale
    low, high = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)  # they differ on a midpoint
    code = torch.where(low % 2 == 0, low, high)
    return (grid[code] * scale * torch.sign(x)).view(rows, -1)[:, :K]


def _values64(codes, scales):
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    grid = torch.tensor(grid + [-v for v in grid], dtype=torch.float64, device=DEVICE)
    both = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], dim=2).view(len(codes), -1)
    return both * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)


def _swiglu64(x, gate, up, down):
    h = torch.nn.functional.silu(x @ _values64(*gate).T) * (x @ _values64(*up).T)
    return _rounded64(h) @ _values64(*down).T


def exact(case, seed):
    c = SimpleNamespace(**case)
    if c.op == "quantize":
        return {"values": _rounded64(_quantize_inputs(c, seed))}
    if c.op == "route":
        logits, bias, count, table = _route_inputs(c, seed)
        score, key = _keys64(c, logits, bias, count)
        experts = _kept64(c, key)[0].topk(c.k, dim=1).indices
        weights = score.gather(1, experts)
        if c.renormalise:
            weights = weights / weights.sum(dim=1, keepdim=True)
        slots = table[experts, torch.arange(c.T, device=DEVICE)[:, None] % count[experts]]
        return {"experts": experts.int(), "weights": weights, "slots": slots}
    x, src_of, offsets, matrices = _ffn_inputs(c, seed)
    x = _rounded64(x)
    y = torch.zeros(c.T * c.k, c.H, dtype=torch.float64, device=DEVICE)
    res, at, P = {"y": y}, offsets.tolist(), len(offsets) - 1
    for p, m in enumerate(matrices):
        if p == P:
            res["shared"] = _swiglu64(x, *m)
        elif at[p] < at[p + 1]:
            y[at[p]:at[p + 1]] = _swiglu64(x[(src_of[at[p]:at[p + 1]] // c.k).long()], *m)
    return res
