"""Microscaled 4-bit floats and the expert FFN on them against the oracle in 64 bits."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx_oracle as mx
from oracle import revive_oracle as orc
from paper_2602_21140_amd import ReviveError, ReviveLayer, binding, mx_dequantize, mx_pack, mx_pack_expert, mx_quantize

pytestmark = pytest.mark.gpu


def make_rows(rows, K, dtype, seed=0):
    """Rows of unlike size with exact midpoints, zero blocks, outliers and every exponent among them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K)) * np.exp(3 * rng.standard_normal((rows, 1)))
    x = np.where(rng.random((rows, K)) < 0.3, np.round(x * 4) / 4, x)
    x *= rng.random((rows, -(-K // 32))).repeat(32, axis=1)[:, :K] > 0.1
    if rows > 4:
        x[1] *= 2.0 ** 120 / max(1e-30, np.abs(x[1]).max())
        x[2] *= 2.0 ** -125
        x[3] *= 2.0 ** -132
    return torch.from_numpy(x).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (3, 31), (5, 33), (64, 64), (7, 129), (130, 1000), (33, 4104), (2, 16384), (1025, 96)])
def test_quantize_and_back(rows, K, dtype):
    x = make_rows(rows, K, dtype, rows + K)
    codes, scales = mx_quantize(x)
    want_codes, want_scales = mx.quantize(f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    want = mx.values(want_codes, want_scales)[:, :K]
    for out in (torch.float32, torch.bfloat16):
        assert np.array_equal(f64(mx_dequantize(codes, scales, K, dtype=out)), want)  # both types hold every value


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_strided_and_unaligned_rows(dtype):
    base = make_rows(40, 300, dtype, 3)
    for x in (base[:, 5:261], base[::2, 8:264], base[1:, 1:2], base[:, :256]):
        codes, scales = mx_quantize(x)
        want_codes, want_scales = mx.quantize(f64(x))
        assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
        out = torch.full((40, 300), 7.0, dtype=dtype, device="cuda")
        part = out[:len(x), 3:3 + x.shape[1]]
        mx_dequantize(codes, scales, out=part)
        assert np.array_equal(f64(part), mx.values(want_codes, want_scales)[:, :x.shape[1]])
        part.fill_(7.0)
        assert bool((out == 7.0).all())  # nothing beside the rows was written


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_not_finite_blocks_are_nan_and_alone(dtype):
    x = make_rows(4, 160, dtype, 9)
    x[0, 40], x[1, 0], x[2, 159], x[3, 70] = float("nan"), float("inf"), -float("inf"), 3e38
    codes, scales = mx_quantize(x)
    want_codes, want_scales = mx.quantize(f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    v = f64(mx_dequantize(codes, scales))
    want = mx.values(want_codes, want_scales)
    assert np.array_equal(np.isnan(v), np.isnan(want)) and np.array_equal(v[~np.isnan(v)], want[~np.isnan(want)])
    assert np.isnan(v).sum() == 3 * 32


def test_quantize_of_no_rows_and_on_another_stream():
    codes, scales = mx_quantize(torch.empty(0, 64, device="cuda"))
    assert codes.shape == (0, 32) and scales.shape == (0, 2) and mx_dequantize(codes, scales).shape == (0, 64)
    s = torch.cuda.Stream()
    x = make_rows(64, 512, torch.float32, 1)
    s.wait_stream(torch.cuda.current_stream())
    codes, scales = mx_quantize(x, stream=s)
    s.synchronize()
    assert np.array_equal(codes.cpu().numpy(), mx.quantize(f64(x))[0])


@pytest.mark.parametrize("rows,K", [(64, 32), (128, 128), (130, 704), (320, 576)])
def test_packed_layout(rows, K):
    """Every byte of the layout that the header states."""
    codes, scales = mx.quantize(np.random.default_rng(K).standard_normal((rows, K)))
    packed = mx_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()).cpu().numpy()
    panels, steps, groups = -(-rows // 128), -(-K // 128), -(-K // 512)
    assert packed.size == binding.mx_packed_bytes(rows, K) == panels * 128 * (steps * 64 + groups * 16)
    c = packed[:panels * 128 * steps * 64].reshape(panels, steps, 8, 64, 16)
    s = packed[c.size:].reshape(panels, groups, 8, 64, 4)
    full = np.zeros((panels * 128, steps * 64), np.uint8)
    full[:rows, :K // 2] = codes
    full_s = np.zeros((panels * 128, groups * 16), np.uint8)
    full_s[:rows, :K // 32] = scales
    for sub in range(8):
        for lane in range(64):
            m = lane % 16
            r = np.arange(panels) * 128 + 32 * (sub // 2) + 8 * (m // 4) + 4 * (sub % 2) + m % 4
            for st in range(steps):
                at = st * 64 + 16 * (lane // 16)
                assert np.array_equal(c[:, st, sub, lane], full[r, at:at + 16])
            for g in range(groups):
                for b in range(4):
                    assert np.array_equal(s[:, g, sub, lane, b], full_s[r, (g * 4 + b) * 4 + lane // 16])


# ---- the expert FFN ------------------------------------------------------------------------------


class Ffn:
    """A layer of random 4-bit experts with a given number of rows per slot, and its oracle."""

    def __init__(self, H, I, k, rows_per_slot, I_shared=0, T=None, seed=0):
        rng = np.random.default_rng(seed)
        self.H, self.I, self.P, self.k = H, I, len(rows_per_slot), k
        n = int(sum(rows_per_slot))
        self.T = T = -(-n // k) if T is None else T
        self.N = T * k
        assert n <= self.N
        cfg = SimpleNamespace(T=T, H=H, E=max(self.P, k), k=k, I=I, I_shared=I_shared, n_ranks=1, slots_per_rank=self.P, max_replicas=1,
                              score_fn="softmax", n_group=1, topk_group=1, dtype="bf16")
        self.L = ReviveLayer(cfg)
        self.L.workspace.fill_(255)  # what a kernel reads before it is written shows as NaN
        self.L._check(self.L.L.revive_bind_workspace(self.L._ctx, self.L.workspace.data_ptr(), self.L.workspace.numel()))
        self.x = torch.from_numpy(rng.standard_normal((T, H))).to(torch.bfloat16).cuda()
        self.offsets = np.concatenate([[0], np.cumsum(rows_per_slot)]).astype(np.int32)
        self.src_of = rng.permutation(self.N).astype(np.int32)
        self.experts, gu, dn = [], [], []
        for p in range(self.P):
            if not rows_per_slot[p]:  # a slot without rows: there is nothing to point at
                gu.append(None), dn.append(None), self.experts.append(None)
                continue
            w = self._draw(rng, I)
            self.experts.append(mx.expert_values({n: f64(t) for n, t in w.items()}))
            a, b = mx_pack_expert(w["gate"], w["up"], w["down"])
            gu.append(a), dn.append(b)
        self.L.set_mx_expert_weights(gu, dn)
        self.shared, self.sh = None, (None, None)
        if I_shared:
            w = self._draw(rng, I_shared)
            self.shared, self.sh = mx.expert_values({n: f64(t) for n, t in w.items()}), mx_pack_expert(w["gate"], w["up"], w["down"])
        self.d_offsets, self.d_src = torch.from_numpy(self.offsets).cuda(), torch.from_numpy(self.src_of).cuda()

    def _draw(self, rng, I):
        shape = {"gate": (self.H, I), "up": (self.H, I), "down": (I, self.H)}
        return {n: torch.from_numpy(rng.standard_normal(s) * self.H ** -0.5).float().cuda() for n, s in shape.items()}

    def run(self, **kw):
        out = (torch.full((self.N, self.H), 5.0, dtype=torch.bfloat16, device="cuda"),
               torch.full((self.T, self.H), 5.0, dtype=torch.bfloat16, device="cuda") if self.shared else None)
        return self.L.mx_expert_ffn(self.x, self.d_src, self.d_offsets, self.T, *self.sh, out=out, **kw)

    def check(self, y, y_shared):
        y, x, n = f64(y), mx.rounded(f64(self.x)), int(self.offsets[-1])
        for p, w in enumerate(self.experts):
            a, b = self.offsets[p], self.offsets[p + 1]
            if a < b:
                check_ffn(y[a:b], x[self.src_of[a:b] // self.k], w, ("slot", p))
        assert (y[n:] == 5.0).all()  # rows of no slot are left alone
        if self.shared:
            check_ffn(f64(y_shared), x, self.shared, "shared")


def check_ffn(y, x, w, what):
    """Element by element.  A product's fp32 sum has an addition per 128 products and the additions inside an instruction: its
    error is at most (K / 128 + 8) 2^-23 of the sum of magnitudes.  h is off by what that and a few roundings in silu make;
    where its rounding to 4 bits (or its block's scale) hangs on less than that, either result is right, and y may differ by the
    step times the weight.  Then y's own sum and its rounding to bf16 (2^-9; 2^-8 here)."""
    def sum_error(a, m):
        return (a.shape[1] / 128 + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(m))

    g, u = x @ w["gate"], x @ w["up"]
    h = orc.silu(g) * u
    # |silu'| <= 1.1, |silu(g)| <= |g|
    dh = 1.1 * sum_error(x, w["gate"]) * (np.abs(u) + sum_error(x, w["up"])) + np.abs(orc.silu(g)) * sum_error(x, w["up"]) + 2.0 ** -20 * np.abs(h)
    ref = mx.rounded(h)
    largest, slack = np.abs(h), np.zeros_like(h)
    low, high = mx.scale_bytes(np.maximum(largest - dh, 0)), mx.scale_bytes(largest + dh)
    for scales in (low, high):
        step = np.exp2(scales.astype(np.float64) - 127).repeat(32, axis=1)[:, :h.shape[1]]
        for moved in (h - dh, h + dh):
            c = mx.codes_for(moved, scales).reshape(len(h), -1)[:, :h.shape[1]]
            v = np.where(c >= 8, -mx.GRID[c & 7], mx.GRID[c & 7]) * step
            slack = np.maximum(slack, np.abs(v - ref))
    want = ref @ w["down"]
    allowed = slack @ np.abs(w["down"]) + sum_error(np.abs(ref) + slack, w["down"]) + 2.0 ** -8 * np.abs(want) + 1e-30
    off = np.abs(y - want)
    assert np.isfinite(y).all(), what
    assert (off <= allowed).all(), (what, float((off / allowed).max()), np.argwhere(off > allowed)[:4].tolist())
    if len(y) >= 8:  # the allowance is the exception (of fewer rows a single tie may make it the rule)
        assert np.median(slack @ np.abs(w["down"])) <= 0.02 * np.sqrt(np.mean(want ** 2)) + 1e-30


# hidden and intermediate sizes that end inside a step (128), a group of steps (512) and a panel of rows (128); slots with one
# row, none, a full tile, one more; rows that fill several tiles
SHAPES = [(64, 64, 1, [1]), (64, 64, 2, [0, 2, 0]), (192, 320, 1, [5, 0, 17]), (128, 128, 4, [16, 1, 0, 3]), (576, 704, 2, [33, 7, 64]),
          (1088, 192, 3, [65, 0, 1, 129]), (640, 1088, 1, [300, 2]), (2112, 512, 6, [40] * 6)]


@pytest.mark.parametrize("H,I,k,rows", SHAPES)
def test_ffn(H, I, k, rows):
    f = Ffn(H, I, k, rows, seed=H + I)
    f.check(*f.run())
    f.L.close()


@pytest.mark.parametrize("H,I,I_shared,k,rows,T", [(128, 64, 64, 1, [1], 1), (192, 128, 320, 2, [3, 0, 5], 37), (576, 320, 192, 2, [100, 0, 30], 131),
                                                   (320, 64, 1088, 1, [0, 0], 300)])
def test_ffn_with_shared_expert(H, I, I_shared, k, rows, T):
    f = Ffn(H, I, k, rows, I_shared, T, seed=T)
    f.check(*f.run())
    f.L.close()


def test_ffn_rows_that_are_not_finite_stay_alone():
    f = Ffn(192, 128, 2, [9, 20, 0, 40], 64, seed=4)
    clean, clean_shared = (t.clone() for t in f.run())
    bad = {3: float("nan"), 20: float("inf")}
    for t, v in bad.items():
        f.x[t, 77] = v
    y, shared = f.run()
    touched = np.isin(f.src_of[:69] // 2, list(bad))
    y, clean = f64(y)[:69], f64(clean)[:69]
    assert np.isnan(y[touched]).all() and np.array_equal(y[~touched], clean[~touched])
    others = [t for t in range(f.T) if t not in bad]
    assert np.isnan(f64(shared)[list(bad)]).all() and np.array_equal(f64(shared)[others], f64(clean_shared)[others])
    f.L.close()


def test_ffn_is_deterministic_on_any_stream_and_in_a_graph():
    f = Ffn(576, 320, 2, [100, 0, 30, 1], 192, T=80, seed=11)
    y, shared = f.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = (torch.zeros_like(y), torch.zeros_like(shared))
    f.L.mx_expert_ffn(f.x, f.d_src, f.d_offsets, f.T, *f.sh, out=out, stream=s)
    s.synchronize()
    n = f.offsets[-1]
    assert torch.equal(out[0][:n], y[:n]) and torch.equal(out[1], shared)
    f.L.graph_begin(s)
    f.L.mx_expert_ffn(f.x, f.d_src, f.d_offsets, f.T, *f.sh, out=out, stream=s)
    graph = f.L.graph_end(s)
    x = f.x.clone()
    for i in range(4):  # other inputs between the replays, and eager work
        f.x.copy_(x * (i - 1.5))
        want = f.run()
        out[0].zero_(), out[1].zero_()
        torch.cuda.synchronize()
        f.L.graph_launch(graph, s)
        s.synchronize()
        assert torch.equal(out[0][:n], want[0][:n]) and torch.equal(out[1], want[1])
    f.L.close()


def test_dispatch_index_is_dispatch_without_rows():
    for T, k, P in ((1, 1, 3), (37, 4, 9), (300, 4, 40), (3000, 8, 300)):
        cfg = SimpleNamespace(T=T, H=64, E=P, k=k, I=64, I_shared=0, n_ranks=1, slots_per_rank=P, max_replicas=1, score_fn="softmax",
                              n_group=1, topk_group=1, dtype="bf16")
        L = ReviveLayer(cfg)
        phys = torch.randint(-1, P + 1, (T, k), generator=torch.Generator().manual_seed(T), dtype=torch.int32).cuda()  # some dropped
        x = torch.zeros(T, 64, dtype=torch.bfloat16, device="cuda")
        out = [torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (P + 1, T * k, T * k)]
        want = [t.clone() for t in out]
        L.dispatch(x, phys, T, out=(torch.empty(T * k, 64, dtype=torch.bfloat16, device="cuda"), *want))
        L.dispatch_index(phys, T, out=out)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        L.close()


# ---- refusals ------------------------------------------------------------------------------------


def test_quantize_refuses():
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(TypeError):
        mx_quantize(x.half())
    with pytest.raises(ValueError):
        mx_quantize(x.t())
    with pytest.raises(ValueError):
        mx_quantize(x[0])
    codes, scales = mx_quantize(x)
    with pytest.raises(ValueError):
        mx_quantize(x, out=(codes, scales[:2]))
    with pytest.raises(ValueError):
        mx_dequantize(codes, scales, 33 * 3)
    with pytest.raises(ValueError):
        mx_dequantize(codes[:, 1:], scales)
    with pytest.raises(TypeError):
        mx_dequantize(codes, scales, dtype=torch.float16)
    L = binding.lib()
    p = codes.data_ptr()
    for args in ((0, 1, 4, 64, 64, p, p, None), (p, 2, 4, 64, 64, p, p, None), (p, 1, -1, 64, 64, p, p, None), (p, 1, 4, 0, 64, p, p, None),
                 (p, 1, 4, 64, 63, p, p, None), (p, 1, 4, 64, 64, p + 8, p, None), (p + 1, 1, 4, 64, 64, p, p, None), (p, 1, 4, 64, 64, p, 0, None)):
        assert L.revive_mx_quantize(*args) == -1 and L.revive_last_error(None)
    for args in ((0, p, 4, 64, 1, p, 64, None), (p, p, 4, 64, 3, p, 64, None), (p, p, 4, 64, 1, p + 1, 64, None), (p, p, 4, 64, 1, p, 60, None)):
        assert L.revive_mx_dequantize(*args) == -1
    with pytest.raises(ReviveError):
        binding.mx_packed_bytes(4, 33)
    assert L.revive_mx_pack(p, p, 4, 64, p + 4, None) == -1 and L.revive_mx_pack(0, p, 4, 64, p, None) == -1
    torch.cuda.synchronize()


def test_ffn_refuses():
    f = Ffn(64, 64, 1, [3], seed=1)
    L, tabs = f.L, f.L._mx_tabs
    y = torch.empty(f.N, 64, dtype=torch.bfloat16, device="cuda")
    good = [f.x.data_ptr(), f.d_src.data_ptr(), f.d_offsets.data_ptr(), tabs[0].data_ptr(), tabs[1].data_ptr(), y.data_ptr(), None, None, None, f.T, None]

    def status(**change):
        a = list(good)
        for i, v in change.items():
            a[int(i[1:])] = v
        return L.L.revive_mx_expert_ffn(L._ctx, *a)

    for i in range(6):
        assert status(**{f"_{i}": None}) == -1
    assert status(_9=-1) == -1 and status(_9=f.T + 1) == -1
    assert status(_8=y.data_ptr()) == -1                       # the layer has no shared expert
    assert status(_5=y.data_ptr() + 8) == -1 and status(_0=f.x.data_ptr() + 1) == -1
    assert status(_9=0) == 0
    with pytest.raises(AssertionError):
        L.set_mx_expert_weights([torch.zeros(3, dtype=torch.uint8, device="cuda")], [None])
    L.close()
    cfg = SimpleNamespace(T=2, H=64, E=1, k=1, I=64, I_shared=0, n_ranks=1, slots_per_rank=1, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="fp32")
    fp32 = ReviveLayer(cfg)
    assert fp32.L.revive_mx_expert_ffn(fp32._ctx, *good) == -1
    fp32.close()


# ---- which kernel serves a call does not show ----------------------------------------------------


# few tokens (their rows are rounded on the way): row counts around its limit, slots with several row tiles, K that ends inside a
# step and inside a group, workgroups of two wavefronts and of four (many slots and wide matrices)
@pytest.mark.parametrize("H,I,I_shared,k,rows,T", [(64, 64, 0, 1, [1], 1), (1088, 192, 64, 3, [1, 0, 2], 1), (192, 576, 320, 3, [40, 0, 5], 15),
                                                   (704, 64, 64, 3, [17, 16, 15], 16), (704, 64, 64, 3, [17, 17, 17], 17), (192, 512, 0, 20, [16] * 20, 16),
                                                   (1088, 64, 64, 20, [16] * 20, 16), (192, 1024, 0, 8, [16] * 20, 40), (2112, 64, 64, 8, [16] * 20, 40)])
def test_ffn_of_few_tokens(H, I, I_shared, k, rows, T):
    f = Ffn(H, I, k, rows, I_shared, T, seed=H + T)
    f.check(*f.run())
    f.L.close()


# up to four rows of a row-tile, and more of them in one slot than there are tokens; workgroups of one wavefront (sizes that would
# leave some CUs twice the work with two)
@pytest.mark.parametrize("H,I,I_shared,k,rows,T", [(64, 64, 64, 1, [1], 1), (64, 64, 0, 3, [4, 0, 5], 3), (192, 320, 64, 3, [0, 12, 0], 4),
                                                   (576, 704, 192, 4, [3, 5, 0, 4, 8], 5), (1600, 704, 0, 20, [4] * 20, 4),
                                                   (1600, 704, 64, 20, [40, 0, 37] + [0] * 17, 4)])
def test_ffn_of_few_rows(H, I, I_shared, k, rows, T):
    f = Ffn(H, I, k, rows, I_shared, T, seed=I + T)
    f.check(*f.run())
    f.L.close()


def test_ffn_of_few_tokens_that_are_not_finite():
    f = Ffn(576, 128, 2, [9, 4, 0, 5], 64, seed=8)
    clean, clean_shared = (f64(t) for t in f.run())
    f.x[3, 570], f.x[7, 0] = float("nan"), -float("inf")
    y, shared = (f64(t) for t in f.run())
    touched = np.isin(f.src_of // 2, [3, 7])
    assert np.isnan(y[touched]).all() and np.array_equal(y[~touched], clean[~touched])
    others = [t for t in range(f.T) if t not in (3, 7)]
    assert np.isnan(shared[[3, 7]]).all() and np.array_equal(shared[others], clean_shared[others])
    f.L.close()


@pytest.mark.parametrize("T", [5, 30, 300])
def test_ffn_of_tokens_at_any_address(T):
    f = Ffn(320, 64, 1, [T], 64, T, seed=T)
    y, shared = f.run()
    whole = torch.zeros(T * 320 + 8, dtype=torch.bfloat16, device="cuda")
    for shift in (1, 3, 4):
        x = whole[shift:shift + T * 320].view(T, 320)
        x.copy_(f.x)
        out = (torch.zeros_like(y), torch.zeros_like(shared))
        f.L.mx_expert_ffn(x, f.d_src, f.d_offsets, T, *f.sh, out=out)
        assert torch.equal(out[0], y) and torch.equal(out[1], shared)
    f.L.close()


def test_ffn_does_not_depend_on_the_token_count():
    """The same tokens among more of them: every form of the kernels adds up in the same order."""
    T = 600
    f = Ffn(1088, 704, 1, [T], 576, T, seed=2)
    f.src_of = np.arange(T, dtype=np.int32)
    f.d_src = torch.from_numpy(f.src_of).cuda()
    y, shared = f.run()
    f.check(y, shared)
    for n in (1, 2, 4, 5, 16, 17, 32, 33, 64, 255, 256, 257, 599):
        offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        some, some_shared = f.L.mx_expert_ffn(f.x, f.d_src, offsets, n, *f.sh)
        assert torch.equal(some, y[:n]) and torch.equal(some_shared, shared[:n]), n
    f.L.close()


# more tokens than are rounded on the way and few rows per slot: tiles of 64 rows, slots with one of 16, 32 and 64 rows and with
# several, workgroups of two wavefronts and of four
@pytest.mark.parametrize("H,I,I_shared,k,rows,T", [(192, 1024, 0, 8, [28] * 20, 70), (2112, 64, 64, 8, [28] * 20, 70), (576, 704, 192, 2, [64, 65, 0, 1, 16, 17, 33], 98),
                                                   (64, 64, 0, 1, [1] * 65, 65), (1088, 320, 64, 3, [90, 0, 0, 0, 0, 100, 0, 5], 65)])
def test_ffn_of_few_rows_per_slot(H, I, I_shared, k, rows, T):
    f = Ffn(H, I, k, rows, I_shared, T, seed=H + len(rows))
    f.check(*f.run())
    f.L.close()


def test_ffn_of_few_rows_per_slot_that_are_not_finite_and_at_any_address():
    f = Ffn(576, 128, 1, [30, 40, 0, 10, 20], 64, 100, seed=12)
    clean, clean_shared = (f64(t) for t in f.run())
    whole = torch.zeros(100 * 576 + 8, dtype=torch.bfloat16, device="cuda")
    x = whole[3:3 + 100 * 576].view(100, 576)
    x.copy_(f.x)
    x[3, 570], x[71, 0] = float("nan"), -float("inf")
    y, shared = (f64(t) for t in f.L.mx_expert_ffn(x, f.d_src, f.d_offsets, 100, *f.sh))
    touched = np.isin(f.src_of, [3, 71])
    assert np.isnan(y[touched]).all() and np.array_equal(y[~touched], clean[~touched])
    others = [t for t in range(100) if t not in (3, 71)]
    assert np.isnan(shared[[3, 71]]).all() and np.array_equal(shared[others], clean_shared[others])
    f.L.close()


def test_ffn_does_not_depend_on_the_token_count_with_many_slots():
    """As above where slots without rows keep the average per slot low."""
    T = 200
    f = Ffn(1088, 704, 1, [0, T, 0, 0, 0, 0, 0, 0], 576, T, seed=3)
    f.src_of = np.arange(T, dtype=np.int32)
    f.d_src = torch.from_numpy(f.src_of).cuda()
    y, shared = f.run()
    f.check(y, shared)
    for n in (1, 16, 17, 64, 65, 128, 199):
        offsets = torch.tensor([0, 0] + [n] * 7, dtype=torch.int32, device="cuda")
        some, some_shared = f.L.mx_expert_ffn(f.x, f.d_src, offsets, n, *f.sh)
        assert torch.equal(some, y[:n]) and torch.equal(some_shared, shared[:n]), n
    f.L.close()


def test_ffn_of_few_tokens_and_many_bytes():
    """A layer too large for its tokens to be rounded on the way: the same bits as with fewer of them."""
    P, H, I, T = 96, 5120, 2048, 48
    cfg = SimpleNamespace(T=T, H=H, E=P, k=2, I=I, I_shared=0, n_ranks=1, slots_per_rank=P, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    gen = torch.Generator().manual_seed(1)
    g, d = mx_pack_expert(*((torch.randn(s, generator=gen) * H ** -0.5).cuda() for s in ((H, I), (H, I), (I, H))))
    L.set_mx_expert_weights([g] * P, [d] * P)
    x = torch.randn(T, H, generator=gen).bfloat16().cuda()
    src_of = torch.arange(2 * T, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0] + [min(2 * T, 5 * (p // 4 + 1)) for p in range(P)], dtype=torch.int32, device="cuda")
    y, _ = L.mx_expert_ffn(x, src_of, offsets, T)
    few, _ = L.mx_expert_ffn(x[:12].contiguous(), src_of, offsets.clamp(max=24), 12)
    assert bool(few.any(dim=1).all()) and torch.equal(y[:24], few)
    L.close()
