"""Every form of the 8-bit products' kernels, which a call does not show: by sizes that its rule sends there."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx8_oracle as mx
from paper_2602_21140_amd import ReviveLayer, mx8_linear, mx8_pack, mx8_pack_expert, mx8_quantize
from test_gpu_mx8 import Ffn, check_ffn
from test_gpu_mx8_linear import Product

pytestmark = pytest.mark.gpu


# tiles of 256 x 256 and of 256 x 128 (256 of these and fewer): K of less than a step, of one, two, three, with a rest of 32, 64 and 96 behind
# each; groups of four steps that end with the row and inside of it; rows that leave one, two, three and four pairs of the last row-tile to multiply
@pytest.mark.parametrize("K", [64, 96, 128, 160, 192, 256, 288, 384, 480, 512, 640, 768, 896, 1024, 1152])
@pytest.mark.parametrize("N", [3457, 2433])
def test_tiles(K, N):
    p = Product(2305 + (K // 32) % 5 * 50, K, N)
    how = dict(bias=K % 64 == 0, activation=("none", "silu", "gelu", "relu")[K // 32 % 4], residual=K % 128 == 0 or K % 96 == 0)
    p.check(p.run(**how), **how)


@pytest.mark.parametrize("K", [544, 512])
@pytest.mark.parametrize("N", [3458, 2434])
def test_tiles_of_strided_and_unaligned_rows_in_place_and_not_finite(K, N):
    rows = 2349
    p = Product(rows, K, N, seed=6)
    want = p.run()
    p.check(want)
    wide = torch.full((2, rows, N + 30), 7.0, dtype=torch.bfloat16, device="cuda")
    out, res = wide[0, :, 5:5 + N], wide[1, :, 3:3 + N]
    res.copy_(p.residual)
    first, p.residual = p.residual, res
    assert torch.equal(p.run(out=out), want)
    out.fill_(7.0)
    assert bool((wide[0] == 7.0).all())
    p.run(out=res)
    assert torch.equal(res, want)
    p.residual = first
    # scales at any address, bytes of NaN behind the last row
    n = K // 32
    codes = torch.full((rows * K + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows * n + 257,), 255, dtype=torch.uint8, device="cuda")
    codes[:rows * K], scales[1:rows * n + 1] = p.form[0].flatten(), p.form[1].flatten()
    p.form = codes[:rows * K].view(rows, K), scales[1:rows * n + 1].view(rows, n)
    assert torch.equal(p.run(), want)
    p.form[1][7, n - 1] = 255
    p.form[0][2300, K - 1] = 0x7F
    got = p.run()
    others = [r for r in range(rows) if r not in (7, 2300)]
    assert bool(got[[7, 2300]].isnan().all()) and torch.equal(got[others], want[others])


# 64 x 64, 32 x 64 and 16 x 64 outputs to a workgroup (224 workgroups and more of each and fewer of the larger ones), and 16 x 32; K below a
# step, with a rest, and with more steps to a wavefront than the 16 whose scales it holds
@pytest.mark.parametrize("rows,N", [(945, 950), (470, 950), (236, 950), (60, 100)])
@pytest.mark.parametrize("K", [32, 96, 640, 1120, 4096, 17440])
def test_streams(rows, N, K):
    p = Product(rows, K, N, seed=7)
    p.check(p.run(activation="gelu"), activation="gelu")
    p.check(p.run(bias=False, residual=False), bias=False, residual=False)


@pytest.mark.parametrize("N", [3456, 2432])
def test_tiles_in_a_graph(N):
    p = Product(2400, 640, N, seed=8)
    out = p.run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        p.run(out=out)
    for i in range(4):
        mx8_quantize(torch.randn(2400, 640, generator=torch.Generator().manual_seed(i)).cuda(), out=p.form)
        want = p.run()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


MANY = [1, 0, 16, 17, 64, 65, 100, 128, 129, 192, 193, 255, 256, 257, 300] + [5, 0, 40] * 12


# tiles (more than 24 rows per slot on average, 36 for the second product, 96 tiles, 2^20 numbers of h): K of whole and of broken steps, scales by words and by bytes, widths that end
# inside a panel; the shared expert beside them, in their launch and in its own
@pytest.mark.parametrize("H,I,I_shared,k,T", [(512, 512, 0, 1, None), (576, 704, 192, 2, 1300), (1024, 512, 576, 1, 2700), (640, 704, 0, 3, None)])
def test_ffn_by_tiles(H, I, I_shared, k, T):
    f = Ffn(H, I, k, MANY, I_shared, T, seed=H)
    f.check(*f.run())
    f.L.close()


# many rows to a slot and too few tiles for the chip
@pytest.mark.parametrize("H,I,I_shared,k,rows,T", [(320, 192, 64, 1, [300, 0, 40], 340), (1152, 128, 0, 2, [64, 65, 63, 0, 1], None)])
def test_ffn_of_many_rows_in_few_slots(H, I, I_shared, k, rows, T):
    f = Ffn(H, I, k, rows, I_shared, T, seed=I)
    f.check(*f.run())
    f.L.close()


def test_ffn_by_tiles_of_rows_that_are_not_finite_and_in_a_graph():
    f = Ffn(576, 512, 1, MANY, 576, sum(MANY), seed=3)
    clean, clean_shared = (t.clone() for t in f.run())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = (torch.zeros_like(clean), torch.zeros_like(clean_shared))
    f.L.graph_begin(stream)
    f.L.mx8_expert_ffn(*f.form, f.d_src, f.d_offsets, f.T, *f.sh, out=out, stream=stream)
    graph = f.L.graph_end(stream)
    for turn in range(4):
        bad = [3 + 11 * turn, 900 + turn]
        x = f.x.clone()
        x[bad[0], 575], x[bad[1], 0] = float("nan"), -float("inf")
        mx8_quantize(x, out=f.form)
        f.run()  # eager work between the replays
        torch.cuda.synchronize()
        f.L.graph_launch(graph, stream)
        stream.synchronize()
        touched = torch.from_numpy(np.isin(f.src_of, bad)).cuda()
        others = torch.tensor([t for t in range(f.T) if t not in bad], device="cuda")
        assert bool(out[0][touched].isnan().all()) and torch.equal(out[0][~touched], clean[~touched])
        assert bool(out[1][bad].isnan().all()) and torch.equal(out[1][others], clean_shared[others])
    f.L.close()


# ---- offsets beyond 32 bits ----------------------------------------------------------------------


def test_quantised_rows_beyond_32_bits():
    rows, K = 140000, 65536
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    some = [0, 65535, 65536, 131071, 131072, rows - 1]
    x[some] = torch.randn(len(some), K, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    codes, scales = mx8_quantize(x)
    want_codes, want_scales = mx.quantize(f64(x[some]))
    assert np.array_equal(codes[some].cpu().numpy(), want_codes) and np.array_equal(scales[some].cpu().numpy(), want_scales)
    assert int((scales != 0).any(dim=1).sum()) == len(some)


@pytest.mark.parametrize("K", [32, 64])  # 64 x 64 outputs to a workgroup, and tiles
def test_results_of_a_product_beyond_32_bits(K):
    rows, N = 1_050_000, 4200
    gen = torch.Generator().manual_seed(K)
    few = torch.randn(4097, K, generator=gen).cuda()
    form = [t[torch.arange(rows, device="cuda") % 4097].contiguous() for t in mx8_quantize(few)]
    w_form = mx8_quantize(torch.randn(N, K, generator=gen).cuda())
    w = mx8_pack(*w_form)
    out = mx8_linear(*form, w, N)
    some = [0, 1, 2 ** 31 // N, 2 ** 31 // N + 1, 2 ** 32 // N, 2 ** 32 // N + 1, rows - 1]
    p = Product.__new__(Product)
    p.x64, p.w64 = (mx.values(*(t.cpu().numpy() for t in f)) for f in ([t[some] for t in form], w_form))
    p.check(out[some], bias=False, residual=False)
    assert torch.equal(out[rows - rows % 4097:], out[:rows % 4097])


# routed rows whose results pass 32 bits, by tiles; and tokens whose codes do (4 GiB), by the streaming kernel
@pytest.mark.parametrize("T,k,P", [(80000, 8, 96), (620000, 1, 8)])
def test_ffn_results_and_tokens_beyond_32_bits(T, k, P):
    H, I = 7168, 64
    cfg = SimpleNamespace(T=T, H=H, E=P, k=k, I=I, I_shared=0, n_ranks=1, slots_per_rank=P, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    gen = torch.Generator().manual_seed(T)
    w = [{n: torch.randn(s, generator=gen) * H ** -0.5 for n, s in (("gate", (H, I)), ("up", (H, I)), ("down", (I, H)))} for _ in range(4)]
    packed = [mx8_pack_expert(*(m.cuda() for m in e.values())) for e in w]
    L.set_mx8_expert_weights([packed[p % 4][0] for p in range(P)], [packed[p % 4][1] for p in range(P)])
    x = torch.randn(4099, H, generator=gen).bfloat16().cuda()
    form = [t[torch.arange(T, device="cuda") % 4099].contiguous() for t in mx8_quantize(x)]
    N = T * k
    ends = sorted([N // 2 - 1000, N // 2, N // 2, N - 700, N - 600, N - 599, N - 300] + [N // 2 + 1000 * p for p in range(P - 8)]) + [N]
    offsets = torch.tensor([0] + ends, dtype=torch.int32, device="cuda")
    src_of = torch.arange(N, dtype=torch.int32, device="cuda")
    y, _ = L.mx8_expert_ffn(*form, src_of, offsets, T)
    values = [mx.expert_values({n: f64(m) for n, m in e.items()}) for e in w]
    x64 = mx.rounded(f64(x))
    for p, (a, b) in enumerate(zip([0] + ends, ends)):
        rows = sorted({r for r in (a, (a + b) // 2, b - 1, 2 ** 31 // H, 2 ** 32 // H, 2 ** 31 // (H // 2)) if a <= r < b})
        if rows:
            check_ffn(f64(y[rows]), x64[[r // k % 4099 for r in rows]], values[p % 4], ("slot", p))
    L.close()


def test_no_tokens():
    cfg = SimpleNamespace(T=4, H=64, E=4, k=2, I=64, I_shared=64, n_ranks=1, slots_per_rank=4, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    L.set_mx8_expert_weights([None] * 4, [None] * 4)
    form = torch.empty(0, 64, dtype=torch.uint8, device="cuda"), torch.empty(0, 2, dtype=torch.uint8, device="cuda")
    y, _ = L.mx8_expert_ffn(*form, none, torch.zeros(5, dtype=torch.int32, device="cuda"), 0)
    assert y.shape == (0, 64)
    L.close()
