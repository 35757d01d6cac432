"""The microscaled 4-bit calls where offsets pass 32 bits, on sampled rows, and where there is nothing to do."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from harness import f64
from oracle import mx_oracle as mx
from paper_2602_21140_amd import ReviveLayer, mx_dequantize, mx_pack_expert, mx_quantize
from test_gpu_mx import check_ffn

pytestmark = pytest.mark.gpu


def test_rows_that_are_two_billion_elements_apart():
    whole = torch.zeros(2 ** 32 + 128, dtype=torch.bfloat16, device="cuda")
    rows = whole.as_strided((3, 100), (2 ** 31, 1))
    rows.copy_(torch.randn(3, 100, generator=torch.Generator().manual_seed(1)).cuda())
    codes, scales = mx_quantize(rows)
    want_codes, want_scales = mx.quantize(f64(rows))
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy(), want_scales)
    rows.zero_()
    mx_dequantize(codes, scales, out=rows)
    assert np.array_equal(f64(rows), mx.values(want_codes, want_scales)[:, :100])
    assert not whole[100:2 ** 31].any() and not whole[2 ** 32 + 100:].any()


def test_codes_beyond_four_gib():
    rows, K = 140000, 65536
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    some = [0, 65535, 65536, 131071, 131072, rows - 1]
    x[some] = torch.randn(len(some), K, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    codes, scales = mx_quantize(x)
    want_codes, want_scales = mx.quantize(f64(x[some]))
    assert np.array_equal(codes[some].cpu().numpy(), want_codes) and np.array_equal(scales[some].cpu().numpy(), want_scales)
    assert int((scales != 0).any(dim=1).sum()) == len(some)
    back = mx_dequantize(codes, scales)
    assert np.array_equal(f64(back[some]), mx.values(want_codes, want_scales))
    assert int((back != 0).any(dim=1).sum()) == len(some)


# routed rows whose results pass 32 bits, by tiles; and tokens whose codes do (4 GiB), by the streaming kernel
@pytest.mark.parametrize("T,k", [(80000, 8), (1250000, 1)])
def test_ffn_results_and_tokens_beyond_32_bits(T, k):
    H, I, P = 7168, 64, 8
    cfg = SimpleNamespace(T=T, H=H, E=P, k=k, I=I, I_shared=0, n_ranks=1, slots_per_rank=P, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    gen = torch.Generator().manual_seed(T)
    w = [{n: torch.randn(s, generator=gen) * H ** -0.5 for n, s in (("gate", (H, I)), ("up", (H, I)), ("down", (I, H)))} for _ in range(P)]
    packed = [mx_pack_expert(*(m.cuda() for m in e.values())) for e in w]
    L.set_mx_expert_weights([a for a, _ in packed], [b for _, b in packed])
    x = torch.randn(4099, H, generator=gen).bfloat16().cuda()[torch.arange(T, device="cuda") % 4099]
    N = T * k
    ends = [N // 2 - 1000, N // 2, N // 2, N - 700, N - 600, N - 599, N - 300, N]  # long slots, one without rows, one with a row
    offsets = torch.tensor([0] + ends, dtype=torch.int32, device="cuda")
    src_of = torch.arange(N, dtype=torch.int32, device="cuda")
    y, _ = L.mx_expert_ffn(x, src_of, offsets, T)
    for p, (a, b) in enumerate(zip([0] + ends, ends)):
        rows = sorted({r for r in (a, a + 1, (a + b) // 2, b - 2, b - 1, 2 ** 31 // H, 2 ** 32 // H, 2 ** 31 // (H // 2)) if a <= r < b})
        if rows:
            values = mx.expert_values({n: f64(m) for n, m in w[p].items()})
            check_ffn(f64(y[rows]), mx.rounded(f64(x[[r // k for r in rows]])), values, ("slot", p))
    L.close()


def test_no_tokens():
    cfg = SimpleNamespace(T=4, H=64, E=4, k=2, I=64, I_shared=64, n_ranks=1, slots_per_rank=4, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    offsets, _, _ = L.dispatch_index(none, 0, out=(torch.full((5,), 7, dtype=torch.int32, device="cuda"), none, none))
    assert not offsets.any()
    L.set_mx_expert_weights([None] * 4, [None] * 4)
    y, _ = L.mx_expert_ffn(torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), none, offsets, 0)
    assert y.shape == (0, 64)
    L.close()
