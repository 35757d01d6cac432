"""The workspace that the bf16 calls need and the one that the 4-bit FFN needs."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import ReviveLayer

pytestmark = pytest.mark.gpu


def test_a_workspace_for_the_bf16_calls_alone():
    """The 4-bit FFN needs more of the workspace than the bf16 calls of a layer with few experts per token do: those run in what they
    need, and it is refused there."""
    T, H = 4096, 7168
    cfg = SimpleNamespace(T=T, H=H, E=4, k=1, I=64, I_shared=0, n_ranks=1, slots_per_rank=4, max_replicas=1, score_fn="softmax", n_group=1,
                          topk_group=1, dtype="bf16")
    L = ReviveLayer(cfg)
    small = torch.empty(2 << 20, dtype=torch.uint8, device="cuda")  # h of 64 numbers a row is 512 KiB, x in 4 bits 14 MiB
    assert L.workspace.numel() > 14 << 20
    gen = torch.Generator().manual_seed(1)
    w = [((torch.randn(256, H, generator=gen) / 64).bfloat16().cuda(), (torch.randn(H, 64, generator=gen) / 8).bfloat16().cuda()) for _ in range(4)]
    L.set_expert_weights([a for a, _ in w], [b for _, b in w])
    x = torch.randn(T, H, generator=gen).bfloat16().cuda()
    phys = (torch.arange(T, dtype=torch.int32, device="cuda") % 4).view(T, 1)

    def layer():
        x_perm, offsets, dst_row, src_of = L.dispatch(x, phys, T)
        return L.expert_ffn(x_perm, offsets, T)[0], src_of, offsets

    want = layer()
    assert L.L.revive_bind_workspace(L._ctx, small.data_ptr(), small.numel()) == 0
    got = layer()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    tab = torch.zeros(4, dtype=torch.int64, device="cuda")
    args = (x.data_ptr(), got[1].data_ptr(), got[2].data_ptr(), tab.data_ptr(), tab.data_ptr(), torch.empty_like(x).data_ptr(), None, None, None)
    assert L.L.revive_mx_expert_ffn(L._ctx, *args, T, None) == -2 and b"workspace" in L.L.revive_last_error(L._ctx)
    assert L.L.revive_bind_workspace(L._ctx, small.data_ptr(), 4096) == -2
    torch.cuda.synchronize()
    L.close()
