"""What the norm, the 8-bit calls and the 8-bit FFN of the binding refuse before the library is called, on tensors that only say where
they are."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import ReviveLayer, add_rms_norm, binding, mx8_dequantize, mx8_linear, mx8_pack, mx8_quantize


class OnDevice(torch.Tensor):
    is_cuda = property(lambda self: True)
    place = 0

    def get_device(self):
        return self.place


class Elsewhere(OnDevice):
    place = 1


def t(*shape, dtype=torch.bfloat16, kind=OnDevice):
    return torch.zeros(*shape, dtype=dtype).as_subclass(kind)


def u8(*shape, kind=OnDevice):
    return t(*shape, dtype=torch.uint8, kind=kind)


def no_library(*_args):
    raise AssertionError("the library was called")


def library(monkeypatch, status):
    real = binding.lib()
    calls = {n: status for n in ("revive_add_rms_norm", "revive_mx_eight_quantize", "revive_mx_eight_dequantize", "revive_mx_eight_pack", "revive_mx_eight_linear")}
    monkeypatch.setattr(binding, "lib", lambda: SimpleNamespace(revive_mx_eight_packed_bytes=real.revive_mx_eight_packed_bytes,
                                                            revive_last_error=real.revive_last_error, revive_status_name=real.revive_status_name, **calls))
    monkeypatch.setattr(binding, "_get_device", lambda: 0)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)


@pytest.fixture
def refused(monkeypatch):
    library(monkeypatch, no_library)


@pytest.fixture
def taken(monkeypatch):
    library(monkeypatch, lambda *a: 0)


STREAM = SimpleNamespace(cuda_stream=0, device_index=0)
ROWS, H, N = 3, 70, 40


def norm(**change):
    a = dict(x=t(ROWS, H), weight=t(H), residual=t(ROWS, H), quantize=True, out=(t(ROWS, H), t(ROWS, H), u8(ROWS, 96), u8(ROWS, 3)), stream=STREAM)
    return {**a, **change}


def linear(**change):
    a = dict(codes=u8(ROWS, 96), scales=u8(ROWS, 3), w=u8(binding.mx8_packed_bytes(N, 96)), n_out=N, bias=t(N, dtype=torch.float32), activation="silu",
             residual=t(ROWS, N), out=t(ROWS, N), stream=STREAM)
    return {**a, **change}


def test_what_fits_is_taken(taken):
    add_rms_norm(**norm())
    add_rms_norm(**norm(out=(None, None, u8(ROWS, 96), u8(ROWS, 3))))
    add_rms_norm(**norm(residual=None, quantize=False, out=(None, t(ROWS, H), None, None)))
    add_rms_norm(**norm(x=t(ROWS, H + 9)[:, 5:5 + H], residual=t(ROWS, H + 2)[:, :H]))
    mx8_linear(**linear())
    mx8_linear(**linear(bias=None, residual=None, activation="none", out=t(ROWS, 60)[:, 3:3 + N]))
    mx8_quantize(t(ROWS, H), out=(u8(ROWS, 96), u8(ROWS, 3)), stream=STREAM)
    mx8_dequantize(u8(ROWS, 96), u8(ROWS, 3), out=t(ROWS, H), stream=STREAM)
    mx8_pack(u8(N, 96), u8(N, 3), out=u8(binding.mx8_packed_bytes(N, 96)), stream=STREAM)


@pytest.mark.parametrize("change", [
    dict(x=t(ROWS, H, dtype=torch.float16)), dict(x=t(H)), dict(x=t(H, ROWS).t()), dict(x=torch.zeros(ROWS, H, dtype=torch.bfloat16)),
    dict(weight=t(H - 1)), dict(weight=t(H, dtype=torch.float32)), dict(weight=t(2 * H)[::2]), dict(weight=torch.zeros(H, dtype=torch.bfloat16)),
    dict(residual=t(ROWS, H + 1)), dict(residual=t(ROWS, H, dtype=torch.float32)), dict(residual=t(H, ROWS).t()),
    dict(residual=torch.zeros(ROWS, H, dtype=torch.bfloat16)), dict(residual=t(ROWS, H, kind=Elsewhere)),
    dict(quantize=False), dict(out=(t(ROWS, H), t(ROWS, H), None, None)), dict(out=(t(ROWS, H), t(ROWS, H), u8(ROWS, 96), None)),
    dict(out=(t(ROWS, H), t(ROWS, H), u8(ROWS, 70), u8(ROWS, 3))), dict(out=(t(ROWS, H + 1)[:, :H], t(ROWS, H), u8(ROWS, 96), u8(ROWS, 3))),
    dict(out=(t(ROWS, H), t(ROWS, H, dtype=torch.float32), u8(ROWS, 96), u8(ROWS, 3))),
    dict(out=(t(ROWS, H), torch.zeros(ROWS, H, dtype=torch.bfloat16), u8(ROWS, 96), u8(ROWS, 3))),
    dict(out=(t(ROWS, H), t(ROWS, H), u8(ROWS, 96, kind=Elsewhere), u8(ROWS, 3))), dict(stream=SimpleNamespace(cuda_stream=0, device_index=1))])
def test_norm_refuses(refused, change):
    with pytest.raises((ValueError, TypeError)):
        add_rms_norm(**norm(**change))


@pytest.mark.parametrize("change", [
    dict(codes=u8(ROWS, 95)), dict(codes=u8(ROWS, 192)[:, ::2]), dict(codes=t(ROWS, 96)), dict(scales=u8(ROWS + 1, 3)), dict(scales=u8(9)),
    dict(codes=torch.zeros(ROWS, 96, dtype=torch.uint8)), dict(w=u8(binding.mx8_packed_bytes(N, 96) - 16)), dict(w=t(binding.mx8_packed_bytes(N, 96))),
    dict(n_out=N + 128), dict(n_out=0), dict(bias=t(N)), dict(bias=t(N + 1, dtype=torch.float32)), dict(activation="tanh"), dict(activation=None),
    dict(residual=t(ROWS, N, dtype=torch.float32)), dict(residual=t(ROWS, N + 1)), dict(residual=t(N, ROWS).t()), dict(out=t(ROWS, N, dtype=torch.float32)),
    dict(out=t(ROWS + 1, N)), dict(out=t(N, ROWS).t()), dict(out=t(ROWS, N, kind=Elsewhere)), dict(bias=torch.zeros(N)),
    dict(stream=SimpleNamespace(cuda_stream=0, device_index=1))])
def test_linear_refuses(refused, change):
    with pytest.raises((ValueError, TypeError, binding.ReviveError)):
        mx8_linear(**linear(**change))


def test_rounding_and_packing_refuse(refused):
    for call in (lambda: mx8_quantize(t(ROWS, H, dtype=torch.float16)), lambda: mx8_quantize(t(H)), lambda: mx8_quantize(t(H, ROWS).t()),
                 lambda: mx8_quantize(t(ROWS, H), out=(u8(ROWS, 96), u8(ROWS, 2))), lambda: mx8_quantize(t(ROWS, H), out=(u8(ROWS, 96), u8(ROWS, 3, kind=Elsewhere))),
                 lambda: mx8_quantize(t(ROWS, H, kind=Elsewhere), out=(u8(ROWS, 96, kind=Elsewhere), u8(ROWS, 3, kind=Elsewhere))),
                 lambda: mx8_dequantize(u8(ROWS, 96), u8(ROWS, 3), 97, out=t(ROWS, H)), lambda: mx8_dequantize(u8(ROWS, 96), u8(ROWS, 3), out=t(ROWS, 97)),
                 lambda: mx8_dequantize(u8(ROWS, 96), u8(ROWS, 3), out=t(ROWS, H, dtype=torch.float16)), lambda: mx8_pack(u8(N, 96), u8(N * 3)),
                 lambda: mx8_pack(u8(N, 96), u8(N, 2)), lambda: mx8_pack(u8(N, 96), u8(N, 3), out=u8(16)),
                 lambda: mx8_pack(u8(N, 96), u8(N, 3), out=torch.zeros(binding.mx8_packed_bytes(N, 96), dtype=torch.uint8))):
        with pytest.raises((ValueError, TypeError)):
            call()


# ---- the FFN -------------------------------------------------------------------------------------

HID, I, I_SHARED, K, P, T = 128, 64, 192, 2, 3, 5
GATE_UP, DOWN = 2 * binding.mx8_packed_bytes(I, HID), binding.mx8_packed_bytes(HID, I)
SHARED = [2 * binding.mx8_packed_bytes(I_SHARED, HID), binding.mx8_packed_bytes(HID, I_SHARED)]


def layer(call, I_shared=I_SHARED):
    L = object.__new__(ReviveLayer)
    L.cfg = SimpleNamespace(H=HID, I=I, I_shared=I_shared, k=K)
    L.P, L.T_max, L.device, L.dtype, L._ctx, L._mx8_tabs = P, T, torch.device("cpu"), torch.bfloat16, None, None
    L.L = SimpleNamespace(revive_mx_eight_expert_ffn=call)
    L.set_mx8_expert_weights([u8(GATE_UP), None, u8(GATE_UP)], [u8(DOWN), None, u8(DOWN)])
    return L


def ffn(**change):
    i32 = torch.int32
    a = dict(codes=u8(T, HID), scales=u8(T, HID // 32), src_of=t(T * K, dtype=i32), slot_offsets=t(P + 1, dtype=i32), T=T, w_sh_gate_up=u8(SHARED[0]),
             w_sh_down=u8(SHARED[1]), out=(t(T * K, HID), t(T, HID)), stream=STREAM)
    return {**a, **change}


def test_ffn_takes_what_fits(taken):
    L = layer(lambda *a: 0)
    L.mx8_expert_ffn(**ffn())
    L.mx8_expert_ffn(**ffn(w_sh_gate_up=None, w_sh_down=None, out=(t(T * K, HID), None)))
    L.mx8_expert_ffn(**ffn(T=2))  # the first tokens of more
    layer(lambda *a: 0, 0).mx8_expert_ffn(**ffn(w_sh_gate_up=None, w_sh_down=None, out=(t(T * K, HID), None)))


@pytest.mark.parametrize("change", [
    dict(codes=torch.zeros(T, HID, dtype=torch.uint8)), dict(codes=u8(T - 1, HID)), dict(codes=u8(T, HID + 64)), dict(codes=t(T, HID)),
    dict(scales=u8(T, 3)), dict(scales=u8(T - 1, 4)), dict(scales=torch.zeros(T, 4, dtype=torch.uint8)), dict(scales=u8(T, 8)[:, ::2]),
    dict(src_of=t(T * K, dtype=torch.int64)), dict(src_of=t(T * K - 1, dtype=torch.int32)), dict(src_of=t(2 * T * K, dtype=torch.int32)[::2]),
    dict(src_of=torch.zeros(T * K, dtype=torch.int32)), dict(slot_offsets=t(P, dtype=torch.int32)), dict(slot_offsets=t(P + 1, dtype=torch.int64)),
    dict(w_sh_gate_up=u8(SHARED[0] - 16)), dict(w_sh_down=u8(SHARED[1] + 16)), dict(w_sh_down=None), dict(w_sh_gate_up=None), dict(w_sh_gate_up=t(SHARED[0])),
    dict(w_sh_gate_up=torch.zeros(SHARED[0], dtype=torch.uint8)), dict(out=(t(T * K, HID), None)), dict(out=(t(T * K - 1, HID), t(T, HID))),
    dict(out=(t(T * K, HID), t(T - 1, HID))), dict(out=(t(T * K, HID, dtype=torch.float32), t(T, HID))),
    dict(out=(torch.zeros(T * K, HID, dtype=torch.bfloat16), t(T, HID))), dict(out=(t(T * K, HID), t(T, HID, kind=Elsewhere))),
    dict(slot_offsets=t(P + 1, dtype=torch.int32, kind=Elsewhere)), dict(stream=SimpleNamespace(cuda_stream=0, device_index=1))])
def test_ffn_refuses(refused, change):
    with pytest.raises(ValueError):
        layer(no_library).mx8_expert_ffn(**ffn(**change))


def test_ffn_refuses_what_the_layer_does_not_have(refused):
    with pytest.raises(ValueError):
        layer(no_library, 0).mx8_expert_ffn(**ffn())
    L = layer(no_library)
    L.device = torch.device("cuda:1")
    with pytest.raises(ValueError):
        L.mx8_expert_ffn(**ffn())
    for gate_up, down in ((torch.zeros(GATE_UP, dtype=torch.uint8), u8(DOWN)), (None, u8(DOWN)), (u8(GATE_UP), None), (u8(GATE_UP - 16), u8(DOWN))):
        with pytest.raises(AssertionError):
            L.set_mx8_expert_weights([gate_up, None, None], [down, None, None])
