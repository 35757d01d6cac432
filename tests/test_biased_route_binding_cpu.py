"""What the gate with a balance bias and the dispatch without rows refuse before the library is called."""
from types import SimpleNamespace

import pytest
import torch

from paper_2602_21140_amd import ReviveLayer
from test_mx_binding_cpu import no_library, on_device

E, K, P, T = 16, 2, 5, 3
I32, F32 = torch.int32, torch.float32


def layer(call=no_library):
    L = object.__new__(ReviveLayer)
    L.cfg, L.P, L._ctx = SimpleNamespace(E=E, k=K), P, None
    L.L = SimpleNamespace(revive_route_biased=call, revive_dispatch_index=call)
    return L


def route(L, **change):
    a = dict(x=None, w_router=None, bias=on_device(E, dtype=F32), T=T, logits=on_device(T, E, dtype=F32), logits_given=True,
             out=(on_device(T, K, dtype=I32), on_device(T, K, dtype=F32), on_device(T, K, dtype=I32)), stream=SimpleNamespace(cuda_stream=0))
    return L.route_biased(**{**a, **change})


def index(L, **change):
    a = dict(topk_phys=on_device(T, K, dtype=I32), T=T, out=tuple(on_device(n, dtype=I32) for n in (P + 1, T * K, T * K)), stream=SimpleNamespace(cuda_stream=0))
    return L.dispatch_index(**{**a, **change})


def test_what_fits_is_taken():
    L = layer(lambda *a: 0)
    route(L), route(L, T=2), index(L), index(L, T=0), index(L, T=0, topk_phys=None, out=(on_device(P + 1, dtype=I32), None, None))


@pytest.mark.parametrize("change", [
    dict(logits=on_device(T, E)), dict(logits=on_device(T - 1, E, dtype=F32)), dict(logits=torch.zeros(T, E)), dict(logits=on_device(E, T, dtype=F32).t()),
    dict(bias=on_device(E - 1, dtype=F32)), dict(bias=on_device(E))])
def test_route_refuses(change):
    with pytest.raises(ValueError):
        route(layer(), **change)


@pytest.mark.parametrize("change", [dict(topk_phys=on_device(T, K, dtype=torch.int64)), dict(topk_phys=on_device(T - 1, K, dtype=I32)),
                                    dict(topk_phys=torch.zeros(T, K, dtype=I32)), dict(topk_phys=on_device(K, T, dtype=I32).t())])
def test_index_refuses(change):
    with pytest.raises(ValueError):
        index(layer(), **change)
