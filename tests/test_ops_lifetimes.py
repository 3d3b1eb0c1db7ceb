"""What the binding hands to the library as a pointer lives until the library's call has returned (CPU only: the library's
call is a stand-in that looks who is still alive)."""
import weakref

import pytest


class Host:
    device = -1  # what a tensor on the host says of itself


@pytest.fixture
def calls(monkeypatch):
    """The names of the calls made, each with how many of the tensors whose pointers were taken for it are gone."""
    from paper_2609_13544_gb300 import ops, ops4
    made, taken = [], []

    def watched(f):
        def g(h, t, *rest):
            if t is not None:
                taken.append(weakref.ref(t))
            return f(h, t, *rest)
        return g

    def call(h, name, *args):
        made.append((name, sum(t() is None for t in taken)))
        taken.clear()
    for f in ("_matrix", "_vector"):
        w = watched(getattr(ops, f))
        monkeypatch.setattr(ops, f, w)
        monkeypatch.setattr(ops4, f, w)
    monkeypatch.setattr(ops4, "_like", watched(ops4._like))
    for m in (ops, ops4):
        monkeypatch.setattr(m, "_call", call)
        monkeypatch.setattr(m, "_stream", lambda h, stream: 0)
    return made


def test_layers_keep_their_copies(calls):
    """Leading dimensions in another order than memory's: whatever has to be copied is kept until the call."""
    import torch
    import paper_2609_13544_gb300 as peat
    turned = lambda *shape, dtype=torch.float32: torch.zeros(shape[1], shape[0], *shape[2:], dtype=dtype).transpose(0, 1)
    layer = peat.Linear8(Host, torch.zeros(4, 32))
    bias = torch.zeros(4)
    layer.forward(turned(3, 5, 32), bias)
    layer.backward(turned(3, 5, 4), turned(3, 5, 32))
    q, scale = turned(3, 5, 32, dtype=torch.int8), turned(3, 5)
    layer.forward_rounded(q, scale, bias=bias)
    layer.forward_rounded(q.contiguous(), scale.contiguous(), bias=bias)
    norm = peat.RMSNorm8(Host, torch.zeros(32))
    norm.forward(turned(3, 5, 32), turned(3, 5, 32))
    norm.backward(turned(3, 5, 32), turned(3, 5, 32), turned(3, 5), turned(3, 5, 32))
    assert [name for name, _ in calls] == (["peat_quantize_i8"] * 2 + ["peat_product_i8"] * 5 + ["peat_rmsnorm",
                                                                                                "peat_rmsnorm_backward"])
    assert [gone for _, gone in calls] == [0] * len(calls), calls
