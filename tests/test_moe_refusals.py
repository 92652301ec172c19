"""What the router and the experts' products refuse, on the host and before anything touches a GPU."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2609_40093_b200 import ep

p = ctypes.c_void_p(256)                                        # never dereferenced: every case fails on the host


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def _router(T=16, E=8, K=2, dtype=0, scoring=0):
    return ep._Router(T, E, K, dtype, scoring, 1, 1.0, 0.1)


def test_router_limits():
    L = ep.lib()
    bal = ep._Balance(256, 256, 256, 256)
    for bad in (_router(T=-1), _router(E=0), _router(E=4097), _router(K=0), _router(K=33), _router(T=1 << 30, K=2), _router(dtype=2),
                _router(scoring=2)):
        assert L.ep_route(ctypes.byref(bad), p, None, p, p, None, None, None, 0, None) == -2
        assert L.ep_balance_loss(ctypes.byref(bad), p, p, ctypes.byref(bal), None, p, 1 << 20, None) == -2
        assert L.ep_route_backward(ctypes.byref(bad), p, p, p, None, None, p, None) == -2
        assert L.ep_route_workspace_bytes(ctypes.byref(bad)) == 0
    ok = ctypes.byref(_router())
    need = L.ep_route_workspace_bytes(ok)
    assert need > 0
    assert L.ep_route(None, p, None, p, p, None, None, None, 0, None) == -1
    for args in ((None, None, p, p), (p, None, None, p), (p, None, p, None)):
        assert L.ep_route(ok, *args, None, None, None, 0, None) == -1
    assert L.ep_route(ok, p, None, p, p, ctypes.byref(bal), None, None, need, None) == -1       # no workspace
    assert L.ep_route(ok, p, None, p, p, ctypes.byref(bal), None, p, need - 1, None) == -3
    assert L.ep_route(ok, p, None, p, p, ctypes.byref(bal), None, ctypes.c_void_p(264), need, None) == -2
    assert L.ep_route(ok, p, None, p, p, ctypes.byref(ep._Balance(256, 256, None, 256)), None, p, need, None) == -1
    assert L.ep_balance_loss(ok, p, p, None, None, p, need, None) == -1
    assert L.ep_route_backward(ok, p, p, None, None, None, p, None) == -2                       # the gradient of nothing
    assert L.ep_route_backward(ok, p, p, None, ctypes.byref(bal), None, p, None) == -1          # no d_loss
    assert L.ep_route_backward(ok, p, None, p, None, None, p, None) == -1


def _mm(rows=16, H=64, N=64, E=4, act=0, op=0):
    return ep._Matmul(rows, H, N, E, act, op)


def test_expert_product_limits():
    L = ep.lib()
    odd = ctypes.c_void_p(264)
    for bad in (_mm(rows=-1), _mm(rows=1 << 31), _mm(H=60), _mm(N=4), _mm(N=12), _mm(E=0), _mm(E=4097), _mm(act=4), _mm(act=-1), _mm(op=2),
                _mm(H=1 << 24)):
        assert L.ep_expert_matmul(ctypes.byref(bad), p, p, p, None, None, p, None, None, None) == -2
        assert L.ep_expert_matmul_backward(ctypes.byref(bad), p, p, p, p, p, None, p, p, None, None, None, p, 1 << 30, None) == -2
        assert L.ep_expert_matmul_backward_workspace_bytes(ctypes.byref(bad)) == 0
    ok = ctypes.byref(_mm())
    assert L.ep_expert_matmul(None, p, p, p, None, None, p, None, None, None) == -1
    for args in ((None, p, p, None, None, p), (p, None, p, None, None, p), (p, p, None, None, None, p), (p, p, p, None, None, None)):
        assert L.ep_expert_matmul(ok, *args, None, None, None) == -1
    for args in ((odd, p, p, None, None, p), (p, p, odd, None, None, p), (p, p, p, odd, None, p), (p, p, p, None, odd, p), (p, p, p, None, None, odd)):
        assert L.ep_expert_matmul(ok, *args, None, None, None) == -2
    need = L.ep_expert_matmul_backward_workspace_bytes(ok)
    assert need > 0

    def backward(m=_mm(), dy=p, x=p, off=p, w=p, pre=p, operand=None, dx=p, dw=p, db=None, dop=None, ws=p, n=need):
        return L.ep_expert_matmul_backward(ctypes.byref(m), dy, x, off, w, pre, operand, dx, dw, db, dop, None, ws, n, None)

    assert backward(n=need - 1) == -3
    assert backward(ws=None) == -1 and backward(ws=odd) == -2
    assert backward(dy=None) == -1 and backward(off=None) == -1 and backward(w=None) == -1 and backward(x=None) == -1
    assert backward(m=_mm(act=ep.ACT_GELU), pre=None) == -1                       # an activation's slope needs z
    assert backward(dop=p) == -2 and backward(operand=p, dop=p) == -2             # no operand, or an added one: its gradient is dy
    assert backward(dx=odd) == -2 and backward(db=odd) == -2


def test_binding_refuses_types_shapes_and_strides():
    r = ep.Router(8, 2)
    with pytest.raises(TypeError, match="logits"):
        ep.ep_route(torch.zeros(4, 8, dtype=torch.float64), r)
    with pytest.raises(ValueError, match="logits"):
        ep.ep_route(torch.zeros(4, 9), r)
    with pytest.raises(ValueError, match="contiguous"):
        ep.ep_route(torch.zeros(4, 16)[:, ::2], r, out=ep.alloc_routing(4, 8, 2, device="cpu"))
    with pytest.raises(ValueError, match="topk_idx"):
        ep.ep_route(torch.zeros(4, 8), r, out=ep.alloc_routing(4, 8, 3, device="cpu"))
    with pytest.raises(TypeError, match="bias"):
        ep.ep_route(torch.zeros(4, 8), r, bias=torch.zeros(8, dtype=torch.bfloat16), out=ep.alloc_routing(4, 8, 2, device="cpu"))
    with pytest.raises(ValueError, match="balance"):
        ep.ep_balance_loss(torch.zeros(4, 8), r, torch.zeros(4, 2, dtype=torch.int32), out=ep.alloc_routing(4, 8, 2, device="cpu"))
    routing = ep.alloc_routing(4, 8, 2, device="cpu")
    with pytest.raises(ValueError, match="counts"):
        ep.ep_route_backward(torch.zeros(4, 8), r, routing, d_loss=torch.ones(1))
    with pytest.raises(TypeError, match="dlogits"):
        ep.ep_route_backward(torch.zeros(4, 8), r, routing, d_weights=torch.zeros(4, 2), dlogits=torch.zeros(4, 8, dtype=torch.bfloat16))
    bf = torch.bfloat16
    x, off, w = torch.zeros(6, 16, dtype=bf), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 8, 16, dtype=bf)
    with pytest.raises(TypeError, match="x must be"):
        ep.ep_expert_matmul(x.float(), off, w)
    with pytest.raises(ValueError, match="x must be"):
        ep.ep_expert_matmul(torch.zeros(6, 24, dtype=bf), off, w)
    with pytest.raises(ValueError, match="expert_offsets"):
        ep.ep_expert_matmul(x, off[:2], w)
    with pytest.raises(TypeError, match="expert_offsets"):
        ep.ep_expert_matmul(x, off.long(), w)
    with pytest.raises(ValueError, match="operand"):
        ep.ep_expert_matmul(x, off, w, operand=torch.zeros(6, 16, dtype=bf))
    with pytest.raises(ValueError, match="contiguous"):
        ep.ep_expert_matmul(torch.zeros(6, 32, dtype=bf)[:, ::2], off, w)
    with pytest.raises(ValueError, match="dy"):
        ep.ep_expert_matmul_backward(torch.zeros(6, 16, dtype=bf), x, off, w, grads=ep.alloc_expert_grads(6, 16, 8, 2, device="cpu"))


def test_binding_refuses_host_tensors():
    """An address of host memory would fault on the GPU: every tensor has to be on the first one's CUDA device."""
    with pytest.raises(ValueError, match="CUDA"):
        ep.ep_route(torch.zeros(4, 8), ep.Router(8, 2), out=ep.alloc_routing(4, 8, 2, device="cpu"))
    bf = torch.bfloat16
    x, off, w = torch.zeros(6, 16, dtype=bf), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 8, 16, dtype=bf)
    with pytest.raises(ValueError, match="CUDA"):
        ep.ep_expert_matmul(x, off, w)
    with pytest.raises(ValueError, match="CUDA"):
        ep.ep_expert_matmul_backward(torch.zeros(6, 8, dtype=bf), x, off, w, grads=ep.alloc_expert_grads(6, 16, 8, 2, device="cpu"))


@pytest.mark.gpu
def test_binding_refuses_a_mix_of_devices():
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_route(torch.zeros(4, 8, device="cuda"), ep.Router(8, 2), out=ep.alloc_routing(4, 8, 2, device="cpu"))
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_route(torch.zeros(4, 8, device="cuda"), ep.Router(8, 2), bias=torch.zeros(8))
    bf = torch.bfloat16
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_expert_matmul(torch.zeros(6, 16, dtype=bf, device="cuda"), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 8, 16, dtype=bf, device="cuda"))
