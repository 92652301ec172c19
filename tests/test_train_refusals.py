"""What the sort's, combine's, dropout's and adapters' calls refuse, on the host and before anything touches a GPU."""
import copy
import ctypes
import pickle

import pytest
import torch

import __graft_entry__ as entry
from paper_2609_40093_b200 import ep

p, odd = ctypes.c_void_p(256), ctypes.c_void_p(264)             # never dereferenced: every case fails on the host
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def _drop(state=256, p=0.1, site=0):
    return ctypes.byref(ep._Dropout(state, p, site))


def test_row_calls():
    L = ep.lib()

    def sort(s=None, x=p, slot=p, w=p, out=p, rows=32):
        return L.ep_sort(ctypes.byref(s or ep._shape(16, 2, 64, 1, 1)), x, slot, w, out, rows, None, None)

    def sort_backward(s=None, d=p, rows=32, slot=p, w=p, x=p, add=None, dx=p, dw=p):
        return L.ep_sort_backward(ctypes.byref(s or ep._shape(16, 2, 64, 1, 1)), d, rows, slot, w, x, add, dx, dw, None, None)

    def combine(s=None, out=p, rows=32, slot=p, w=p, res=None, drop=None, y=p):
        return L.ep_combine_residual(ctypes.byref(s or ep._shape(16, 2, 64, 1, 1)), out, rows, slot, w, res, drop, y, None, None)

    def combine_backward(s=None, dy=p, out=p, rows=32, slot=p, w=p, drop=None, d_out=p, dw=p):
        return L.ep_combine_backward(ctypes.byref(s or ep._shape(16, 2, 64, 1, 1)), dy, out, rows, slot, w, drop, d_out, dw, None, None)

    for bad in (ep._shape(-1, 2, 64, 1, 1), ep._shape(16, 0, 64, 1, 1), ep._shape(16, 33, 64, 1, 1), ep._shape(16, 2, 60, 1, 1),
                ep._shape(16, 2, 0, 1, 1), ep._shape(1 << 30, 2, 64, 1, 1)):
        for call in (sort, sort_backward, combine, combine_backward):
            assert call(s=bad) == -2
    for call in (sort, sort_backward, combine, combine_backward):
        assert call(rows=-1) == -2 and call(slot=None) == -1
    assert L.ep_sort(None, p, p, p, p, 1, None, None) == -1
    assert sort(x=None) == -1 and sort(out=None) == -1 and sort(x=odd) == -2 and sort(out=odd) == -2
    assert sort_backward(d=None) == -1 and sort_backward(x=None) == -1 and sort_backward(dx=None, dw=None) == -1
    assert sort_backward(w=None) == -2                           # unit weights have no gradient
    assert sort_backward(d=odd) == -2 and sort_backward(x=odd) == -2 and sort_backward(add=odd) == -2 and sort_backward(dx=odd) == -2
    assert combine(out=None) == -1 and combine(w=None) == -1 and combine(y=None) == -1
    assert combine(out=odd) == -2 and combine(res=odd) == -2 and combine(y=odd) == -2
    assert combine_backward(dy=None) == -1 and combine_backward(w=None) == -1 and combine_backward(out=None) == -1
    assert combine_backward(d_out=None, dw=None) == -1
    assert combine_backward(dy=odd) == -2 and combine_backward(out=odd) == -2 and combine_backward(d_out=odd) == -2
    for bad in (-0.1, 1.5, float("nan")):
        assert combine(drop=_drop(p=bad)) == -2 and combine_backward(drop=_drop(p=bad)) == -2
        assert L.ep_dropout(p, None, p, 4, 64, None, _drop(p=bad), None) == -2
    assert combine(drop=_drop(state=None)) == -1 and combine(drop=_drop(state=260)) == -2


def test_dropout_limits():
    L = ep.lib()

    def call(x=p, res=None, y=p, rows=4, cols=64):
        return L.ep_dropout(x, res, y, rows, cols, None, _drop(), None)

    assert call(rows=-1) == -2 and call(rows=1 << 31) == -2 and call(cols=60) == -2 and call(cols=0) == -2 and call(cols=-8) == -2
    assert call(x=None) == -1 and call(y=None) == -1 and call(x=odd) == -2 and call(res=odd) == -2 and call(y=odd) == -2
    assert call(rows=(1 << 31) - 1, cols=1 << 20) == -2          # more blocks than a grid has


def _ad(rows=16, entries=16, H=64, N=64, r=8, A=4):
    return ep._Adapter(rows, entries, H, N, r, A)


def test_adapter_limits():
    L = ep.lib()

    def forward(m=None, x=p, off=p, index=p, down=p, up=p, base=p, y=p, mid=p):
        return L.ep_adapter_matmul(ctypes.byref(m or _ad()), x, off, index, down, up, None, base, y, mid, None, None)

    need = L.ep_adapter_matmul_backward_workspace_bytes(ctypes.byref(_ad()))
    assert need > 0

    def backward(m=None, dy=p, x=p, off=p, index=p, down=p, up=p, mid=p, base=p, dx=p, dd=p, du=p, ws=p, n=need):
        return L.ep_adapter_matmul_backward(ctypes.byref(m or _ad()), dy, x, off, index, down, up, None, mid, base, dx, dd, du, None, ws, n, None)

    for bad in (_ad(rows=-1), _ad(rows=1 << 31), _ad(entries=-1), _ad(entries=1 << 31), _ad(H=60), _ad(H=0), _ad(N=4), _ad(N=1 << 24),
                _ad(r=0), _ad(r=12), _ad(r=136), _ad(A=0), _ad(A=4097)):
        assert forward(m=bad) == -2 and backward(m=bad) == -2
        assert L.ep_adapter_matmul_backward_workspace_bytes(ctypes.byref(bad)) == 0
    assert forward(m=_ad(rows=15), index=None) == -2 and backward(m=_ad(rows=15), index=None) == -2      # entry 15 has no row
    assert L.ep_adapter_matmul(None, p, p, p, p, p, None, p, p, p, None, None) == -1
    assert forward(x=None) == -1 and forward(off=None) == -1 and forward(down=None) == -1 and forward(up=None) == -1
    assert forward(y=None, mid=None) == -1
    for name in ("x", "down", "up", "base", "y", "mid"):
        assert forward(**{name: odd}) == -2
    assert backward(dy=None) == -1 and backward(off=None) == -1 and backward(up=None) == -1 and backward(down=None) == -1
    assert backward(x=None) == -1 and backward(mid=None) == -1 and backward(dx=None, dd=None, du=None) == -1
    assert backward(ws=None) == -1 and backward(ws=ctypes.c_void_p(128)) == -2 and backward(n=need - 1) == -3
    for name in ("dy", "x", "down", "up", "mid", "base", "dx", "dd", "du"):
        assert backward(**{name: odd}) == -2


def test_binding_refuses_types_shapes_and_strides():
    x, slot, w = torch.zeros(4, 16, dtype=BF), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    rows = torch.zeros(8, 16, dtype=BF)
    with pytest.raises(TypeError, match="x must be"):
        ep.ep_sort(x.float(), slot, rows)
    with pytest.raises(TypeError, match="slot"):
        ep.ep_sort(x, slot.long(), rows)
    with pytest.raises(ValueError, match="sorted"):
        ep.ep_sort(x, slot, torch.zeros(8, 24, dtype=BF))
    with pytest.raises(ValueError, match="weights"):
        ep.ep_sort(x, slot, rows, weights=torch.zeros(4, 3))
    with pytest.raises(ValueError, match="contiguous"):
        ep.ep_sort(torch.zeros(4, 32, dtype=BF)[:, ::2], slot, rows)
    with pytest.raises(ValueError, match="x must be"):
        ep.ep_sort_backward(rows, slot, x.clone(), weights=w, x=torch.zeros(5, 16, dtype=BF), d_weights=w)
    with pytest.raises(TypeError, match="topk_weights"):
        ep.ep_combine_residual(rows, slot, w.double(), x)
    with pytest.raises(ValueError, match="residual"):
        ep.ep_combine_residual(rows, slot, w, x, residual=rows)
    with pytest.raises(ValueError, match="d_out"):
        ep.ep_combine_backward(x, slot, w)
    with pytest.raises(ValueError, match="out must be"):
        ep.ep_combine_backward(x, slot, w, rows, out=torch.zeros(9, 16, dtype=BF), d_weights=w)
    state = torch.zeros(2, dtype=torch.int64)
    for bad, kind in ((state.int(), TypeError), (torch.zeros(3, dtype=torch.int64), ValueError)):
        with pytest.raises(kind, match="state"):
            ep.ep_dropout(x, ep.Dropout(0.1, bad), y=x)
    for site in (-1, 1 << 32):
        with pytest.raises(ValueError, match="site"):
            ep.Dropout(0.1, state, site)
    with pytest.raises(ValueError, match="limit"):
        ep.ep_dropout(x, ep.Dropout(0.1, state), limit=torch.zeros(2, dtype=torch.int32))
    off = torch.zeros(3, dtype=torch.int32)
    ad = ep.Adapters(torch.zeros(2, 8, 16, dtype=BF), torch.zeros(2, 24, 8, dtype=BF), torch.ones(2))
    y = torch.zeros(4, 24, dtype=BF)
    with pytest.raises(ValueError, match="x must be"):
        ep.ep_adapter_matmul(torch.zeros(4, 24, dtype=BF), off, ad, y)
    with pytest.raises(ValueError, match="adapter_offsets"):
        ep.ep_adapter_matmul(x, off[:2], ad, y)
    with pytest.raises(TypeError, match="row_index"):
        ep.ep_adapter_matmul(x, off, ad, y, row_index=torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="up must be"):
        ep.ep_adapter_matmul(x, off, ep.Adapters(ad.down, torch.zeros(2, 24, 16, dtype=BF)), y)
    with pytest.raises(TypeError, match="scale"):
        ep.ep_adapter_matmul(x, off, ep.Adapters(ad.down, ad.up, torch.ones(2, dtype=BF)), y)
    with pytest.raises(ValueError, match="mid"):
        ep.ep_adapter_matmul(x, off, ad, y, mid=torch.zeros(4, 16, dtype=BF))
    with pytest.raises(ValueError, match="dy"):
        ep.ep_adapter_matmul_backward(x, x, off, ad, None, ep.alloc_adapter_grads(x, ad))
    with pytest.raises(ValueError, match="2\\^31"):
        ep.ep_adapter_matmul_backward_workspace_bytes(8, 8, 1 << 31, 64, 8, 2)


def test_binding_refuses_host_tensors():
    x, slot, w = torch.zeros(4, 16, dtype=BF), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    rows, state = torch.zeros(8, 16, dtype=BF), torch.zeros(2, dtype=torch.int64)
    ad = ep.Adapters(torch.zeros(2, 8, 16, dtype=BF), torch.zeros(2, 24, 8, dtype=BF))
    off = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: ep.ep_sort(x, slot, rows), lambda: ep.ep_sort_backward(rows, slot, x), lambda: ep.ep_combine_residual(rows, slot, w, x),
                 lambda: ep.ep_combine_backward(x, slot, w, rows), lambda: ep.ep_dropout(x, ep.Dropout(0.1, state)),
                 lambda: ep.ep_adapter_matmul(x, off, ad, torch.zeros(4, 24, dtype=BF)),
                 lambda: ep.ep_adapter_matmul_backward(torch.zeros(4, 24, dtype=BF), x, off, ad, None, ep.alloc_adapter_grads(x, ad, down=False, up=False))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_a_dropout_can_be_copied_and_pickled():
    d = ep.Dropout(0.25, torch.tensor([1, 2]), 7)
    d._struct()
    for other in (copy.copy(d), copy.deepcopy(d), pickle.loads(pickle.dumps(d))):
        assert other.p == d.p and other.site == 7 and torch.equal(other.state, d.state)
        s = other._struct().contents
        assert s.state == other.state.data_ptr() and s.p == 0.25 and s.site == 7


@pytest.mark.gpu
def test_binding_refuses_a_mix_of_devices():
    x, slot, w = torch.zeros(4, 16, dtype=BF, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    rows = torch.zeros(8, 16, dtype=BF, device="cuda")
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_sort(x, slot.cpu(), rows)
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_dropout(x, ep.Dropout(0.1, torch.zeros(2, dtype=torch.int64)))
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_combine_residual(rows, slot, w, x, dropout=ep.Dropout(0.1, torch.zeros(2, dtype=torch.int64)))
    ad = ep.Adapters(torch.zeros(2, 8, 16, dtype=BF), torch.zeros(2, 24, 8, dtype=BF))
    with pytest.raises(ValueError, match="one CUDA device"):
        ep.ep_adapter_matmul(x, torch.zeros(3, dtype=torch.int32, device="cuda"), ad, torch.zeros(4, 24, dtype=BF, device="cuda"))
