"""ep_adapter_matmul and its gradients in calls without rows or without entries, whose offsets may still name some: what the header says of
an entry whose row does not exist, and of an offset past the entries."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2609_40093_b200 import ep

BF, p, odd = torch.bfloat16, ctypes.c_void_p(256), ctypes.c_void_p(264)     # never dereferenced on the host
H, N, r, A = 64, 72, 24, 3


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_host_checks():
    L = ep.lib()

    def forward(rows, entries, off=p, mid=p, status=None):
        return L.ep_adapter_matmul(ctypes.byref(ep._Adapter(rows, entries, H, N, r, A)), None, off, p, None, None, None, None, None, mid, status, None)

    def backward(rows, entries, off=p, status=None):
        return L.ep_adapter_matmul_backward(ctypes.byref(ep._Adapter(rows, entries, H, N, r, A)), None, None, off, p, None, None, None, None, None, None,
                                            None, None, status, None, 0, None)

    assert forward(0, 0) == 0 and forward(4, 0) == 0 and forward(4, 0, off=None, mid=odd) == 0      # nothing to write, nobody to tell
    assert forward(0, 5, off=None) == -1 and forward(0, 5, mid=odd) == -2
    assert backward(0, 0) == 0 and backward(0, 0, off=None, status=p) == 0     # a dx of no rows has no address
    assert backward(0, 5, off=None) == -1 and backward(4, 0) == -1


def _weights():
    return ep.Adapters(torch.ones(A, r, H, dtype=BF, device="cuda"), torch.ones(A, N, r, dtype=BF, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("offsets,named,bits", [([0, 0, 0, 0], 0, 0), ([0, 2, 2, 4], 4, ep.STATUS_BAD_INDEX),
                                                ([0, 3, 9, 9], 5, ep.STATUS_BAD_INDEX | ep.STATUS_CAPACITY)])
def test_entries_without_rows(offsets, named, bits):
    off, index = torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    x, y, ad = torch.empty(0, H, dtype=BF, device="cuda"), torch.empty(0, N, dtype=BF, device="cuda"), _weights()
    status, whole = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((7, r), 5.0, dtype=BF, device="cuda")
    mid = whole[1:6]
    ep.ep_adapter_matmul(x, off, ad, y, base=y, row_index=index, mid=mid, status=status)
    assert int(status) == bits and (mid[:named] == 0).all() and (mid[named:] == 5).all() and (whole[[0, 6]] == 5).all()
    status.zero_()
    ep.ep_adapter_matmul(x, off, ad, y, row_index=index, status=status)
    assert int(status) == bits
    for down in (True, False):                                                 # with the weights' gradients, and dx alone
        status.zero_()
        grads = ep.alloc_adapter_grads(x, ad, entries=5, down=down, up=down)
        if down:
            grads.ddown.fill_(3.0), grads.dup.fill_(3.0)
        ep.ep_adapter_matmul_backward(y, x, off, ad, mid, grads, base=grads.dx, row_index=index, status=status)
        assert int(status) == bits
        assert not down or ((grads.ddown == 0).all() and (grads.dup == 0).all())


@pytest.mark.gpu
def test_many_entries_without_rows():
    n = 200003                                                                 # more vectors than the launch has threads
    off = torch.tensor([0, 7, n - 9, n - 2], dtype=torch.int32, device="cuda")
    mid, status = torch.full((n, 128), 5.0, dtype=BF, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ad = ep.Adapters(torch.ones(A, 128, H, dtype=BF, device="cuda"), torch.ones(A, N, 128, dtype=BF, device="cuda"))
    ep.ep_adapter_matmul(torch.empty(0, H, dtype=BF, device="cuda"), off, ad, row_index=torch.zeros(n, dtype=torch.int32, device="cuda"), mid=mid, status=status)
    assert int(status) == ep.STATUS_BAD_INDEX and (mid[:n - 2] == 0).all() and (mid[n - 2:] == 5).all()


@pytest.mark.gpu
def test_offsets_past_no_entries():
    off, empty = torch.tensor([0, 1, 1, 2], dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    x, y, ad = torch.ones(4, H, dtype=BF, device="cuda"), torch.full((4, N), 5.0, dtype=BF, device="cuda"), _weights()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ep.ep_adapter_matmul(x, off, ad, y, row_index=empty, status=status)
    assert int(status) == ep.STATUS_CAPACITY and (y == 5).all()
    status.zero_()
    ep.ep_adapter_matmul_backward(y, x, off, ad, torch.empty(0, r, dtype=BF, device="cuda"), ep.alloc_adapter_grads(x, ad, entries=0), row_index=empty, status=status)
    assert int(status) == ep.STATUS_CAPACITY
