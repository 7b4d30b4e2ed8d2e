"""A caller's workspace: what the binding tells the library of it.  Nothing is launched; the tensors are stand-ins with an
address, a size and a place."""
import pytest
import torch

from paper_2302_12510_b200 import binding


class Tensor:
    def __init__(self, address, n, itemsize=1, is_cuda=True, device="cuda:0", contiguous=True):
        self.address, self.n, self.itemsize, self.is_cuda, self.device, self.contiguous = address, n, itemsize, is_cuda, device, contiguous

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.n

    def element_size(self):
        return self.itemsize

    def is_contiguous(self):
        return self.contiguous


LIKE = Tensor(0, 0)


@pytest.mark.parametrize("address,n,want", [(4096, 5000, (4096, 5000)), (4096 + 512, 5000, (5120, 4488)), (4096 + 512, 512, (5120, 0)),
                                            (4096 + 512, 8, (5120, 0)), (4096 + 16, 1000, (5120, 0)), (4096, 0, (4096, 0))])
def test_what_lies_behind_the_boundary(address, n, want):
    # a workspace that ends before its first 1024-byte boundary has no bytes, not a negative number of them
    ws = Tensor(address, n)
    assert binding._ws_span(ws, LIKE) == want
    at, size, kept = binding._workspace(100, ws, LIKE)
    assert (at, size) == want and kept is ws


def test_bytes_are_counted_whatever_the_type():
    assert binding._ws_span(Tensor(4096 + 512, 1024, itemsize=4), LIKE) == (5120, 4096 - 512)


@pytest.mark.parametrize("bad", [dict(is_cuda=False, device="cpu"), dict(device="cuda:1"), dict(contiguous=False)])
def test_a_workspace_elsewhere_is_refused(bad):
    ws = Tensor(4096, 1 << 20, **bad)
    with pytest.raises(ValueError):
        binding._ws_span(ws, LIKE)
    with pytest.raises(ValueError):
        binding._workspace(100, ws, LIKE)


def test_every_call_refuses_a_workspace_in_host_memory():
    # decided before the library is called, so stand-ins on the host do for the operands
    ws, u8 = torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros((64, 128), dtype=torch.uint8)
    s, c = torch.ones(2), torch.zeros((64, 64))
    desc = binding.ConvDesc(1, 4, 4, 64, 64, 1, 1)
    calls = [lambda: binding.dybit_gemm(64, 64, 128, u8, (8, 1), s, u8, (8, 1), s, C_out=c, ws=ws),
             lambda: binding.dybit_gemm_requant(64, 64, 128, u8, (8, 1), s, u8, (8, 1), s, (8, 1), s, Q=u8, ws=ws),
             lambda: binding.dybit_gemm_batched(64, 64, 128, u8[None], (8, 1), s, u8[None], (8, 1), s, C=c[None], ws=ws),
             lambda: binding.dybit_conv2d(desc, u8, (8, 1), s, u8, (8, 1), s, Y=c, ws=ws),
             lambda: binding.dybit_conv2d_requant(desc, u8, (8, 1), s, u8, (8, 1), s, (8, 1), s, Q=u8, ws=ws)]
    for call in calls:
        with pytest.raises(ValueError, match="ws"):
            call()
