"""Sizes that a C argument of 32 bits does not hold are refused by the binding: ctypes would pass their low bits."""
import pytest
import torch

import paper_2506_17506_amd as vl
from paper_2506_17506_amd import binding


class Tensor:
    """what the binding asks of a float32 or int32 tensor of n elements on device 0; there is no memory behind it"""
    is_cuda = True

    def __init__(self, n, dtype=torch.float32):
        self.n, self.dtype, self.shape = n, dtype, (n,)

    def get_device(self):
        return 0

    def numel(self):
        return self.n

    def element_size(self):
        return 4

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("n,n_offsets", [(2 ** 31, 2), (2 ** 32 + 5, 2), (2 ** 33 + 1, 2), (8, 2 ** 31 + 1), (8, 2 ** 32 + 3)])
def test_more_samples_or_groups_than_the_header_allows(monkeypatch, n, n_offsets):
    called = []

    class Library:
        @staticmethod
        def vl_group_advantages(*args):
            called.append(args)
            return 0
        vl_strerror, vl_last_hip_error = vl.load().vl_strerror, vl.load().vl_last_hip_error
    torch_side = binding._Torch()
    torch_side.device, torch_side.stream = (lambda: 0), (lambda device: 0)
    monkeypatch.setattr(binding, "_t", torch_side)
    monkeypatch.setattr(binding, "_lib", Library)
    with pytest.raises(vl.VlError) as err:
        vl.vl_group_advantages(None, Tensor(n_offsets, torch.int32), (1, 0, 0, 0), 1e-6, Tensor(n), extra=Tensor(n))
    assert err.value.code == -2 and not called
    vl.vl_group_advantages(None, Tensor(3, torch.int32), (1, 0, 0, 0), 1e-6, Tensor(2 ** 31 - 1), extra=Tensor(2 ** 31 - 1))
    (args,) = called
    assert args[2] == 2 ** 31 - 1 and args[4] == 2
