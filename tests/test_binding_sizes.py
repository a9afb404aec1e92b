"""Sizes that a C argument of 32 bits does not hold are refused by the binding: ctypes would pass their low bits."""
import pytest
import torch

import paper_2506_17506_amd as vl
from paper_2506_17506_amd import binding
from stand_in import in_own_process
from test_host_paths import analysed, jobs_of


class Tensor:
    """what the binding asks of a float32 or int32 tensor of n elements on device 0; there is no memory behind it"""
    is_cuda = True

    def __init__(self, n, dtype=None):
        self.n, self.dtype, self.shape = n, dtype or torch.float32, (n,)

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


@in_own_process
def test_candidates_that_32_bits_do_not_count(s):
    """more than 2^32 candidates, and fewer than none"""
    (hm,), (hl,) = analysed(s, 1)
    jobs, keep = jobs_of(s, [hm], [hl], 8)
    _, _, cand, _, ld, out = jobs[0]
    for K in (2 ** 32 + 8, 2 ** 33 + 8, -1, -2 ** 32 + 8):
        s.launches.clear()
        for call in (lambda: s.vl.vl_verify_batch(hm, hl, cand, K, ld, out, stream=1), lambda: s.vl.vl_verify_batch_static(hm, hl, cand, K, ld, out, stream=1),
                     lambda: s.vl.vl_verify_multi([(hm, hl, cand, K, ld, out)], stream=1), lambda: s.vl.vl_verify_multi_occ_major([(hm, hl, cand, K, ld, out)], stream=1),
                     lambda: s.vl.vl_count_violations_multi([(hm, hl, cand, K, ld, out)], stream=1), lambda: s.vl.vl_bank_conflicts(hm, cand, K, ld, 4, out, stream=1),
                     lambda: s.vl.vl_lanes_expand(hm, cand, K, ld, out, ld, stream=1), lambda: s.vl.vl_summarize_multi([(hm, hl, cand, K, ld, out)], out, stream=1)):
            try:
                call()
            except s.vl.VlError as e:
                assert e.code == -2, e
            else:
                raise AssertionError(f"{K} candidates taken")
        assert not s.launches
    for n_banks in (2 ** 32 + 4, -1):
        try:
            s.vl.vl_bank_conflicts(hm, cand, 8, ld, n_banks, out, stream=1)
        except s.vl.VlError as e:
            assert e.code == -3, e
        else:
            raise AssertionError(f"{n_banks} banks taken")
    assert not s.launches
