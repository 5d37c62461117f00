"""More of what the 4-bit cache's entry points turn into a status or an error on the host (nothing below reaches a launch)."""
import ctypes
import types

import pytest
import torch

import paper_2407_11062_amd as eq
from test_kv_refusals import HYPER, NULL, P, attend, batch, desc, strides


@pytest.mark.parametrize("scale,code", [(2.0 ** 100, NULL), (1.3e30, HYPER), (3.0e38, HYPER), (1e-45, NULL)])
def test_scales(scale, code):
    """up to 2^100 (the call without a pool goes on to its next refusal)"""
    assert attend(desc(), batch(), qs=strides(), os_=strides(), scale=scale, pool=None) == code


class OnTheDevice:
    """what the binding asks of a tensor, without a device"""

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, "cuda", True

    def stride(self):
        return (self.shape[1] * self.shape[2], self.shape[2], 1)

    def data_ptr(self):
        return P

    def is_contiguous(self):
        return True

    def numel(self):
        return 1 << 40


def test_pools_in_host_memory():
    """a cache may be made of host memory, to look at its size; no call takes it to the device (a batch without tokens: not even a launch that does nothing)"""
    cache = eq.KvCache(2, 128, 64, 64, 3, device="cpu")
    none = types.SimpleNamespace(ref=ctypes.byref(eq.KvBatchDesc(P, P, P, 0, 1, 1, 0, 0)), tokens=0)
    rows, q = OnTheDevice(0, 2, 128), OnTheDevice(0, 4, 128)
    for call in (lambda: eq.eqat_kv_write(cache, none, rows, rows), lambda: eq.eqat_kv_read(cache, none, k=rows, v=rows),
                 lambda: eq.eqat_kv_attention(cache, none, q, out=q, ws=OnTheDevice(1, 1, 1))):
        with pytest.raises(ValueError, match="device"):
            call()


def test_numbers_beyond_32_bits():
    """none of them is cut to its low half"""
    big = 2 ** 32
    for numbers in ((big + 2, 128, 64, 64, 3), (2, big + 128, 64, 64, 3), (2, 128, big + 64, 64, 3), (2, 128, 64, big + 64, 3), (2, 128, 64, 64, big + 3)):
        with pytest.raises(ValueError, match="32 bits"):
            eq.KvCache(*numbers, device="cpu")
    class Counts(OnTheDevice):
        def numel(self):
            return self.shape[0]

        def dim(self):
            return len(self.shape)
    lens, starts, table = Counts(2, dtype=torch.int32), Counts(3, dtype=torch.int32), Counts(2, 5, dtype=torch.int32)
    assert eq.KvBatch(table, lens, starts, 4, 2, 100).desc.max_len == 100
    for numbers in ((4, big + 2, 100), (4, 2, big + 100)):
        with pytest.raises(ValueError, match="32 bits"):
            eq.KvBatch(table, lens, starts, *numbers)
    cache = eq.KvCache(2, 128, 64, 64, 3, device="cpu")
    none = types.SimpleNamespace(ref=ctypes.byref(eq.KvBatchDesc(P, P, P, 0, 1, 1, 0, 0)), tokens=0)
    q = OnTheDevice(0, 4, 128)
    with pytest.raises(ValueError, match="32 bits"):
        eq.eqat_kv_attention(cache, none, q, out=q, ws=OnTheDevice(1, 1, 1), window=big + 16)
    with pytest.raises(ValueError, match="32 bits"):
        eq.kv_workspace(cache, none, big + 4)
