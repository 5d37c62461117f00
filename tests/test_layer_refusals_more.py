"""Refusals of the binding that no tensor of one device reaches: workspaces and batches on another device than a call's tensors.  No GPU: nothing is launched."""
import pytest
import torch

import paper_2407_11062_amd as eq


class Elsewhere:
    """What the binding looks at of a device tensor, on device 1."""

    def __init__(self, shape, dtype, device=1):
        self.shape, self.dtype, self.index, self.is_cuda, self.device = torch.Size(shape), dtype, device, True, f"cuda:{device}"

    def dim(self): return len(self.shape)
    def numel(self): return self.shape.numel()
    def get_device(self): return self.index
    def is_contiguous(self): return True
    def data_ptr(self): return 1 << 20


WS = Elsewhere((1 << 30,), torch.uint8)


def test_workspaces_on_another_device():
    x, w = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="ws: .* on cuda:1"):
        eq.eqat_norm_bwd(x, w, 1e-5, x, ws=WS)
    W, s, z = torch.zeros(32, 16, dtype=torch.uint8), torch.zeros(32, 2), torch.zeros(32, 4, dtype=torch.uint8)
    ready, dH = torch.zeros(eq._prepared_bytes(16, 64, 2, 32, eq.F32), dtype=torch.uint8), torch.zeros(4, 16)
    for call in (lambda: eq.eqat_gated_fwd(x, W, s, z, 2, 32, ws=WS), lambda: eq.eqat_gated_bwd(x, W, s, z, dH, 2, 32, ws=WS),
                 lambda: eq.eqat_gated_fwd_prepared(x, ready, s, 16, 2, 32, ws=WS), lambda: eq.eqat_gated_bwd_prepared(x, ready, s, dH, 2, 32, ws=WS)):
        with pytest.raises(ValueError, match="ws: .* on cuda:1"):
            call()
    with pytest.raises(ValueError, match="ws: .* contiguous"):
        eq.eqat_norm_bwd(x, w, 1e-5, x, ws=torch.zeros(1 << 20, 2, dtype=torch.uint8)[:, 0])


def test_batches_on_another_device():
    def batch(*devices):
        table, lens, starts = (Elsewhere(shape, torch.int32, d) for shape, d in zip(((1, 1), (1,), (2,)), devices))
        return eq.KvBatch(table, lens, starts, tokens=4, max_new=4, max_len=4)

    cache = eq.KvCache(1, 64, 64, 32, 1, dtype=torch.float32, device="cpu")
    rot, q = eq.Rotary.__new__(eq.Rotary), torch.zeros(4, 1, 64)
    rot.device, rot.head_dim = -1, 64
    for devices in ((0, 0, 1), (0, 1, 0), (1, 0, 0)):
        with pytest.raises(ValueError, match="on devices"):
            eq.eqat_kv_rotary_write(cache, batch(*devices), rot, q, q, q)
    with pytest.raises(ValueError, match="table, lens and starts on device 1"):
        eq.eqat_kv_rotary_write(cache, batch(1, 1, 1), rot, q, q, q)
