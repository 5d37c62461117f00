"""Refusals of the binding that no tensor of one device reaches (workspaces and batches on another device than a call's tensors), and what it hands over by address.  No GPU: nothing is launched."""
import ctypes

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


def test_strides_live_until_the_call_returns(monkeypatch):
    """what a call hands over by address does not go with the entries of a cache that other threads' calls push out"""
    seen = []

    class Calls:
        def look(self, *addresses):
            eq._both_rows.cache_clear()
            eq._kv_strides.cache_clear()
            others = [(ctypes.c_int64 * 2)(7, 7) for _ in range(1000)]
            seen.append([list((ctypes.c_int64 * 2).from_address(a)) for a in addresses])
            return 0 * len(others)

        def eqat_rotary(self, ref, tokens, pos, q, qs, qh, qo, qos, k, ks, kh, ko, kos, inverse, stream): return self.look(qs, qos, ks, kos)
        def eqat_kv_rotary_write(self, c, b, r, q, qs, qh, qo, qos, k, ks, v, vs, pool, stream): return self.look(qs, qos, ks, vs)

    cache = eq.KvCache(1, 64, 64, 32, 1, dtype=torch.float32, device="cpu")
    rot, batch = eq.Rotary.__new__(eq.Rotary), eq.KvBatch.__new__(eq.KvBatch)
    rot.device, rot.head_dim, rot.refs = -1, 64, {torch.float32: 0}
    batch.device, batch.tokens, batch.ref = -1, 4, None
    monkeypatch.setattr(eq, "lib", Calls)
    monkeypatch.setattr(eq, "_stream_at", lambda device: 0)
    q, k, out = torch.zeros(4, 5, 64), torch.zeros(4, 1, 96)[..., :64], torch.zeros(4, 5, 72)[..., :64]
    eq.eqat_rotary(rot, torch.zeros(4, dtype=torch.int32), q, k, q_out=out, k_out=torch.zeros(4, 1, 128)[..., :64])
    eq.eqat_kv_rotary_write(cache, batch, rot, q, k, k, q_out=out)
    assert seen == [[[320, 64], [360, 72], [96, 96], [128, 128]], [[320, 64], [360, 72], [96, 96], [96, 96]]]
