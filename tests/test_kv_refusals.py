"""The 4-bit cache's entry points without a GPU: sizes, and every bad argument turned into its status on the host (nothing below reaches a launch)."""
import ctypes

import pytest
import torch

import paper_2407_11062_amd as eq

OK, NULL, SHAPE, BITS, GROUP, DTYPE, ALIGN, WORKSPACE, DEVICE, HYPER = range(10)
P = 0x10000              # a fake 256-byte aligned "device pointer", never dereferenced on these paths


def desc(pages=10, heads=8, head_dim=128, group=64, page_tokens=64, act=eq.BF16):
    return eq.KvDesc(pages, heads, head_dim, group, page_tokens, act)


def batch(table=P, lens=P, starts=P, tokens=4, sequences=2, table_stride=5, max_new=3, max_len=320):
    return eq.KvBatchDesc(table, lens, starts, tokens, sequences, table_stride, max_new, max_len)


def strides(token=1024, head=128):
    return (ctypes.c_int64 * 2)(token, head)


def write(d=None, b=None, K=P, ks=None, V=P, vs=None, pool=P):
    r = lambda x: None if x is None else ctypes.byref(x)
    return eq.lib().eqat_kv_write(r(d), r(b), K, ks, V, vs, pool, None)


def attend(d=None, b=None, q_heads=16, causal=1, window=0, scale=0.0, Q=P, qs=None, out=P, os_=None, lse=None, pool=P, ws=P, ws_bytes=1 << 40, a=True):
    r = lambda x: None if x is None else ctypes.byref(x)
    at = eq.KvAttn(q_heads, causal, window, scale)
    return eq.lib().eqat_kv_attention(r(d), r(b), ctypes.byref(at) if a else None, Q, qs, out, os_, lse, pool, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(act=2), DTYPE), (dict(act=-1), DTYPE), (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=512), SHAPE),
    (dict(group=16), GROUP), (dict(group=256), GROUP), (dict(group=96), GROUP), (dict(group=0), GROUP), (dict(group=-2), GROUP), (dict(head_dim=64, group=128), GROUP),
    (dict(heads=0), SHAPE), (dict(heads=-1), SHAPE), (dict(heads=1 << 17), SHAPE), (dict(page_tokens=0), SHAPE), (dict(page_tokens=48), SHAPE),
    (dict(page_tokens=-32), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 31), SHAPE), (dict(pages=(1 << 31) - 1, page_tokens=1 << 20), SHAPE),
])
def test_descriptors(kw, code):
    d = desc(**kw)
    assert eq.lib().eqat_kv_pool_bytes(ctypes.byref(d)) == 0
    assert write(d, batch(), ks=strides(), vs=strides()) == code
    assert attend(d, batch(), qs=strides(), os_=strides()) == code
    assert eq.lib().eqat_kv_read(ctypes.byref(d), ctypes.byref(batch()), P, strides(), None, None, P, None) == code
    assert eq.lib().eqat_kv_workspace_bytes(ctypes.byref(d), ctypes.byref(batch()), 16) == 0


def test_sizes():
    L = eq.lib()
    for D, g, held in [(64, 32, 80), (64, 64, 72), (128, 32, 160), (128, 64, 144), (128, 128, 136), (128, -1, 136), (256, -1, 264), (256, 32, 320)]:
        d = desc(head_dim=D, group=g, pages=7, heads=3, page_tokens=96)
        assert L.eqat_kv_pool_bytes(ctypes.byref(d)) == 7 * 3 * 96 * held
    big = desc(pages=1 << 20, heads=8, head_dim=128, group=128, page_tokens=256)
    assert L.eqat_kv_pool_bytes(ctypes.byref(big)) == (1 << 28) * 8 * 136            # beyond 32 bits
    assert L.eqat_kv_pool_bytes(None) == 0
    # the workspace follows the cache's heads, not the sequences, and stays modest
    for heads in (1, 8, 32, 40):
        d = desc(heads=heads)
        a, b = (L.eqat_kv_workspace_bytes(ctypes.byref(d), ctypes.byref(batch(sequences=n, tokens=n, max_new=1, max_len=1 << 17)), heads * 4) for n in (1, 500))
        assert 0 < a <= b < 64 << 20
    assert L.eqat_kv_workspace_bytes(ctypes.byref(desc()), ctypes.byref(batch()), 12) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), SHAPE), (dict(sequences=-1), SHAPE), (dict(table_stride=-1), SHAPE), (dict(max_new=-1), SHAPE), (dict(max_len=-1), SHAPE),
    (dict(max_len=2 ** 31 - 1), SHAPE), (dict(tokens=1 << 29), SHAPE), (dict(sequences=0), SHAPE), (dict(lens=None), NULL), (dict(starts=None), NULL), (dict(table=None), NULL),
    (dict(table=P + 2), ALIGN), (dict(lens=P + 1), ALIGN), (dict(starts=P + 3), ALIGN),
])
def test_batches(kw, code):
    assert write(desc(), batch(**kw), ks=strides(), vs=strides()) == code
    assert attend(desc(), batch(**kw), qs=strides(), os_=strides()) == code


def test_tensors_and_workspace():
    d, b, s = desc(), batch(), strides()
    assert write(None, b, ks=s, vs=s) == NULL and write(d, None, ks=s, vs=s) == NULL
    assert write(d, b, K=None, ks=s, vs=s) == NULL and write(d, b, ks=s, V=None, vs=s) == NULL and write(d, b, ks=None, vs=s) == NULL and write(d, b, ks=s, vs=s, pool=None) == NULL
    assert write(d, b, K=P + 8, ks=s, vs=s) == ALIGN and write(d, b, ks=strides(1028), vs=s) == ALIGN and write(d, b, ks=s, vs=strides(1024, 132)) == ALIGN
    assert write(d, b, ks=s, vs=s, pool=P + 128) == ALIGN
    f32 = desc(act=eq.F32)
    assert write(f32, b, ks=strides(1026), vs=s) == ALIGN and write(f32, b, ks=strides(1028), vs=s, pool=None) == NULL          # four floats are 16 bytes
    assert attend(d, b, qs=s, os_=s, a=False) == NULL and attend(d, b, Q=None, qs=s, os_=s) == NULL and attend(d, b, qs=s, out=None, os_=s) == NULL
    assert attend(d, b, qs=s, os_=s, out=P + 8) == ALIGN and attend(d, b, qs=s, os_=strides(1024, 4)) == ALIGN and attend(d, b, qs=s, os_=s, lse=P + 2) == ALIGN
    need = eq.lib().eqat_kv_workspace_bytes(ctypes.byref(d), ctypes.byref(b), 16)
    assert attend(d, b, qs=s, os_=s, ws=None) == WORKSPACE and attend(d, b, qs=s, os_=s, ws_bytes=need - 1) == WORKSPACE and attend(d, b, qs=s, os_=s, ws=P + 16) == ALIGN
    for q_heads in (0, 4, 12, -8, 1 << 21):
        assert attend(d, b, q_heads=q_heads, qs=s, os_=s) == SHAPE
    for kw in (dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1)):
        assert attend(d, b, qs=s, os_=s, **kw) == HYPER
    assert attend(d, batch(tokens=1 << 27, max_new=1 << 27), q_heads=1024, qs=s, os_=s) == SHAPE


def test_nothing_new_is_nothing_to_do():
    """no rows: no pointer is looked at and nothing is launched"""
    none = batch(tokens=0, sequences=0, table=None, lens=None, starts=None)
    assert write(desc(), none, K=None, V=None, pool=None) == OK
    assert attend(desc(), none, Q=None, out=None, pool=None, ws=None, ws_bytes=0) == OK
    assert eq.lib().eqat_kv_read(ctypes.byref(desc()), ctypes.byref(batch()), None, None, None, None, None, None) == OK


def test_the_binding_refuses_other_tensors():
    with pytest.raises(ValueError):
        eq.KvCache(8, 96, 32, 64, 10, device="cpu")
    with pytest.raises(TypeError):
        eq.KvCache(8, 128, 32, 64, 10, dtype=torch.float16, device="cpu")
    cache = eq.KvCache(2, 128, 64, 64, 3, device="cpu")
    assert cache.pool.numel() == 3 * 64 * 2 * 144
    with pytest.raises(ValueError):
        eq.KvCache(2, 128, 64, 64, 3, pool=cache.pool[1:])
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(TypeError):
        eq.KvBatch(i32(2, 3).long(), i32(2), i32(3), 4, 2, 100)
    with pytest.raises(ValueError):
        eq.KvBatch(i32(2, 3), i32(2), i32(2), 4, 2, 100)
    with pytest.raises(ValueError):
        eq.KvBatch(i32(2, 3), i32(2), i32(3), 4, 2, 100)               # not on the device


def test_what_is_numbered_in_32_bits():
    """records, rows and workgroups: the first count that does not fit is refused, in the products too"""
    assert eq.lib().eqat_kv_pool_bytes(ctypes.byref(desc(pages=(1 << 24) - 1, heads=64))) > 0                       # 2^31 - 128 records
    assert eq.lib().eqat_kv_pool_bytes(ctypes.byref(desc(pages=1 << 24, heads=64))) == 0                            # 2^31
    wide = desc(heads=1 << 16, head_dim=64, group=64)
    assert write(wide, batch(tokens=1 << 13), ks=strides(), vs=strides()) == SHAPE and write(wide, batch(tokens=(1 << 13) - 1), ks=strides(), vs=strides(), pool=None) == NULL
    assert write(desc(), batch(tokens=1 << 62), ks=strides(), vs=strides()) == SHAPE                                # times the heads: not an overflow
    one = desc(heads=1)
    assert attend(one, batch(sequences=1, max_new=1 << 20), q_heads=1 << 10, qs=strides(), os_=strides()) == SHAPE
    assert attend(one, batch(sequences=1, max_new=(1 << 20) - 1), q_heads=1 << 10, qs=strides(), os_=strides(), pool=None) == NULL
    assert attend(one, batch(sequences=1 << 24, max_new=1, max_len=4096), q_heads=1, qs=strides(), os_=strides()) == SHAPE          # 2^26 units of up to 128 records


@pytest.mark.parametrize("pool", [torch.empty(1 << 10, dtype=torch.uint8), torch.empty(1 << 20, dtype=torch.int8), torch.empty(1 << 21, dtype=torch.uint8)[::2]])
def test_pools_that_are_none(pool):
    with pytest.raises(ValueError):
        eq.KvCache(2, 128, 64, 64, 3, device="cpu", pool=pool)
