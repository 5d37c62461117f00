"""Refusals of the norm, rotary and gated entry points: every status, without a GPU (nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2407_11062_amd as eq

OK, NULL, SHAPE, BITS, GROUP, DTYPE, ALIGN, WORKSPACE, DEVICE, HYPER = range(10)
P = 1 << 20                              # stands for a device pointer, 256-byte aligned; nothing is launched


def L():
    return eq.lib()


def norm(**kw):
    return eq.NormDesc(**{**dict(tokens=4, width=256, group=-1, act_dtype=eq.BF16, w_dtype=eq.F32, eps=1e-5), **kw})


def norm_fwd(d, X=P, R=None, w=None, S=None, Y=P, codes=None, scales=None):
    return L().eqat_norm_fwd(ctypes.byref(d), X, R, w, S, Y, codes, scales, None)


def norm_bwd(d, S=P, w=None, dY=P, dS=None, dX=P, dw=None, ws=None, n=0):
    return L().eqat_norm_bwd(ctypes.byref(d), S, w, dY, dS, dX, dw, ws, n, None)


@pytest.mark.parametrize("kw, status", [
    (dict(act_dtype=2), DTYPE), (dict(w_dtype=-1), DTYPE), (dict(tokens=-1), SHAPE), (dict(tokens=1 << 31), SHAPE), (dict(width=0), SHAPE), (dict(width=-8), SHAPE),
    (dict(width=12), SHAPE), (dict(width=32768 + 8), SHAPE), (dict(eps=-1.0), HYPER), (dict(eps=float("nan")), HYPER), (dict(eps=float("inf")), HYPER)])
def test_norm_descriptor(kw, status):
    assert norm_fwd(norm(**kw)) == status and norm_bwd(norm(**kw)) == status
    assert L().eqat_norm_workspace_bytes(ctypes.byref(norm(**kw))) == 0


def test_norm_pointers():
    assert L().eqat_norm_fwd(None, P, None, None, None, P, None, None, None) == NULL
    assert norm_fwd(norm(), X=None) == NULL
    assert norm_fwd(norm(), codes=P) == NULL and norm_fwd(norm(), scales=P) == NULL
    for name in ("X", "R", "w", "S", "Y"):
        assert norm_fwd(norm(), **{name: P + 8}) == ALIGN, name
    assert norm_fwd(norm(), codes=P + 4, scales=P) == ALIGN and norm_fwd(norm(), codes=P, scales=P + 4) == ALIGN
    assert norm_fwd(norm(), Y=None) == OK and norm_fwd(norm(tokens=0), X=None) == OK          # nothing to do
    for group in (0, 16, 48, 1024, -2):
        assert norm_fwd(norm(group=group), codes=P, scales=P) == GROUP, group
    assert norm_fwd(norm(width=264, group=32), codes=P, scales=P) == GROUP
    for name in ("S", "w", "dY", "dS", "dX"):
        assert norm_bwd(norm(), **{name: P + 8}) == ALIGN, name
    assert norm_bwd(norm(), S=None) == NULL and norm_bwd(norm(), dY=None) == NULL
    assert norm_bwd(norm(), dX=None) == OK and norm_bwd(norm(tokens=0), S=None, dY=None) == OK
    need = L().eqat_norm_workspace_bytes(ctypes.byref(norm()))
    assert need > 0
    assert norm_bwd(norm(), dw=P) == WORKSPACE and norm_bwd(norm(), dw=P, ws=P, n=need - 1) == WORKSPACE and norm_bwd(norm(), dw=P, ws=P + 16, n=need) == ALIGN


def rotary(**kw):
    return eq.RotaryDesc(**{**dict(frequencies=P, head_dim=128, part=128, interleaved=0, act_dtype=eq.BF16, amplitude=1.0), **kw})


def strides(*v):
    return ctypes.addressof(keep := (ctypes.c_int64 * 2)(*v)), keep


def turn(d, tokens=4, pos=P, Q=P, qs=(1024, 128), qh=8, qo=P, qos=(1024, 128), K=None, ks=None, kh=0, ko=None, kos=None):
    keep = [strides(*v) if v is not None else (None, None) for v in (qs, qos, ks, kos)]
    return L().eqat_rotary(ctypes.byref(d) if d is not None else None, tokens, pos, Q, keep[0][0], qh, qo, keep[1][0], K, keep[2][0], kh, ko, keep[3][0], 0, None)


@pytest.mark.parametrize("kw, status", [
    (dict(act_dtype=5), DTYPE), (dict(head_dim=4, part=2), SHAPE), (dict(head_dim=100, part=2), SHAPE), (dict(head_dim=1032, part=2), SHAPE), (dict(part=0), SHAPE), (dict(part=3), SHAPE),
    (dict(part=130), SHAPE), (dict(part=-2), SHAPE), (dict(amplitude=float("nan")), HYPER), (dict(amplitude=float("inf")), HYPER), (dict(frequencies=P + 2), ALIGN),
    (dict(frequencies=None), NULL)])
def test_rotary_descriptor(kw, status):
    assert turn(rotary(**kw)) == status
    assert kv_turn(rotary(**kw)) == status


def test_rotary_arguments():
    d = rotary()
    assert turn(None) == NULL and turn(d, tokens=-1) == SHAPE and turn(d, tokens=1 << 31) == SHAPE and turn(d, qh=0) == SHAPE and turn(d, qh=(1 << 20) + 1) == SHAPE
    assert turn(d, tokens=1 << 28, qh=8) == SHAPE
    assert turn(d, qo=None) == NULL and turn(d, Q=None) == NULL and turn(d, pos=None) == NULL and turn(d, qs=None) == NULL and turn(d, qos=None) == NULL
    assert turn(d, pos=P + 2) == ALIGN and turn(d, Q=P + 8) == ALIGN and turn(d, qo=P + 8) == ALIGN and turn(d, qs=(1028, 128)) == ALIGN and turn(d, qos=(1024, 132)) == ALIGN
    assert turn(d, K=P, ks=(1024, 128), kh=8) == NULL and turn(d, K=P, ks=(1024, 128), kh=0, ko=P, kos=(1024, 128)) == SHAPE
    assert turn(d, Q=None, qo=None, qs=None, qos=None) == OK and turn(d, tokens=0, pos=None) == OK                       # nothing to do


def kv_turn(r, d=None, b=None, **kw):
    d = eq.KvDesc(4, 8, 128, 64, 64, eq.BF16) if d is None else d
    b = eq.KvBatchDesc(P, P, P, 4, 4, 1, 1, 64) if b is None else b
    a = {**dict(Q=P, qs=(1024, 128), qh=8, qo=P, qos=(1024, 128), K=P, ks=(1024, 128), V=P, vs=(1024, 128), pool=P), **kw}
    keep = {n: strides(*a[n]) if a[n] is not None else (None, None) for n in ("qs", "qos", "ks", "vs")}
    return L().eqat_kv_rotary_write(ctypes.byref(d), ctypes.byref(b), ctypes.byref(r) if r is not None else None, a["Q"], keep["qs"][0], a["qh"], a["qo"], keep["qos"][0], a["K"], keep["ks"][0],
                                    a["V"], keep["vs"][0], a["pool"], None)


def test_rotary_write_arguments():
    r = rotary()
    assert kv_turn(None) == NULL and kv_turn(rotary(head_dim=64, part=64)) == SHAPE and kv_turn(rotary(act_dtype=eq.F32)) == DTYPE
    assert kv_turn(r, qh=0) == SHAPE and kv_turn(r, pool=None) == NULL and kv_turn(r, pool=P + 16) == ALIGN
    for name in ("Q", "qo", "K", "V", "qs", "qos", "ks", "vs"):
        assert kv_turn(r, **{name: None}) == NULL, name
    for name in ("Q", "qo", "K", "V"):
        assert kv_turn(r, **{name: P + 8}) == ALIGN, name
    assert kv_turn(r, d=eq.KvDesc(4, 8, 96, 32, 64, eq.BF16)) == SHAPE and kv_turn(r, b=eq.KvBatchDesc(P, None, P, 4, 4, 1, 1, 64)) == NULL
    assert kv_turn(r, b=eq.KvBatchDesc(P, P, P, 0, 4, 1, 1, 64), Q=None) == OK                                            # no rows


def gated(**kw):
    return eq.Desc(**{**dict(tokens=4, in_features=256, out_features=512, bits=2, group=64, act_dtype=eq.BF16, w_dtype=eq.F32), **kw})


def gated_calls(d, kind=0, X=P, layer=P, s=P, z=P, dH=P, dY=P, H=P, ws=P, n=1 << 40):
    r = ctypes.byref(d) if d is not None else None
    return [L().eqat_gated_fwd(r, kind, X, layer, s, z, H, ws, n, None), L().eqat_gated_bwd(r, kind, X, layer, s, z, dH, dY, H, ws, n, None),
            L().eqat_gated_fwd_prepared(r, kind, X, layer, s, H, ws, n, None), L().eqat_gated_bwd_prepared(r, kind, X, layer, s, dH, dY, H, ws, n, None)]


@pytest.mark.parametrize("kw, status", [
    (dict(tokens=-1), SHAPE), (dict(in_features=48), SHAPE), (dict(out_features=504), SHAPE), (dict(out_features=0), SHAPE), (dict(bits=5), BITS), (dict(group=48), GROUP), (dict(act_dtype=3), DTYPE),
    (dict(tokens=1 << 21, out_features=1024), SHAPE), (dict(in_features=1 << 22, group=-1, out_features=16), SHAPE)])
def test_gated_descriptor(kw, status):
    assert gated_calls(gated(**kw)) == [status] * 4
    assert L().eqat_gated_workspace_bytes(ctypes.byref(gated(**kw))) == 0


def test_gated_arguments():
    d = gated(tokens=100)
    assert gated_calls(None) == [NULL] * 4 and L().eqat_gated_workspace_bytes(None) == 0
    assert gated_calls(d, kind=2) == [HYPER] * 4 and gated_calls(d, kind=-1) == [HYPER] * 4
    for name in ("X", "layer", "s"):
        assert gated_calls(d, **{name: None}) == [NULL] * 4, name
        assert gated_calls(d, **{name: P + 8}) == [ALIGN] * 4, name
    assert gated_calls(d, layer=P + 16)[2:] == [ALIGN] * 2
    assert gated_calls(gated(tokens=0), z=None) == [NULL, NULL, OK, OK] and gated_calls(d, z=P + 8)[:2] == [ALIGN] * 2
    assert [gated_calls(d, H=None)[i] for i in (0, 2)] == [NULL] * 2 and [gated_calls(d, dH=None)[i] for i in (1, 3)] == [NULL] * 2
    assert [gated_calls(d, H=None, dY=None, dH=None)[i] for i in (1, 3)] == [OK] * 2                                      # nothing wanted
    for prepared in (0, 1):
        need = L().eqat_gated_workspace_bytes(ctypes.byref(d))
        assert gated_calls(d, ws=None)[2 * prepared] == WORKSPACE and gated_calls(d, n=need - 1)[2 * prepared] == WORKSPACE and gated_calls(d, ws=P + 16)[2 * prepared] == ALIGN
        assert L().eqat_gated_workspace_bytes(ctypes.byref(gated(tokens=1))) == 256                             # a few tokens need none
    assert gated_calls(gated(tokens=0), X=None, H=None, dH=None) == [OK] * 4


def test_gated_workspace_of_more_tokens_serves_fewer():
    for act in (eq.F32, eq.BF16):
        sizes = [L().eqat_gated_workspace_bytes(ctypes.byref(gated(tokens=t, act_dtype=act, in_features=1024, out_features=5504))) for t in (1, 2, 16, 17, 64, 65, 100, 333, 1000, 4096, 8192)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("back", (False, True))
def test_gate_arguments(back):
    def call(T=4, F=64, dtype=eq.BF16, kind=0, Y=P, dH=P, dY=P, H=P):
        return L().eqat_gate_bwd(T, F, dtype, kind, Y, dH, dY, H, None) if back else L().eqat_gate_fwd(T, F, dtype, kind, Y, H, None)
    assert call(T=-1) == SHAPE and call(F=0) == SHAPE and call(F=12) == SHAPE and call(F=1 << 31) == SHAPE and call(T=1 << 31) == SHAPE and call(dtype=2) == DTYPE
    assert call(T=(1 << 31) - 1, F=16) == SHAPE and call(T=1 << 28, F=64) == SHAPE
    assert call(kind=2) == HYPER and call(Y=None) == NULL and call(Y=P + 8) == ALIGN and call(H=P + 8) == ALIGN and call(T=0, Y=None) == OK
    if back:
        assert call(dH=None) == NULL and call(dH=P + 8) == ALIGN and call(dY=P + 8) == ALIGN and call(dY=None, H=None) == OK
    else:
        assert call(H=None) == NULL


def test_binding_refusals():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device"):
        eq.eqat_norm_fwd(x, None, 1e-5)
    with pytest.raises(ValueError, match="group"):
        eq.eqat_norm_fwd(x, None, 1e-5, want=("codes",))
    with pytest.raises(TypeError):
        eq.Rotary(torch.zeros(4, dtype=torch.float64), 64)
    with pytest.raises(TypeError):
        eq.eqat_norm_fwd(x.half(), None, 1e-5)
    with pytest.raises(ValueError, match="32 bits"):
        eq.eqat_norm_fwd(x, None, 1e-5, group=1 << 33, want=("codes",), out={"codes": x, "scales": x})


def test_binding_looks_at_the_layer():
    X, s, z = torch.zeros(4, 64), torch.zeros(32, 2), torch.zeros(32, 4, dtype=torch.uint8)
    for W, s_, z_ in ((torch.zeros(32, 16, dtype=torch.uint8), s, z[:16]), (torch.zeros(32, 24, dtype=torch.uint8), s, z), (torch.zeros(31, 16, dtype=torch.uint8), s[:31], z[:31]),
                      (torch.zeros(32, 16, dtype=torch.uint8), s[:, :1], z), (torch.zeros(32, 16, dtype=torch.int8), s, z)):
        with pytest.raises(ValueError, match="packed layer"):
            eq.eqat_gated_fwd(X, W, s_, z_, 2, 32)
    need = eq._prepared_bytes(16, 64, 2, 32, eq.F32)
    assert need > 0
    for n, s_ in ((need - 1, s), (need, s[:30])):
        with pytest.raises(ValueError, match="prepared layer"):
            eq.eqat_gated_fwd_prepared(X, torch.zeros(n, dtype=torch.uint8), s_, 16, 2, 32)


def test_rotary_frequencies():
    import paper_2407_11062_amd as eq
    for kw in ({"part": 7}, {"part": 8, "base": 0.0}, {"part": 8, "stretch": 0.5}, {"part": 8, "stretch": 2.0, "short": 64.0, "long": 64.0}, {"part": 8, "short": 0.0}):
        with pytest.raises(ValueError):
            eq.rotary_frequencies(**kw)
    f = eq.rotary_frequencies(128, base=10000.0).double()
    assert len(f) == 64 and all(abs(float(f[i]) * 10000.0 ** (i / 64) - 1.0) < 1e-7 for i in range(64))
    g = eq.rotary_frequencies(128, stretch=8.0).double()
    waves = 2 * 3.141592653589793 / f
    assert (g[waves < 256.0] == f[waves < 256.0]).all() and ((g * 8.0 - f)[waves > 2048.0].abs() <= 1e-7 * f[waves > 2048.0]).all() and (g <= f).all() and (g >= f / 8.0 * (1 - 1e-7)).all()
