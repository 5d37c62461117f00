"""A decoder layer's norm, rotary positions, attention over the 4-bit cache and gated feed-forward as they are used together: a training step of the feed-forward half with its gradients,
and a serving step of a whole layer, replayed."""
import math

import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


def packed(seed, O, I, bits, group):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    W = torch.empty((O, I), device="cuda").normal_(0.0, I ** -0.5, generator=gen).bfloat16()
    s, z = eq.eqat_init_minmax(W, bits, group)
    return (*eq.eqat_pack(W, s, z, bits, group), s)


@pytest.mark.parametrize("T", (7, 300))
def test_a_training_step_of_the_feed_forward(T):
    """S = X + R, H = gate(norm(S)), out = S + H Wd^T, all in fp32, where the plain step in 64 bits says how far: each of some six binary32 stages of sums of up to 768 terms loses at
    most 768 roundings of its terms' absolute sum, for random signs some 28 of its 2-norm; 6 x 28 x 2^-24 = 1e-5"""
    I, F, bits, g = 256, 768, 4, 64
    Wp, zp, s = packed(1, 2 * F, I, bits, g)
    Wd, zd, sd = packed(2, I, F, bits, g)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    new = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=gen)
    X, R, w, dout = new(T, I), new(T, I), 1.0 + 0.2 * new(I), new(T, I)
    # forward: S, its norm and H's inputs are kept
    f = eq.eqat_norm_fwd(X, w, EPS, R=R, want=("S", "Y"))
    H = eq.eqat_gated_fwd(f["Y"], Wp, s, zp, bits, g)
    out = f["S"] + eq.eqat_qlinear_fwd(H, Wd, sd, zd, bits, g)
    # backward: H is made anew
    down = eq.eqat_qlinear_bwd(H, Wd, sd, zd, dout, F, bits, g)
    gate = eq.eqat_gated_bwd(f["Y"], Wp, s, zp, down["dX"], bits, g)
    assert torch.equal(gate["H"], H)
    up = eq.eqat_qlinear_bwd(f["Y"], Wp, s, zp, gate["dY"], I, bits, g)
    n = eq.eqat_norm_bwd(f["S"], w, EPS, up["dX"], dS=dout)
    # the same in 64 bits
    leaf = lambda t: t.double().clone().requires_grad_()
    x, wl, sl, sdl = leaf(X + R), leaf(w), leaf(s), leaf(sd)
    weights = lambda packed_, z, step, n_in: ((ref.codes_of(packed_, n_in, bits).double().unflatten(1, (step.shape[1], -1)) - ref.codes_of(z, step.shape[1], bits).double()[..., None])
                                              * step[..., None]).flatten(1)
    y = (x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * wl) @ weights(Wp, zp, sl, I).t()
    o = x + (ref.act(0, y[:, :F])[0] * y[:, F:]) @ weights(Wd, zd, sdl, F).t()
    o.backward(dout.double())
    for got, want in ((out, o.detach()), (n["dX"], x.grad), (n["dW"], wl.grad), (up["ds"], sl.grad), (down["ds"], sdl.grad)):
        assert float((got.double() - want).norm() / want.norm()) <= 1e-5


def test_a_serving_step_replayed():
    """bf16, one token for each of three sequences through a whole layer, captured: every replay is bitwise the eager step, and near the plain step over the cache's values"""
    hidden, heads, kv, D, F, bits, g, B = 256, 4, 2, 64, 512, 4, 64, 3
    qkv, o, up, down = packed(1, (heads + 2 * kv) * D, hidden, bits, g), packed(2, hidden, hidden, bits, g), packed(3, 2 * F, hidden, bits, g), packed(4, hidden, F, bits, g)
    w1, w2 = (1.0 + 0.1 * torch.randn(hidden, device="cuda") for _ in range(2))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, lens = torch.arange(2 * B).int().view(B, 2).cuda(), i32([4, 31, 40])
    batch = eq.KvBatch(table, lens, i32(list(range(B + 1))), tokens=B, max_new=1, max_len=64)
    rot = eq.Rotary(eq.rotary_frequencies(D).cuda(), D)
    x = torch.randn((B, hidden), device="cuda").bfloat16()
    lin = lambda t, p: eq.eqat_qlinear_fwd(t, p[0], p[2], p[1], bits, g)

    def layer(cache, ws):
        y = lin(eq.eqat_norm_fwd(x, w1, EPS)["Y"], qkv).view(B, -1, D)
        q = eq.eqat_kv_rotary_write(cache, batch, rot, y[:, :heads], y[:, heads:heads + kv], y[:, heads + kv:])
        a = eq.eqat_kv_attention(cache, batch, q, ws=ws)
        f = eq.eqat_norm_fwd(lin(a.view(B, -1), o), w2, EPS, R=x, want=("S", "Y"))
        return f["S"] + lin(eq.eqat_gated_fwd(f["Y"], up[0], up[2], up[1], bits, g), down), q, a

    caches = [eq.KvCache(kv, D, 64, 32, 2 * B) for _ in range(2)]
    past = eq.KvBatch(table, lens, i32([0, 4, 35, 75]), tokens=75, max_new=40, max_len=64)
    k, v = (torch.randn((75, kv, D), device="cuda").bfloat16() for _ in "kv")
    for c in caches:
        c.pool.zero_()
        eq.eqat_kv_write(c, past, k, v)
    ws = [eq.kv_workspace(c, batch, heads) for c in caches]
    lens.add_(1)
    layer(caches[1], ws[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _, _ = layer(caches[1], ws[1])
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want, q, a = layer(caches[0], ws[0])
        assert torch.equal(out, want) and torch.equal(caches[0].pool, caches[1].pool)
        now = lens.tolist()
        K, V = eq.eqat_kv_read(caches[0], eq.KvBatch(table, lens, i32([0, *torch.tensor(now).cumsum(0).tolist()]), tokens=sum(now), max_new=max(now), max_len=64))
        at = 0
        for b, n in enumerate(now):
            Kb, Vb = (t[at:at + n].double().repeat_interleave(heads // kv, 1).transpose(0, 1) for t in (K, V))
            p = torch.softmax((Kb @ q[b].double()[:, :, None])[..., 0] / math.sqrt(D), -1)
            plain = (p[:, None] @ Vb)[:, 0]
            assert float((a[b].double() - plain).norm() / plain.norm()) <= 2.0 ** -7         # a bf16 result, keys and values exact in bf16 but for their own rounding on the way out
            at += n
        x.copy_(torch.randn((B, hidden), device="cuda"))
        lens.add_(1)


def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch):
    """a launch would go to the current device's stream with addresses of the other one; nothing is launched here"""
    X, w = torch.ones((2, 64), dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    q, pos = torch.ones((2, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    rot, layer = eq.Rotary(eq.rotary_frequencies(64).cuda(), 64), eq.eqat_pack(torch.ones((32, 64), device="cuda"), torch.ones((32, 1), device="cuda"), torch.zeros((32, 1), device="cuda"), 2, 64)
    s, cache = torch.ones((32, 1), device="cuda"), eq.KvCache(1, 64, 64, 32, 1)
    batch = eq.KvBatch(torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1,), 2, dtype=torch.int32, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda"), tokens=2, max_new=2, max_len=2)
    ready = eq.eqat_qlinear_prepare(*layer, 64, 2, 64)
    dH = torch.ones((2, 16), dtype=torch.bfloat16, device="cuda")
    before = cache.pool.clone()
    monkeypatch.setattr(eq, "_device", lambda: 1)
    for call in (lambda: eq.eqat_norm_fwd(X, w, 1e-5), lambda: eq.eqat_norm_bwd(X, w, 1e-5, X), lambda: eq.eqat_rotary(rot, pos, q), lambda: eq.eqat_kv_rotary_write(cache, batch, rot, q, q, q),
                 lambda: eq.eqat_gate_fwd(X), lambda: eq.eqat_gate_bwd(X, X[:, :32].contiguous()), lambda: eq.eqat_gated_fwd(X, layer[0], s, layer[1], 2, 64),
                 lambda: eq.eqat_gated_bwd(X, layer[0], s, layer[1], dH, 2, 64), lambda: eq.eqat_gated_fwd_prepared(X, ready, s, 16, 2, 64), lambda: eq.eqat_gated_bwd_prepared(X, ready, s, dH, 2, 64)):
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    rot.device = 1                                    # frequencies elsewhere
    for call in (lambda: eq.eqat_rotary(rot, pos, q), lambda: eq.eqat_kv_rotary_write(cache, batch, rot, q, q, q)):
        with pytest.raises(ValueError, match="frequencies"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(cache.pool, before)
