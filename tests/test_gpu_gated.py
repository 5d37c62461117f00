"""The gated feed-forward against a plain implementation in 64 bits, over the weights as the bf16 kernels hold them and over those that the layer stands for; every kernel, ragged sizes,
both directions, from packed arrays and prepared layers; and the gate by itself."""
import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, seed, I, F, bits, group):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        W = torch.empty((2 * F, I), device="cuda").normal_(0.0, I ** -0.5, generator=gen).bfloat16()
        self.I, self.F, self.bits, self.group = I, F, bits, group
        self.s, z = eq.eqat_init_minmax(W, bits, group)
        self.s = self.s * torch.empty(self.s.shape, device="cuda").normal_(0.0, 0.1, generator=gen).exp_()
        self.Wp, self.zp = eq.eqat_pack(W, self.s, z, bits, group)
        self.args = (bits, group)

    def prepared(self, dtype):
        return eq.eqat_qlinear_prepare(self.Wp, self.zp, self.I, self.bits, self.group, act_dtype=eq.BF16 if dtype == torch.bfloat16 else eq.F32)

    def check(self, T, dtype=torch.bfloat16, kind=0, seed=1, back=(False, True), prepared=(False, True)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        X = torch.empty((T, self.I), device="cuda").normal_(generator=gen).to(dtype)
        dH = torch.empty((T, self.F), device="cuda").normal_(0.0, 0.1, generator=gen).to(dtype)
        W = ref.what(self.Wp, self.s, self.zp, self.I, self.bits, rounded=dtype == torch.bfloat16)
        y, loose = X.double() @ W.t(), X.double().abs() @ W.abs().t()
        # a sum of I products in binary32, in any order: I roundings of their absolute sum (fp32: and three of a weight and a product)
        d = loose * (self.I + 3) * ref.F32
        F = self.F
        for b in back:
            want = ref.gate(kind, y[:, :F], y[:, F:], dH if b else None, dtype, d[:, :F], d[:, F:], near=dtype == torch.bfloat16)
            for p in prepared:
                if p:
                    layer = self.prepared(dtype)
                    got = (eq.eqat_gated_bwd_prepared(X, layer, self.s, dH, *self.args, kind=kind) if b else
                           {"H": eq.eqat_gated_fwd_prepared(X, layer, self.s, F, *self.args, kind=kind)})
                else:
                    got = (eq.eqat_gated_bwd(X, self.Wp, self.s, self.zp, dH, *self.args, kind=kind) if b else {"H": eq.eqat_gated_fwd(X, self.Wp, self.s, self.zp, *self.args, kind=kind)})
                assert set(got) == set(want)
                for name, (value, bound) in want.items():
                    ref.within(got[name], value, bound)
        return X, dH


# one token and a few: matrix-vector kernels, any group, rows that no block of eight divides evenly among workgroups
@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("I, F, group", [(256, 8, 64), (512, 24, 32), (1024, 200, 128), (2048, 136, 256), (480, 40, 96), (2560, 72, -1), (96, 16, 32), (8448, 64, 64)])
def test_few_tokens(I, F, group, bits):
    layer = Layer(I + F, I, F, bits, group)
    for T in (1, 2, 5, 7, 8, 9, 16):
        layer.check(T, kind=T % 2, back=(False,), prepared=(False,))
    layer.check(3)


@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("I, F, group", [(4096, 11008, 64), (8192, 14336, 128)])
def test_one_token_of_large_layers(I, F, group, bits):
    Layer(bits, I, F, bits, group).check(1, back=(False,), prepared=(False,))


# the kernel for few output tiles with token tiles of 64, 96 and 128
@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("T, I, F, group", [(17, 512, 64, 64), (64, 256, 8, 32), (65, 1056, 72, 96), (100, 512, 520, -1), (190, 1024, 4096, 128), (333, 1024, 1376, 64), (128, 2048, 8000, 128), (70, 96, 40, 96)])
def test_few_tiles(T, I, F, group, bits):
    Layer(T, I, F, bits, group).check(T, kind=T % 2)


# tiles of 128 (two rounds of them at most) and of 256, whole contractions and ragged ones, several tiles to a workgroup
@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("T, I, F, group", [(900, 1024, 2752, 64), (900, 1056, 2752, 32), (4097, 256, 2760, 128), (2000, 480, 5504, 96), (1025, 128, 11008, -1)])
def test_many_tiles(T, I, F, group, bits):
    Layer(T, I, F, bits, group).check(T, kind=bits % 2)


@pytest.mark.parametrize("bits, I, F, group", [(2, 256, 24, 64), (3, 480, 520, 96), (4, 1024, 200, -1), (3, 2080, 72, 32), (2, 32, 8, 32), (4, 4128, 40, 32)])
def test_fp32(bits, I, F, group):
    layer = Layer(I, I, F, bits, group)
    for T in (1, 2, 5, 16, 17, 33, 200):
        layer.check(T, dtype=torch.float32, kind=T % 2)


# tiles of 16 x 16, 32 x 16, 32 x 32 and 64 x 32 tokens and rows, fewer segments than waves of a tile, groups of one segment to all of them
@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("T, I, F, group", [(17, 4096, 136, 64), (20, 256, 8000, 32), (130, 1056, 1000, 96), (600, 512, 2760, 128), (1000, 480, 5504, -1), (40, 64, 24, 64), (1030, 96, 4104, 96)])
def test_tiles_in_fp32(T, I, F, group, bits):
    Layer(T + I, I, F, bits, group).check(T, dtype=torch.float32, kind=bits % 2)


@pytest.mark.parametrize("tokens, I, F, bits, group", [((1, 2, 3, 5, 16), 4096, 2816, 2, 64), ((1, 3, 6), 1056, 16424, 3, 32), ((1, 2, 3), 8192, 136, 4, 128), ((1, 3), 36352, 8, 2, 64),
                                                       ((1, 3), 36384, 8, 4, 32)])
def test_few_tokens_in_fp32(tokens, I, F, bits, group):
    """up to 16 of large layers, more couples of rows than a launch has waves, inputs of which LDS holds four tokens, one or none"""
    layer = Layer(F, I, F, bits, group)
    for T in tokens:
        layer.check(T, dtype=torch.float32, kind=T % 2)


@pytest.mark.parametrize("T", (1, 8, 100, 2000))
def test_against_the_weights_that_the_layer_stands_for(T):
    """Beside the bounds above each weight is rounded once: at most 2^-8 of it, independent of the others, so the 2-norm of G's error is at most 2^-8 of that of its products'
    random sum, |G|; H takes G's, 1.13 times at most (times |U| / |act| where act is small: silu's slope is 1/2 at 0), U's, and a rounding: sqrt(3.3) 2^-8 = 7.1e-3 of |H|"""
    layer = Layer(5, 1024, 2752, 4, 64)
    X, _ = layer.check(T, back=(False,), prepared=(False,))
    H = eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 4, 64).double()
    y = X.double() @ ref.what(layer.Wp, layer.s, layer.zp, 1024, 4, rounded=False).t()
    want = ref.act(0, y[:, :2752])[0] * y[:, 2752:]
    assert float((H - want).norm() / want.norm()) <= 7.1e-3


def test_rows_of_a_batch_do_not_meet():
    """NaN in one row of X stays in that row of H and dY, in every kernel, and what lies beside the outputs is left"""
    for T, I, F in ((3, 256, 72), (9, 512, 40), (100, 480, 72), (2000, 480, 5504), (4097, 256, 2760)):
        layer = Layer(T, I, F, 2, 32 if I == 480 else 64)
        X = torch.randn((T, I), device="cuda").bfloat16()
        dH = torch.randn((T, F), device="cuda").bfloat16()
        clean = eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, *layer.args)
        h = eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, *layer.args)
        X[T // 2] = float("nan")
        flat = {"H": torch.full((T * F + 128,), 7.0, dtype=torch.bfloat16, device="cuda"), "dY": torch.full((2 * T * F + 128,), 7.0, dtype=torch.bfloat16, device="cuda")}
        out = {"H": flat["H"][64:-64].view(T, F), "dY": flat["dY"][64:-64].view(T, 2 * F)}
        eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, *layer.args, out=out)
        others = [t for t in range(T) if t != T // 2]
        for name in out:
            assert torch.equal(out[name][others], clean[name][others]) and out[name][T // 2].isnan().all()
            assert (flat[name][:64] == 7).all() and (flat[name][-64:] == 7).all()
        eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, *layer.args, H=out["H"])
        assert torch.equal(out["H"][others], h[others]) and out["H"][T // 2].isnan().all() and (flat["H"][:64] == 7).all() and (flat["H"][-64:] == 7).all()


def test_outputs_that_are_not_wanted():
    for T, F in ((20, 72), (2000, 5504)):
        layer = Layer(1, 256, F, 3, 64)
        X, dH = torch.randn((T, 256), device="cuda").bfloat16(), torch.randn((T, F), device="cuda").bfloat16()
        both = eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, 3, 64)
        for name in ("dY", "H"):
            one = eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, 3, 64, want=(name,))
            assert set(one) == {name} and torch.equal(one[name], both[name])
        again = eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, 3, 64)
        assert all(torch.equal(again[k], both[k]) for k in both)
        if T > 64:                        # one kernel for both directions
            assert torch.equal(eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 3, 64), both["H"])
    assert eq.eqat_gated_fwd(X[:0], layer.Wp, layer.s, layer.zp, 3, 64).shape == (0, 5504)


def test_one_workspace_for_all_token_counts():
    layer = Layer(1, 512, 2752, 4, 64)
    ws = eq.gated_workspace(4097, 512, 2752, 4, 64)
    for T in (4097, 1, 900, 16, 100):
        ws.fill_(255)
        X = torch.randn((T, 512), device="cuda").bfloat16()
        assert torch.equal(eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 4, 64, ws=ws), eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 4, 64))


def test_replayed_and_on_another_stream():
    for T in (1, 100, 2000):
        layer = Layer(T, 512, 2752, 2, 64)
        prepared = layer.prepared(torch.bfloat16)
        X, dH = torch.randn((T, 512), device="cuda").bfloat16(), torch.randn((T, 2752), device="cuda").bfloat16()
        H, out = torch.empty_like(dH), {"H": torch.empty_like(dH), "dY": torch.empty((T, 5504), dtype=torch.bfloat16, device="cuda")}
        ws, wp = eq.gated_workspace(T, 512, 2752, 2, 64), eq.gated_workspace(T, 512, 2752, 2, 64, prepared=True)

        def step():
            eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 2, 64, H=H, ws=ws)
            eq.eqat_gated_bwd_prepared(X, prepared, layer.s, dH, 2, 64, out=out, ws=wp)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        side = torch.cuda.Stream()
        for k in range(3):
            X.copy_(torch.randn((T, 512), device="cuda"))
            layer.s.mul_(1.0 + 0.1 * k)
            want = eq.eqat_gated_fwd(X, layer.Wp, layer.s, layer.zp, 2, 64)
            back = eq.eqat_gated_bwd_prepared(X, prepared, layer.s, dH, 2, 64)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(H, want) and all(torch.equal(out[n], back[n]) for n in back)
            with torch.cuda.stream(side):
                step()
            side.synchronize()
            assert torch.equal(H, want) and all(torch.equal(out[n], back[n]) for n in back)


@pytest.mark.parametrize("kind", (0, 1))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_the_gate_alone(dtype, kind):
    for T, F in ((1, 8), (3, 72), (33, 1000), (5, 11008)):
        Y, dH = (3.0 * torch.randn((T, 2 * F), device="cuda")).to(dtype), torch.randn((T, F), device="cuda").to(dtype)
        Y[0, :8] = torch.tensor([0.0, -0.0, 90.0, -90.0, 1e4, -1e4, 1e-30, -1e-30]).to(dtype)
        want = ref.gate(kind, Y[:, :F].double(), Y[:, F:].double(), dH, dtype)
        got = eq.eqat_gate_bwd(Y, dH, kind, want=("dY", "H"))
        for name, (value, bound) in want.items():
            ref.within(got[name], value, bound)
        assert torch.equal(eq.eqat_gate_fwd(Y, kind), got["H"])
        kept = Y.clone(), dH.clone()
        eq.eqat_gate_bwd(Y, dH, kind, want=("dY", "H"), out={"dY": Y, "H": dH})          # in place
        assert torch.equal(Y, got["dY"]) and torch.equal(dH, got["H"])
        only = eq.eqat_gate_bwd(*kept, kind)
        assert set(only) == {"dY"} and torch.equal(only["dY"], got["dY"])


@pytest.mark.parametrize("kind", (0, 1))
def test_the_gates_gradient_against_differences(kind):
    """of H summed with weights dH; a central difference of steps of 1e-4 in 64 bits is good to 1e-8, the binary32 gradient to some 1e-6"""
    Y, dH = 2.0 * torch.randn((4, 64), device="cuda"), torch.randn((4, 32), device="cuda")
    dY = eq.eqat_gate_bwd(Y, dH, kind)["dY"]
    f = lambda y: ref.act(kind, y[:, :32])[0] * y[:, 32:] * dH.double()
    h = 1e-4
    for half in (0, 1):
        e = torch.zeros(64, dtype=torch.float64, device="cuda")
        e[32 * half:32 * half + 32] = h
        d = (f(Y.double() + e) - f(Y.double() - e)) / (2 * h)
        ref.within(dY[:, 32 * half:32 * half + 32], d, 1e-6 * (1.0 + dH.double().abs() * (1.0 + Y[:, 32:].double().abs() + Y[:, :32].double().abs())))


def test_extremes_of_the_gate():
    """infinite products give what the formulas give: act(inf) = inf; large finite ones no NaN"""
    big = torch.tensor([[1e30, -1e30, 3e38, -3e38, 1e14, -1e14, 1e5, -1e5] + [1.0] * 8], device="cuda")
    for kind in (0, 1):
        H = eq.eqat_gate_fwd(big, kind)
        assert torch.equal(H[0], torch.tensor([1e30, 0.0, 3e38, 0.0, 1e14, 0.0, 1e5, 0.0], device="cuda") + 0.0)
        inf = big.clone()
        inf[0, 0] = float("inf")
        assert eq.eqat_gate_fwd(inf, kind)[0, 0] == float("inf")


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_extremes_of_the_gradient(dtype):
    """act' is 1 or 0 far out, also where the square of G is no binary32 number; |act(g)| < 2e38 for the G below"""
    Y = torch.tensor([[1e18, -1e18, 1e20, -1e20, 1e38, -1e38, 1e6, -1e6] + [2.0] * 8], device="cuda").to(dtype)
    dH = torch.ones((1, 8), dtype=dtype, device="cuda")
    for kind in (0, 1):
        dY = eq.eqat_gate_bwd(Y, dH, kind)["dY"][0]
        assert torch.equal(dY[:8], torch.tensor([2.0, 0.0] * 4, device="cuda").to(dtype) + 0.0)
        assert torch.equal(dY[8:], Y[0, :8].clamp_min(0.0))


@pytest.mark.parametrize("T", (1, 100, 2000))          # (few tokens, few tiles, many)
def test_extremes_of_the_fused_gradient(T):
    """the same where G comes out of the products: the first input of every token is 2^67, the other ones 0"""
    I, F = 64, 2048
    layer = Layer(9, I, F, 4, 64)
    X, dH = torch.zeros((T, I), dtype=torch.bfloat16, device="cuda"), torch.ones((T, F), dtype=torch.bfloat16, device="cuda")
    X[:, 0] = 2.0 ** 67
    back = eq.eqat_gated_bwd(X, layer.Wp, layer.s, layer.zp, dH, 4, 64, kind=1)
    y = X.double() @ ref.what(layer.Wp, layer.s, layer.zp, I, 4, rounded=True).t()
    g, u = y[:, :F], y[:, F:]
    h = 2.0 ** -8                                     # one product a sum, binary32: exact; the results are rounded once, and the product of two is once more, 2^-23 of it
    for got, want in ((back["dY"][:, :F], u * (g > 0)), (back["dY"][:, F:], g.clamp_min(0.0)), (back["H"], g.clamp_min(0.0) * u)):
        some = (g.abs() > 1e6) & (want.abs() < 1e38)  # (0 where a weight stands for 0)
        assert some.float().mean() > 0.3
        ref.within(got.double()[some], want[some], ((h + 2.0 ** -20) * want.abs())[some])


def test_the_gate_beyond_32_bits():
    T, F = 100_000, 11008                             # Y is 4.4 GB
    Y = torch.zeros((T, 2 * F), dtype=torch.bfloat16, device="cuda")
    Y[-1] = torch.randn(2 * F, device="cuda")
    H = eq.eqat_gate_fwd(Y)
    assert torch.equal(H[-1:], eq.eqat_gate_fwd(Y[-1:])) and not H[:-1].any()
    dH = torch.zeros_like(H)
    dH[-1] = 1.0
    want = eq.eqat_gate_bwd(Y[-1:].clone(), dH[-1:])["dY"]
    eq.eqat_gate_bwd(Y, dH, out={"dY": Y})
    assert torch.equal(Y[-1:], want) and not Y[:-1].any()
