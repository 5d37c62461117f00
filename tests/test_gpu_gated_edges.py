"""The gated feed-forward on layers whose sums are exact, so that a lost, doubled or misplaced segment shows at any length, and on prepared layers with 9 to 16 tokens."""
import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref
from test_gpu_gated import Layer

pytestmark = pytest.mark.gpu


class Whole(Layer):
    """Codes and zero points at random, steps of 2^-10 and 2^-11.  With inputs that are whole numbers of up to 3 every product (q - z) s x is a whole multiple of 2^-11, and a sum of up to 36384 of them
    (15 * 3 * 36384 * 2 < 2^22 such multiples) is exact in binary32 in any order; (q - z) s and q s - z s are exact in bf16 too.  G and U have no error at all, and the bounds of H and dY are those of
    the activation and the last rounding."""

    def __init__(self, seed, I, F, bits, group):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.I, self.F, self.bits, self.group, self.args = I, F, bits, group, (bits, group)
        G = 1 if group == -1 else I // group
        rand = lambda most, *shape: torch.randint(0, most, shape, generator=gen, device="cuda").float()
        q, z = rand(1 << bits, 2 * F, G, I // G), rand(1 << bits, 2 * F, G)
        self.s = 2.0 ** (-10.0 - rand(2, 2 * F, G))
        self.W = ((q - z[..., None]) * self.s[..., None]).flatten(1)
        self.Wp, self.zp = eq.eqat_pack(self.W, self.s, z, bits, group)

    def check(self, T, dtype=torch.bfloat16, kind=0, seed=1, back=(False, True), prepared=(False, True)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        X = torch.randint(-3, 4, (T, self.I), generator=gen, device="cuda")
        X[:, ::32] = X[:, ::32] | 1                           # something in every segment
        X[:, -32:] = 3 - 2 * (X[:, -32:] & 1)                 # 1 and 3 in the last one
        dH = torch.empty((T, self.F), device="cuda").normal_(0.0, 0.1, generator=gen).to(dtype)
        y, F = X.double() @ self.W.double().t(), self.F
        X = X.to(dtype)
        for b in back:
            want = ref.gate(kind, y[:, :F], y[:, F:], dH if b else None, dtype, near=dtype == torch.bfloat16)
            for p in prepared:
                layer = (self.prepared(dtype), self.s) if p else (self.Wp, self.s, self.zp)
                if b:
                    got = (eq.eqat_gated_bwd_prepared if p else eq.eqat_gated_bwd)(X, *layer, dH, *self.args, kind=kind)
                else:
                    got = {"H": eq.eqat_gated_fwd_prepared(X, *layer, F, *self.args, kind=kind) if p else eq.eqat_gated_fwd(X, *layer, *self.args, kind=kind)}
                assert set(got) == set(want)
                for name, (value, bound) in want.items():
                    ref.within(got[name], value, bound)
        # the bounds see a lost segment: the last one of a token, 32 products of 1 and 3, is far beyond them in most elements
        last = (X[:, -32:].double() @ self.W[:, -32:].double().t())[:, F:].abs() * ref.act(kind, y[:, :F])[0].abs()
        value, bound = want["H"]
        assert (last > 4 * bound).float().mean() > 0.5


@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("tokens, I, F, group", [((1, 3, 17), 36352, 8, 64), ((1, 3, 20, 70), 36384, 8, 32), ((1, 2, 5, 9, 16, 33, 64), 8192, 72, 128), ((1, 16, 200), 8448, 40, 64), ((3, 16, 40), 2080, 520, 32),
                                                 ((100, 333), 4096, 136, -1), ((7, 90), 480, 40, 96), ((900, 4097), 1024, 2752, 64), ((600, 2000), 1056, 2760, 96)])
def test_sums_that_are_exact(tokens, I, F, group, dtype, bits):
    layer = Whole(I + F, I, F, bits, group)
    for T in tokens:
        layer.check(T, dtype, kind=T % 2)


@pytest.mark.parametrize("bits", (2, 3, 4))
@pytest.mark.parametrize("I, F, group", [(256, 8, 64), (512, 24, 32), (1024, 200, 128), (2048, 136, 256), (480, 40, 96), (2560, 72, -1), (8448, 64, 64), (4096, 1376, 64)])
def test_prepared_layers_with_few_tokens(I, F, group, bits):
    """every number of tokens that the matrix-vector kernels hold at once, on prepared layers, forward and backward"""
    for layer in (Layer(I + F, I, F, bits, group), Whole(I + F, I, F, bits, group)):
        for T in (1, 2, 5, 8, 9, 12, 16):
            layer.check(T, kind=T % 2, back=(False, True) if T in (1, 9, 16) else (False,), prepared=(True,))
        layer.check(32, back=(False,), prepared=(True,))
