"""The norm at its edges: eps = 0 in workgroups that its rows do not fill, 8-bit codes at the ties of the quotient and beside infinities, eps as a tensor."""
import pytest
import torch

import paper_2407_11062_amd as eq
import layer_reference as ref
from test_gpu_norm import rows, weight

pytestmark = pytest.mark.gpu


# 32, 16, 8 and 4 rows to a workgroup, and one (forms of 256 lanes and more); numbers of rows that fill the last workgroup and that do not, one workgroup and several
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n", (8, 64, 72, 128, 136, 256, 264, 512, 520, 1024, 1032, 4096, 16392))
def test_no_eps(n, dtype):
    for T in (1, 3, 13, 32, 33, 517):
        S, W, dY, dS = rows(n, T, n, dtype), weight(n + 2, n, torch.float32), rows(n + 3, T, n, dtype, 0.02), rows(n + 4, T, n, dtype, 0.02)
        _, _, Y = ref.norm(S, W, 0.0)
        ref.within(eq.eqat_norm_fwd(S, W, 0.0)["Y"], Y, Y.abs() * (ref.half(dtype) + ref.NORM_ROUNDINGS * ref.F32))
        out = eq.eqat_norm_bwd(S, W, 0.0, dY, dS)
        dX, dW, bound, terms = ref.norm_back(S, W, 0.0, dY, dS)
        ref.within(out["dX"], dX, bound)
        # rows that a workgroup adds up one after the other (a 256th of them at most), up to 32 rows of the same workgroup and 48 parts; rstd's and the product's roundings
        ref.within(out["dW"], dW, terms.abs().sum(0) * (T // 256 + 1 + 32 + 48 + ref.NORM_ROUNDINGS + 2) * ref.F32)


@pytest.mark.parametrize("T, n, group", [(515, 5120, 128), (515, 5120, -1), (700, 1024, 32), (300, 8192, 512), (40, 32768, 256), (3, 64, 64)])
def test_codes_are_those_of_the_quotient(T, n, group):
    """Y leaves in fp32 as the codes are made from it: they are e4m3 of Y / scale, the quotient rounded to binary32 (of a 64-bit one: the same number), and at its ties, of which inputs and weights of a
    few bits make many, those of the even neighbour"""
    X, W = rows(n, T, n, torch.bfloat16).float(), weight(n + 1, n, torch.bfloat16).float()
    X[0, 1::5] = 0.0
    X[0, 3::5] = -0.0
    out = eq.eqat_norm_fwd(X, W, 0.0, group=group, want=("Y", "codes"))
    per = n if group == -1 else group
    q = (out["Y"].double().unflatten(1, (-1, per)) / out["scales"].double()[..., None]).float().flatten(1)
    assert torch.equal(out["codes"].view(torch.uint8), q.to(torch.float8_e4m3fn).view(torch.uint8))


def test_codes_beside_an_infinity():
    """a scale that is infinite: finite elements of its group are 0, the infinite one is NaN"""
    X, W = torch.ones((2, 64), device="cuda"), torch.ones(64, device="cuda")
    X[:, 5], W[5] = 100.0, 3.0e38
    out = eq.eqat_norm_fwd(X, W, 1e-5, group=32, want=("Y", "codes"))
    assert (out["Y"][:, 5] == float("inf")).all() and (out["scales"][:, 0] == float("inf")).all()
    codes = out["codes"].float()
    assert codes[:, 5].isnan().all() and not codes[:, :5].any() and not codes[:, 6:32].any() and (codes[:, 32:] == 448.0).all()


def test_eps_that_is_a_tensor():
    """goes by its value, at every call"""
    S, dY = rows(1, 3, 64, torch.float32), rows(2, 3, 64, torch.float32)
    eps = torch.tensor(1e-5)
    for value in (1e-5, 100.0):
        eps.fill_(value)
        assert torch.equal(eq.eqat_norm_fwd(S, None, eps)["Y"], eq.eqat_norm_fwd(S, None, float(eps))["Y"])
        assert torch.equal(eq.eqat_norm_bwd(S, None, eps, dY)["dX"], eq.eqat_norm_bwd(S, None, float(eps), dY)["dX"])
