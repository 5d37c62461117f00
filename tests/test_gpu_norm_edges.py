"""The norm where the formula has nothing but its own terms to hold it: eps = 0, in workgroups that its rows do not fill."""
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
