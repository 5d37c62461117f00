// The GEMM for few output tiles (gemm_mid.h) of the gated feed-forward: both projections, the activation and the product, or its gradient, in one launch.
#include "gemm_mid.h"

namespace eqat {

// From the packed arrays (zpacked), or on a prepared layer (its codes and zero points).  dH NULL: H; else H (may be NULL) and dY (may be NULL).
void launch_mid_gated(const Problem &p, const GatedOut &out, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, hipStream_t st)
{
    MidArgs a = zpacked != nullptr ? packed_args(p, X, codes, s, zpacked, nullptr, out.H) : prepared_args(p, X, codes, s, z, out.H);
    a.dH = (const bf16_t *)out.dH; a.dY = (bf16_t *)out.dY; a.kind = out.kind;
    if (zpacked != nullptr) launch_src<kPackedZ, true>(p, a, st); else launch_src<kPrepared, true>(p, a, st);
}

}  // namespace eqat
