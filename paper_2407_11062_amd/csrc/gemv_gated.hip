// The matrix-vector kernels (gemv.h) of the gated feed-forward: up to 16 tokens, from the packed arrays, both projections, the activation and the product in one launch.
#include "gemv.h"

namespace eqat {

// as gemv_applies, up to 16 tokens
bool gemv_gated_applies(const Problem &p) { return p.act_bf16 && p.T >= 1 && p.T <= 16 && (gemv_tokens_fit(p) || wide_groups(p) != 0); }

void launch_gemv_gated(const Problem &p, int kind, const void *X, const void *Wpacked, const float *s, const void *zpacked, void *H, hipStream_t st)
{
    launch_gemv_packed<true>(p, X, Wpacked, s, zpacked, nullptr, H, kind, st);
}

}  // namespace eqat
