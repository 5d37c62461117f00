// The GEMM for few output tiles (gemm_mid.h) of the gated feed-forward: both projections, the activation and the product, or its gradient, in one launch.
#include "gemm_mid.h"

namespace eqat {

// What it takes, in us, with the best of its token tiles (*tokens), from the packed arrays or on a prepared layer: rounds of workgroups, a beginning each and so much for every 64 inputs.  Fitted to 60
// sizes (65 to 2000 tokens, 1024 -> 2 x 2752, 2 bit, to 8192 -> 2 x 28672, 4 bit; prepared): us a round, 64 / 96 / 128 tokens, 2 bit, 1024 inputs 10.4 / 12.3 / 14.3, 4096 21 / 26 / 33; 3 bit, 5120
// 26 / 36 / 41; 4 bit, 8192 42 / 58 / 64.  From 3-bit codes as packed a step of 256 inputs takes 0.45 us longer.
double mid_gated_us(const Problem &p, bool packed, int *tokens)
{
    static const double first[3] = {7.0, 7.0, 8.1}, each[3][3] = {{0.225, 0.245, 0.27}, {0.285, 0.36, 0.395}, {0.381, 0.405, 0.44}};
    double best = 1e30;
    for (int k = 0; k < 3; ++k) {
        const int bm = k == 0 ? 64 : k == 1 ? 96 : 128;
        if (bm == 128 && !(p.g == 32 || p.g == 64 || p.g % 128 == 0)) continue;          // (see tall_applies)
        const double us = (double)rounds_of(p, bm) * (first[k] + (each[k][p.bits - 2] + (packed && p.bits == 3 ? 0.11 : 0.0)) * (double)((p.I + 63) / 64));
        if (us < best) { best = us; *tokens = bm; }
    }
    return best;
}

// From the packed arrays (zpacked), or on a prepared layer (its codes and zero points).  dH NULL: H; else H (may be NULL) and dY (may be NULL).
void launch_mid_gated(const Problem &p, int tokens, const GatedOut &out, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, hipStream_t st)
{
    MidArgs a = zpacked != nullptr ? packed_args(p, X, codes, s, zpacked, nullptr, out.H) : prepared_args(p, X, codes, s, z, out.H);
    a.dH = (const bf16_t *)out.dH; a.dY = (bf16_t *)out.dY; a.kind = out.kind;
    if (zpacked != nullptr) launch_src<kPackedZ, true>(p, a, st, tokens); else launch_src<kPrepared, true>(p, a, st, tokens);
}

}  // namespace eqat
