// The matrix-vector kernels (gemv.h) of the gated feed-forward: up to 64 tokens, from the packed arrays or on a prepared layer, both projections, the activation and the product in one launch.
// Bound by the codes' bytes, for one token by their latency: 4096 -> 2 x 11008, 2 bit, 9.6 us for 28.6 MB, as long as the plain product of the same rows takes (9.9), without its results' way through memory.
#include "gemv.h"

namespace eqat {
namespace {

template <int BITS, int SRC, int NG> void wide_tokens(const GemvArgs &a, hipStream_t st)
{
    if (a.T <= 8) launch_wide_t<BITS, SRC, NG, 8, 1, true>(a, st);
    else if (a.T <= 16) launch_wide_t<BITS, SRC, NG, 16, 1, true>(a, st);
    else if (a.T <= 32) launch_wide_t<BITS, SRC, NG, 32, 1, true>(a, st);
    else launch_wide_t<BITS, SRC, NG, 64, 1, true>(a, st);
}
template <int BITS, int SRC> void wide_ng(int ng, const GemvArgs &a, hipStream_t st)
{
    if (ng == 4) wide_tokens<BITS, SRC, 4>(a, st); else if (ng == 2) wide_tokens<BITS, SRC, 2>(a, st); else wide_tokens<BITS, SRC, 1>(a, st);
}
template <int SRC> void wide(const Problem &p, const GemvArgs &a, hipStream_t st)
{
    const int ng = wide_groups(p);
    if (p.bits == 2) wide_ng<2, SRC>(ng, a, st); else if (p.bits == 3) wide_ng<3, SRC>(ng, a, st); else wide_ng<4, SRC>(ng, a, st);
}

// The kernel that stages all token rows, from the packed arrays.  Where the wide one takes the groups it is the faster one from four tokens on, and with 4-bit codes of up to 2^25 weights for any
// number.  us, staged / wide: 4096 -> 2 x 11008, 2 bit, 2 tokens 11.4 / 14.5, 4 14.9 / 14.5, 6 17.5 / 14.4; 3 bit, 5120 -> 2 x 13824, 2 tokens 19.6 / 23.7, 4 24.1 / 23.8, 6 34 / 24; 4 bit, 4096 -> 2 x 11008, one 15.4 / 17.2,
// 2048 -> 2 x 5504 7.5 / 6.6.
bool staged(const Problem &p, bool packed)
{
    if (!packed || !gemv_tokens_fit(p)) return false;
    return wide_groups(p) == 0 || (p.T <= 3 && !wide_is_faster(p) && (p.bits != 4 || p.O * p.I > (int64_t)1 << 25));
}

}  // namespace

// Up to 16 tokens wherever it can (8192 -> 2 x 3584, 2 bit, 16 tokens 13 us, k_gemm_mid 37), up to 64 where it is estimated to be the faster one: 6 us and 0.30 us per million weights, 8 and 0.5 beyond 32
// tokens.  us, here / there: 17 tokens, 4 bit, 2048 -> 2 x 5504 12.5 / 14.8, 4096 -> 2 x 1024 9.3 / 23.0, 2 bit, 4096 -> 2 x 11008 35 / 24; 64 tokens 4096 -> 2 x 1024 12.8 / 23.0, 2048 -> 2 x 5504 20 / 15.
bool gemv_gated_applies(const Problem &p, bool packed, double mid_us)
{
    if (!p.act_bf16 || p.T < 1 || p.T > 64) return false;
    if (staged(p, packed)) return true;
    if (wide_groups(p) == 0) return false;
    const double weights = (double)p.O * (double)p.I;
    return p.T <= 16 || (p.T <= 32 ? 6.0 + 0.30e-6 * weights : 8.0 + 0.5e-6 * weights) <= mid_us;
}

// zpacked: the packed arrays; else a prepared layer's codes and zero points
void launch_gemv_gated(const Problem &p, int kind, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, void *H, hipStream_t st)
{
    if (staged(p, zpacked != nullptr)) { launch_gemv_packed<true>(p, X, codes, s, zpacked, nullptr, H, kind, st); return; }
    GemvArgs a = gemv_args(p, X, codes, s, H);
    a.kind = kind;
    a.s_bytes = (uint32_t)(p.O * p.G * 4);
    if (zpacked != nullptr) {
        a.zp = (const uint32_t *)zpacked;
        a.w_row_bytes = (uint32_t)(p.I * p.bits / 8);
        a.z_row_words = (uint32_t)((p.G * p.bits + 31) / 32);
        a.w_bytes = (uint32_t)(p.O * p.I * p.bits / 8);
        a.z_bytes = (uint32_t)(p.O * a.z_row_words * 4);
        wide<kPackedZ>(p, a, st);
    } else {
        a.zf = z;
        a.w_row_bytes = (uint32_t)(work_code_bytes(p) / p.O);
        a.w_bytes = (uint32_t)work_code_bytes(p);
        a.z_bytes = a.s_bytes;
        wide<kPrepared>(p, a, st);
    }
}

}  // namespace eqat
