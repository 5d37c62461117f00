// The matrix-vector kernels (gemv.h) of the plain forward, and which of them a call takes.
#include "gemv.h"

namespace eqat {

// 17 to 64 tokens, on every forward entry point alike (bitwise equal results).  Above 32 tokens k_gemm_mid is the faster one
// where the rows fill the chip and the contraction is short.  This kernel takes about 8 us and 0.5 us per million weights
// there: 4096 x 4096 16 us against 25, 4096 x 11008 32 against 58; 13824 x 5120 40 against 30, 28672 x 8192 96 against 60.
bool gemv_work_applies(const Problem &p)
{
    if (!p.act_bf16 || wide_groups(p) == 0 || p.T <= 16 || p.T > 64) return false;
    return p.T <= 32 || 8.0 + 0.5e-6 * (double)(p.O * p.I) <= mid_us(p);
}

bool gemv_applies(const Problem &p)
{
    return p.act_bf16 && p.T >= 1 && (gemv_tokens_fit(p) || (p.T <= 16 && wide_groups(p) != 0) || gemv_work_applies(p));
}

FwdRoute gemv_route(const Problem &p, bool floatz)
{
    if (gemv_tokens_fit(p) && !wide_is_faster(p)) {
        const FwdKernel kernel = run_groups(p) == 0 ? FWD_GEMV_ANY : static_cast<FwdKernel>(FWD_GEMV_RUN + run_form(p, floatz));
        return FwdRoute{kernel, 16, kGemvRows};
    }
    const int tokens = p.T <= 8 ? 8 : p.T <= 16 ? 16 : p.T <= 32 ? 32 : 64;
    return FwdRoute{FWD_GEMV_WIDE, tokens, tokens >= 32 && p.O >= 2 * kGemvRows * 256 ? 2 * kGemvRows : kGemvRows};
}

void launch_gemv_work(const Problem &p, const void *X, const void *codes, const void *sz, void *Y, hipStream_t st)
{
    GemvArgs a = gemv_args(p, X, codes, sz, Y);
    a.w_row_bytes = (uint32_t)(work_code_bytes(p) / p.O);
    a.w_bytes = (uint32_t)work_code_bytes(p);
    a.s_bytes = (uint32_t)(p.O * p.G * 8);
    launch_wide<kWorking>(p, a, st);
}

void launch_gemv(const Problem &p, const void *X, const void *Wpacked, const float *s, const void *zpacked,
                 const float *zfloat, void *Y, hipStream_t st)
{
    launch_gemv_packed<false>(p, X, Wpacked, s, zpacked, zfloat, Y, 0, st);
}

}  // namespace eqat
