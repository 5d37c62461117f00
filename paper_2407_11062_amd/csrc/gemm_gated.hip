// The tile GEMM (tile_gemm.h) of the gated feed-forward, for more tokens than gemm_mid_gated.hip takes: both projections, the activation and the product, or its gradient, in one launch.
//
// The main loop is the plain forward's (the weight operand rebuilt from codes in LDS, v_mfma_f32_32x32x16_bf16); rows of the two halves take turns in its columns, and G and U meet in
// the registers that they were summed in, binary32.  Against the plain forward and a gate behind it this leaves out 3 T F elements of traffic and a launch, and two roundings.
// Whole tiles only: no tile is cut along the contraction, and no scratch is needed.
#include "common.h"
#include "kernels.h"
#include "tile_gemm.h"

#include <algorithm>
#include <atomic>

namespace eqat {
namespace {

template <int BITS, int MODE, typename TS, int GATE>
__global__ __launch_bounds__(64 * TS::WGM * TS::WGN) void k_gemm_gated(const GemmQArgs a)
{
    gemm_q_body<BITS, false, MODE, TS::BM, TS::BN, TS::BK, TS::WGM, TS::WGN, GATE>(a, (int)blockIdx.x, (int)gridDim.x);
}

int device_now()
{
    int dev = 0;
    return hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 64 ? dev : 0;
}

template <int BITS, int MODE, typename TS, int GATE> void launch_t(GemmQArgs a, hipStream_t st)
{
    constexpr size_t smem = q_smem_bytes<false, TS>();
    static_assert(smem <= 160 * 1024, "LDS of one CU");
    constexpr int per_cu = smem * 2 <= 160 * 1024 ? 2 : 1;
    static std::atomic<uint64_t> allowed{0};          // more dynamic LDS than the default limit: once per device
    static std::atomic<int> cus_of[64];
    const int dev = device_now();
    if (!((allowed.load(std::memory_order_relaxed) >> dev) & 1u)) {
        (void)hipFuncSetAttribute((const void *)k_gemm_gated<BITS, MODE, TS, GATE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 8) n = 256;
        cus_of[dev].store(n, std::memory_order_relaxed);
        allowed.fetch_or((uint64_t)1 << dev, std::memory_order_release);
    }
    const int n_cus = cus_of[dev].load(std::memory_order_relaxed), resident = ((n_cus > 0 ? n_cus : 256) * per_cu) & ~7;
    a.tiles_m = (a.M + TS::BM - 1) / TS::BM;
    a.tiles_n = (a.N + TS::BN - 1) / TS::BN;
    a.band = std::max(2, std::min(8, a.tiles_m / 8));
    const int ntiles = a.tiles_m * a.tiles_n;
    a.sk = SkPlan{};
    a.sk.pairs = ((a.K + TS::BK - 1) / TS::BK + 1) / 2;
    a.sk.walk = ntiles > resident ? 1 : 0;            // several tiles to a workgroup: the first of the next is on its way when one ends
    a.sk.dp_rounds = (ntiles + resident - 1) / resident;
    k_gemm_gated<BITS, MODE, TS, GATE><<<dim3((unsigned)(a.sk.walk ? resident : ntiles)), dim3(64 * TS::WGM * TS::WGN), smem, st>>>(a);
}

template <int BITS, int GATE> void launch_bits(const GemmQArgs &a, hipStream_t st)
{
    // as the plain forward: big tiles where they fill most of the chip or the small ones do not fit twice a compute unit
    const int64_t big = (int64_t)((a.M + 255) / 256) * ((a.N + 255) / 256), small = (int64_t)((a.M + 127) / 128) * ((a.N + 127) / 128);
    const bool whole = a.K % 128 == 0;
    if (big >= 160 || small > 512) {
        if (whole) launch_t<BITS, kWhole, TileBig, GATE>(a, st); else launch_t<BITS, kRagged, TileBig, GATE>(a, st);
    } else {
        if (whole) launch_t<BITS, kWhole, TileSmall, GATE>(a, st); else launch_t<BITS, kRagged, TileSmall, GATE>(a, st);
    }
}

}  // namespace

void launch_tiles_gated(const Problem &p, const GatedOut &out, const void *X, const void *codes, const void *sz, hipStream_t st)
{
    GemmQArgs a{};
    a.A = (const bf16_t *)X; a.codes = (const uint32_t *)codes; a.sz = (const floatx2 *)sz; a.C = (bf16_t *)out.H;
    a.M = (int)p.T; a.N = (int)p.O; a.K = (int)p.I; a.I = (int)p.I; a.G = (int)p.G; a.g = (int)p.g;
    a.a_bytes = (uint32_t)(p.T * p.I * 2); a.codes_bytes = (uint32_t)work_code_bytes(p); a.sz_bytes = (uint32_t)(p.O * p.G * 8);
    a.c_bytes = out.H != nullptr ? (uint32_t)(p.T * p.O) : 0u;
    a.dH = (const bf16_t *)out.dH; a.dY = (bf16_t *)out.dY; a.kind = out.kind;
    a.dh_bytes = out.dH != nullptr ? (uint32_t)(p.T * p.O) : 0u; a.dy_bytes = out.dY != nullptr ? (uint32_t)(p.T * p.O * 2) : 0u;
#define EQAT_GATED(B) do { if (out.dH != nullptr) launch_bits<B, kGateBwd>(a, st); else launch_bits<B, kGateFwd>(a, st); } while (0)
    if (p.bits == 2) EQAT_GATED(2); else if (p.bits == 3) EQAT_GATED(3); else EQAT_GATED(4);
#undef EQAT_GATED
}

}  // namespace eqat
