// The tile GEMM (tile_gemm.h) of the gated feed-forward, for more tokens than gemm_mid_gated.hip takes: both projections, the activation and the product, or its gradient, in one launch.
//
// The main loop is the plain forward's (the weight operand rebuilt from codes in LDS, v_mfma_f32_32x32x16_bf16); rows of the two halves take turns in its columns, and G and U meet in
// the registers that they were summed in, binary32.  Against the plain forward and a gate behind it this leaves out 3 T F elements of traffic and a launch, and two roundings.
// A packed layer's codes are read as packed: the same main loop with another segment load and some more arithmetic, against a re-layout in front of it, us, re-laid / as packed: 333 tokens, 3 bit,
// 5120 -> 2 x 13824 123 / 111; 2048 tokens, 4 bit, 8192 -> 2 x 28672 1641 / 1572, 2 bit, 4096 -> 2 x 11008 315 / 311; only 3-bit codes lose from some 3000 tokens on (4096 tokens 945 / 958).
// Whole tiles only: no tile is cut along the contraction, and no scratch is needed.  Bound by the matrix cores: 2048 tokens, 8192 -> 2 x 28672, 4 bit, 1530 to 1620 us (1258 to 1186 TFLOP/s; a plain product
// reaches 1303), 333 tokens, 5120 -> 2 x 13824 106 (216 tiles on 256 compute units), backward of 4096 tokens, 4096 -> 2 x 11008 654 (5.4 rounds of tiles).
// The weights are what all bf16 kernels here multiply with: q s - z s by one multiply-add, rounded to bf16, so that a matrix instruction takes 16 inputs; exact codes would need sums a group of their own.
#include "common.h"
#include "kernels.h"
#include "tile_gemm.h"

#include <algorithm>
#include <atomic>

namespace eqat {
namespace {

typedef Tile<192, 256, 64, 2, 4> TileMiddle;      // 8 waves, 96x64 per wave

template <int BITS, int MODE, typename TS, int GATE, bool DENSE>
__global__ __launch_bounds__(64 * TS::WGM * TS::WGN) void k_gemm_gated(const GemmQArgs a)
{
    gemm_q_body<BITS, false, MODE, TS::BM, TS::BN, TS::BK, TS::WGM, TS::WGN, GATE, DENSE>(a, (int)blockIdx.x, (int)gridDim.x);
}

// (step size, zero point) pairs, four neighbouring groups of a row to a lane.  57344 x 64 of them, 4 bit, 45 MB, 16.7 (one to a lane) -> 11.9 us;
// 27648 x 40 5.9 -> 5.7.
template <int BITS, bool FLOATZ>
__global__ __launch_bounds__(256) void k_gated_pairs(const float *__restrict__ s, const uint32_t *__restrict__ zp, const float *__restrict__ zf, floatx2 *__restrict__ sz, int quads, int row_quads,
                                                     int z_row_words)
{
    const int t = (int)(blockIdx.x * 256u + threadIdx.x);
    if (t >= quads) return;
    const floatx4 step = reinterpret_cast<const floatx4 *>(s)[t];
    floatx4 z;
    if constexpr (FLOATZ) {
        z = reinterpret_cast<const floatx4 *>(zf)[t];
    } else {
        const int row = quotient(t, row_quads);
        const uint32_t bit = (uint32_t)(t - row * row_quads) * (4u * BITS), *const at = zp + (size_t)row * z_row_words + (bit >> 5);
        uint64_t four = at[0];
        if (BITS == 3 && (bit & 31u) > 20u) four |= (uint64_t)at[1] << 32;
        four >>= bit & 31u;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (float)((uint32_t)(four >> (e * BITS)) & ((1u << BITS) - 1u));
    }
    floatx4 *const to = reinterpret_cast<floatx4 *>(sz) + 2 * (size_t)t;
    to[0] = floatx4{step[0], z[0], step[1], z[1]};
    to[1] = floatx4{step[2], z[2], step[3], z[3]};
}

int device_now()
{
    int dev = 0;
    return hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 64 ? dev : 0;
}

template <int BITS, int MODE, typename TS, int GATE, bool DENSE> void launch_t(GemmQArgs a, hipStream_t st)
{
    constexpr size_t smem = q_smem_bytes<false, TS>();
    static_assert(smem <= 160 * 1024, "LDS of one CU");
    constexpr int per_cu = smem * 2 <= 160 * 1024 ? 2 : 1;
    static std::atomic<uint64_t> allowed{0};          // more dynamic LDS than the default limit: once per device
    static std::atomic<int> cus_of[64];
    const int dev = device_now();
    if (!((allowed.load(std::memory_order_relaxed) >> dev) & 1u)) {
        (void)hipFuncSetAttribute((const void *)k_gemm_gated<BITS, MODE, TS, GATE, DENSE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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
    k_gemm_gated<BITS, MODE, TS, GATE, DENSE><<<dim3((unsigned)(a.sk.walk ? resident : ntiles)), dim3(64 * TS::WGM * TS::WGN), smem, st>>>(a);
}

template <int BITS, int GATE, bool DENSE> void launch_bits(const GemmQArgs &a, int tokens, hipStream_t st)
{
    const bool whole = a.K % 128 == 0;
    if (tokens == TileBig::BM) {
        if (whole) launch_t<BITS, kWhole, TileBig, GATE, DENSE>(a, st); else launch_t<BITS, kRagged, TileBig, GATE, DENSE>(a, st);
    } else {
        if (whole) launch_t<BITS, kWhole, TileMiddle, GATE, DENSE>(a, st); else launch_t<BITS, kRagged, TileMiddle, GATE, DENSE>(a, st);
    }
}

template <int BITS, int GATE> void launch_dense(const GemmQArgs &a, int tokens, bool dense, hipStream_t st)
{
    if (dense) launch_bits<BITS, GATE, true>(a, tokens, st); else launch_bits<BITS, GATE, false>(a, tokens, st);
}

}  // namespace

// What it takes, in us, with the better of its token tiles: rounds of one workgroup a compute unit, a beginning each and so much for every K tile of 64, the more the longer they run (the chip's power).
// Fitted to the same sizes as mid_gated_us, which also says why there are tiles of 192: 333 tokens are two of them, 11008 x 4096 91 -> 77 us, 515 tokens of 28672 x 8192 640 -> 527, 1500 of 4096 301 -> 251.
// (128 x 128, two workgroups a compute unit, was never the best.)
double tiles_gated_us(const Problem &p, int *tokens)
{
    const double k = (double)((p.I + 63) / 64);
    auto us = [&](int bm, double first, double each, double more) {
        const int64_t tiles = ((p.T + bm - 1) / bm) * ((p.O + 255) / 256);
        return (double)((tiles + 255) / 256) * (first + k * (each + more * k));
    };
    const double big = us(256, 10.0, 1.27, 0.003), middle = us(192, 8.0, 1.03, 0.0025);
    *tokens = middle < big ? 192 : 256;
    return (middle < big ? middle : big) + 2.5;            // the launch in front that pairs step sizes and zero points
}

void launch_gated_pairs(const Problem &p, const float *s, const void *zpacked, const float *z, void *sz, hipStream_t st)
{
    if (p.G % 4 != 0) { launch_e2e_prepare(p, nullptr, nullptr, s, zpacked, z, sz, nullptr, nullptr, 0, st); return; }          // rows begin between vectors
    const int quads = (int)(p.O * p.G / 4), row_words = (int)((p.G * p.bits + 31) / 32);
    const unsigned blocks = (unsigned)((quads + 255) / 256);
#define EQAT_PAIRS(B, FZ) k_gated_pairs<B, FZ><<<blocks, 256, 0, st>>>(s, (const uint32_t *)zpacked, z, (floatx2 *)sz, quads, (int)p.G / 4, row_words)
    if (zpacked == nullptr) EQAT_PAIRS(2, true);
    else if (p.bits == 2) EQAT_PAIRS(2, false); else if (p.bits == 3) EQAT_PAIRS(3, false); else EQAT_PAIRS(4, false);
#undef EQAT_PAIRS
}

void launch_tiles_gated(const Problem &p, int tokens, bool dense, const GatedOut &out, const void *X, const void *codes, const void *sz, hipStream_t st)
{
    GemmQArgs a{};
    a.A = (const bf16_t *)X; a.codes = (const uint32_t *)codes; a.sz = (const floatx2 *)sz; a.C = (bf16_t *)out.H;
    a.M = (int)p.T; a.N = (int)p.O; a.K = (int)p.I; a.I = (int)p.I; a.G = (int)p.G; a.g = (int)p.g;
    a.a_bytes = (uint32_t)(p.T * p.I * 2); a.codes_bytes = dense ? (uint32_t)(p.O * p.I * p.bits / 8) : (uint32_t)work_code_bytes(p); a.sz_bytes = (uint32_t)(p.O * p.G * 8);
    a.c_bytes = out.H != nullptr ? (uint32_t)(p.T * p.O) : 0u;
    a.dH = (const bf16_t *)out.dH; a.dY = (bf16_t *)out.dY; a.kind = out.kind;
    a.dh_bytes = out.dH != nullptr ? (uint32_t)(p.T * p.O) : 0u; a.dy_bytes = out.dY != nullptr ? (uint32_t)(p.T * p.O * 2) : 0u;
#define EQAT_GATED(B) do { if (out.dH != nullptr) launch_dense<B, kGateBwd>(a, tokens, dense, st); else launch_dense<B, kGateFwd>(a, tokens, dense, st); } while (0)
    if (p.bits == 2) EQAT_GATED(2); else if (p.bits == 3) EQAT_GATED(3); else EQAT_GATED(4);
#undef EQAT_GATED
}

}  // namespace eqat
