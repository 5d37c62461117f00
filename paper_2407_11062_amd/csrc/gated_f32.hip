// The gated feed-forward of a few tokens in fp32: both projections from the codes as packed, the activation and the product (or its gradient) in one launch, all in binary32.
//
//   G[t] = sum over groups of s (sum over the group of (q - z) x[t]):  q - z is exact (z a whole number of N bits), the group's step multiplies a segment's sum of 32 products.
//
// The GEMM of this path computes tiles of 32 tokens; with a few the codes' bytes and the instructions that spread them are what counts: some 2.5 a code (four come out of a shift and a mask, a conversion
// each, the zero point off) and one a token.  A workgroup holds one, two or four tokens in LDS, a lane's segment of 32 apart from its neighbour's by 36, and its eight waves take turns at couples: two rows
// of the gate and their partners, a lane a segment of each row; where couples are few two, four or all eight waves share one, a part of the segments each.  Sums meet over the lanes, then over the waves,
// in a fixed order.
#include "common.h"
#include "dense_codes.h"
#include "gate.h"
#include "kernels.h"

#include <algorithm>
#include <atomic>

namespace eqat {
namespace {

constexpr int kWaves = 8, kPairs = 2, kRows = 2 * kPairs, kApart = 36;

struct FewArgs {
    const float *X; const uint32_t *codes; const float *s; const uint32_t *zp; const float *zf; const float *dH; float *H, *dY;
    int T, I, F, G, segs_per_group, kind, share;      // share: waves to a couple
    uint32_t codes_bytes, z_row_words;
};

// Sixteen codes, half H of a segment, four at a time in the bytes of a register: byte b of register k is code place<BITS>(k, b) of the sixteen.
template <int BITS> constexpr int place(int k, int b) { return BITS == 2 ? k + 4 * b : BITS == 4 ? 8 * (k / 2) + 2 * b + k % 2 : 4 * k + b; }
template <int BITS, int H, int K> __device__ __forceinline__ uint32_t four_codes(const CodeWords<BITS> &c)
{
    if constexpr (BITS == 2) return (c.w[H] >> (2 * K)) & 0x03030303u;
    else if constexpr (BITS == 4) return (c.w[2 * H + K / 2] >> (4 * (K % 2))) & 0x0F0F0F0Fu;
    else return spread_3bit(twelve_at<48 * H + 12 * K>(c));
}

template <int BITS, bool FLOATZ, int TT> __global__ __launch_bounds__(64 * kWaves) void k_gated_few_f32(const FewArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float xs[];                // [TT][segments][kApart], then [kWaves][kRows][TT] sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_segs = a.I >> 5, t0 = (int)blockIdx.y * TT, tokens = min(TT, a.T - t0);
    const __amdgpu_buffer_rsrc_t rW = make_rsrc(a.codes, a.codes_bytes);
    for (int e = threadIdx.x; e < TT * n_segs * 8; e += 64 * kWaves) {        // (tokens that are none: the last one again)
        const int t = quotient(e, n_segs * 8), in = e - t * (n_segs * 8);
        *reinterpret_cast<floatx4 *>(xs + (t * n_segs + in / 8) * kApart + in % 8 * 4) = *reinterpret_cast<const floatx4 *>(a.X + (size_t)(t0 + min(t, tokens - 1)) * a.I + in * 4);
    }
    float *const sums = xs + TT * n_segs * kApart;
    __syncthreads();
    const int couples = a.F / kPairs, slots = kWaves / a.share, slot = wave / a.share, part = wave % a.share;
    const int first = (int)blockIdx.x * slots, step = (int)gridDim.x * slots, turns = (couples - first + step - 1) / step;
    for (int turn = 0; turn < turns; ++turn) {
        const int couple = first + turn * step + slot;
        float acc[kRows][TT];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[r][t] = 0.0f;
        int row[kRows];                               // the gate's, then their partners
#pragma unroll
        for (int r = 0; r < kRows; ++r) row[r] = couple * kPairs + r % kPairs + (r < kPairs ? 0 : a.F);
        for (int seg = part * 64 + lane; seg < n_segs && couple < couples; seg += 64 * a.share) {
            const int j = quotient(seg, a.segs_per_group);
            CodeWords<BITS> c[kRows];
            float s[kRows], z[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                c[r] = load_code_words<BITS>(rW, ((uint32_t)row[r] * (uint32_t)n_segs + (uint32_t)seg) * (4u * BITS));
                s[r] = a.s[(size_t)row[r] * a.G + j];
                if constexpr (FLOATZ) {
                    z[r] = a.zf[(size_t)row[r] * a.G + j];
                } else {
                    const uint32_t bit = (uint32_t)j * BITS, *const zw = a.zp + (size_t)row[r] * a.z_row_words + (bit >> 5);
                    uint64_t two = zw[0];
                    if (BITS == 3 && (bit & 31u) > 29u) two |= (uint64_t)zw[1] << 32;
                    z[r] = (float)((uint32_t)(two >> (bit & 31u)) & ((1u << BITS) - 1u));
                }
            }
            float sum[kRows][TT];
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) sum[r][t] = 0.0f;
            auto sixteen = [&](auto half) {
                constexpr int H = decltype(half)::value;
                float x[TT][16];
#pragma unroll
                for (int t = 0; t < TT; ++t)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const floatx4 v = *reinterpret_cast<const floatx4 *>(xs + (t * n_segs + seg) * kApart + 16 * H + 4 * q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[t][4 * q + e] = v[e];
                    }
                auto four = [&](auto k4) {
                    constexpr int K = decltype(k4)::value;
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        const uint32_t v = four_codes<BITS, H, K>(c[r]);
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const float w = byte_to_float(v, b) - z[r];
#pragma unroll
                            for (int t = 0; t < TT; ++t) sum[r][t] = __builtin_fmaf(w, x[t][place<BITS>(K, b)], sum[r][t]);
                        }
                    }
                };
                four(IC<0>{}); four(IC<1>{}); four(IC<2>{}); four(IC<3>{});
            };
            sixteen(IC<0>{});
            sixteen(IC<1>{});
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[r][t] = __builtin_fmaf(s[r], sum[r][t], acc[r][t]);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                float v = acc[r][t];
#pragma unroll
                for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
                if (lane == 0) sums[(wave * kRows + r) * TT + t] = v;
            }
        __syncthreads();
        const int p = lane / TT, t = lane % TT;
        if (part == 0 && p < kPairs && t < tokens && couple < couples) {
            float g = 0.0f, u = 0.0f;
            for (int w = 0; w < a.share; ++w) { g += sums[((wave + w) * kRows + p) * TT + t]; u += sums[((wave + w) * kRows + kPairs + p) * TT + t]; }
            const int f = couple * kPairs + p;
            const size_t at = (size_t)(t0 + t) * a.F + f;
            float act, slope;
            if (a.kind == EQAT_GATE_SILU) gate_both<EQAT_GATE_SILU>(g, act, slope); else gate_both<EQAT_GATE_GELU>(g, act, slope);
            if (a.H != nullptr) a.H[at] = act * u;
            if (a.dY != nullptr) {
                const float d = a.dH[at];
                float *const dy = a.dY + (size_t)(t0 + t) * 2 * a.F + f;
                dy[0] = d * u * slope;
                dy[a.F] = d * act;
            }
        }
        __syncthreads();
    }
}

size_t lds_bytes(const Problem &p, int tt) { return ((size_t)tt * (p.I / 32) * kApart + kWaves * kRows * tt) * sizeof(float); }

template <int BITS, bool FLOATZ, int TT> void launch_tt(const Problem &p, FewArgs a, hipStream_t st)
{
    constexpr int kMost = 160 * 1024;
    static std::atomic<uint64_t> allowed{0};          // more dynamic LDS than the default limit: once per device
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev > 63) dev = 0;
    if (!((allowed.load(std::memory_order_relaxed) >> dev) & 1u)) {
        (void)hipFuncSetAttribute((const void *)k_gated_few_f32<BITS, FLOATZ, TT>, hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
        allowed.fetch_or((uint64_t)1 << dev, std::memory_order_relaxed);
    }
    const int couples = a.F / kPairs;
    a.share = 1;
    while (a.share < kWaves && couples * a.share < 4096 && 64 * a.share < a.I / 32) a.share *= 2;
    const int slots = kWaves / a.share, blocks = std::min((couples + slots - 1) / slots, 1024);
    k_gated_few_f32<BITS, FLOATZ, TT><<<dim3((unsigned)blocks, (unsigned)((a.T + TT - 1) / TT)), 64 * kWaves, lds_bytes(p, TT), st>>>(a);
}

}  // namespace

// Up to four tokens, up to sixteen of more than 2^24 weights; one token's inputs have to fit LDS.  us, the GEMM and a gate behind it / here: one token, 4096 -> 2 x 11008, 2 bit 172 / 17, 4 172 / 37, 16 172 / 125; 3 bit
// 16 172 / 93; 4 tokens, 4 bit, 2048 -> 2 x 5504 33 / 14, 16 33 / 33; 1024 -> 2 x 2752 4 13.5 / 8.8, 8 13.5 / 16.
bool gated_few_f32_applies(const Problem &p) { return !p.act_bf16 && (p.T <= 4 || (p.T <= 16 && p.O * p.I > (int64_t)1 << 24)) && lds_bytes(p, 1) <= 160 * 1024; }

// zpacked, or zero points as floats (a prepared layer's)
void launch_gated_few_f32(const Problem &p, const GatedOut &out, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, hipStream_t st)
{
    FewArgs a{};
    a.X = (const float *)X; a.codes = (const uint32_t *)codes; a.s = s; a.zp = (const uint32_t *)zpacked; a.zf = z; a.dH = (const float *)out.dH; a.H = (float *)out.H; a.dY = (float *)out.dY;
    a.T = (int)p.T; a.I = (int)p.I; a.F = (int)(p.O / 2); a.G = (int)p.G; a.segs_per_group = (int)(p.g / 32); a.kind = out.kind;
    a.codes_bytes = (uint32_t)(p.O * p.I * p.bits / 8);
    a.z_row_words = (uint32_t)((p.G * p.bits + 31) / 32);
    const int tt = a.T >= 3 && lds_bytes(p, 4) <= 80 * 1024 ? 4 : a.T >= 2 && lds_bytes(p, 2) <= 80 * 1024 ? 2 : 1;
#define EQAT_FEW_T(B, FZ) do { if (tt == 4) launch_tt<B, FZ, 4>(p, a, st); else if (tt == 2) launch_tt<B, FZ, 2>(p, a, st); else launch_tt<B, FZ, 1>(p, a, st); } while (0)
#define EQAT_FEW(B) do { if (zpacked != nullptr) EQAT_FEW_T(B, false); else EQAT_FEW_T(B, true); } while (0)
    if (p.bits == 2) EQAT_FEW(2); else if (p.bits == 3) EQAT_FEW(3); else EQAT_FEW(4);
#undef EQAT_FEW_T
#undef EQAT_FEW
}

}  // namespace eqat
