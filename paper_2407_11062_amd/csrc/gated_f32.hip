// The gated feed-forward in fp32: both projections from the codes as packed, the activation and the product (or its gradient) in one launch, all in binary32.
//
// ---- a few tokens ----------------------------------------------------------------------------
//   G[t] = sum over groups of s (sum over the group of (q - z) x[t]):  q - z is exact (z a whole number of N bits), the group's step multiplies a segment's sum of 32 products.
//
// With a few tokens the codes' bytes and the instructions that spread them are what counts: some 2.5 a code (four come out of a shift and a mask, a conversion
// each, the zero point off) and one a token.  A workgroup holds one, two or four tokens in LDS, a lane's segment of 32 apart from its neighbour's by 36, and its eight waves take turns at couples: two rows
// of the gate and their partners, a lane a segment of each row; where couples are few two, four or all eight waves share one, a part of the segments each.  Sums meet over the lanes, then over the waves,
// in a fixed order.
#include "common.h"
#include "dense_codes.h"
#include "gate.h"
#include "kernels.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

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

// ---- more tokens: v_mfma_f32_32x32x2_f32, v_mfma_f32_16x16x4_f32 ---------------------------------------
// A workgroup's tile is MB blocks of R tokens (32 or 16) of R rows of the gate and their partners, which meet in the same registers.  Four waves share it, each a run of segments of 32 inputs, of which a
// group of R lanes multiplies a part; the next segment's inputs and codes, and step sizes and zero points where its group begins, are on their way while one is multiplied.  Operands go straight from memory
// into registers; what bounds it is the matrix cores (512 tokens, 4096 -> 2 x 11008, 2 bit: 763 us, 121 TFLOP/s of 157), where tiles are few the length of a tile's chain.  A weight is
// (q - z) s, rounded once.  Against the fp32 GEMM, a pairing launch before and a gate behind it: 512 tokens 918 -> 763 us, 64 193 -> 127, 17 (4 bit) 173 -> 70; 105 tokens, 6016 -> 2 x 656, backward 54 -> 43; 16
// tokens, 1024 -> 2 x 2752 14.3 -> 8.9.
struct TilesArgs {
    const float *X; const uint32_t *codes; const float *s; const uint32_t *zp; const float *zf; const float *dH; float *H, *dY;
    int T, I, F, G, segs_per_group, kind, z_row_words;
};

// N elements (t[k], f) of G and U leave, the gradients of H on their way together
template <int N> __device__ __forceinline__ void leave(const TilesArgs &a, const int (&t)[N], int f, const float (&g)[N], const float (&u)[N])
{
    float d[N];
    if (a.dY != nullptr) {
#pragma unroll
        for (int k = 0; k < N; ++k) d[k] = a.dH[(size_t)min(t[k], a.T - 1) * a.F + min(f, a.F - 1)];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float act, slope;
        if (a.kind == EQAT_GATE_SILU) gate_both<EQAT_GATE_SILU>(g[k], act, slope); else gate_both<EQAT_GATE_GELU>(g[k], act, slope);
        if (t[k] >= a.T || f >= a.F) continue;
        if (a.H != nullptr) a.H[(size_t)t[k] * a.F + f] = act * u[k];
        if (a.dY != nullptr) {
            float *const dy = a.dY + (size_t)t[k] * 2 * a.F + f;
            dy[0] = d[k] * u[k] * slope;
            dy[a.F] = d[k] * act;
        }
    }
}

// The codes of a segment that a lane multiplies: 16 of half q (R = 32) or 8 of quarter q, two words that hold them; then four of them in the bytes of a register, byte b of register k code
// place_in<BITS, R>(k, b) of the lane's.
struct Codes { uint32_t a, b; };
template <int BITS, int R> __device__ __forceinline__ Codes lane_codes(const uint32_t *w, int q)
{
    Codes c;
    if constexpr (R == 32) {
        if constexpr (BITS == 2) { c.a = w[q]; c.b = 0; }
        else if constexpr (BITS == 3) { c.a = w[q]; c.b = w[q + 1]; }
        else { const uintx2 both = *reinterpret_cast<const uintx2 *>(w + 2 * q); c.a = both[0]; c.b = both[1]; }
    } else {
        if constexpr (BITS == 2) { c.a = w[q >> 1]; c.b = 0; }
        else if constexpr (BITS == 3) { const int at = (24 * q) >> 5; c.a = w[at]; c.b = w[min(at + 1, 2)]; }
        else { c.a = w[q]; c.b = 0; }
    }
    return c;
}
template <int BITS, int R> constexpr int place_in(int k, int b) { return R == 32 ? place<BITS>(k, b) : BITS == 4 ? k + 2 * b : 4 * k + b; }
template <int BITS, int R> __device__ __forceinline__ void lane_fours(const Codes &c, int q, uint32_t (&four)[R / 8])
{
    if constexpr (R == 32) {
        const uint32_t lo = BITS == 3 && q ? __builtin_amdgcn_alignbit(c.b, c.a, 16) : c.a, hi = BITS == 3 && q ? c.b >> 16 : c.b;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            four[k] = BITS == 2 ? (lo >> (2 * k)) & 0x03030303u : BITS == 4 ? ((k < 2 ? lo : hi) >> (4 * (k % 2))) & 0x0F0F0F0Fu
                    : spread_3bit((k < 2 ? lo >> (12 * k) : k == 2 ? __builtin_amdgcn_alignbit(hi, lo, 24) : hi >> 4) & 0xFFFu);
    } else {
        const uint32_t lo = BITS == 2 ? c.a >> (16 * (q & 1)) : BITS == 3 ? __builtin_amdgcn_alignbit(c.b, c.a, (24 * q) & 31) : c.a;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if constexpr (BITS == 2) { const uint32_t x = (lo >> (8 * k)) & 0xFFu, pairs = (x | (x << 12)) & 0x000F000Fu; four[k] = (pairs | (pairs << 6)) & 0x03030303u; }
            else if constexpr (BITS == 3) four[k] = spread_3bit((lo >> (12 * k)) & 0xFFFu);
            else four[k] = (lo >> (4 * k)) & 0x0F0F0F0Fu;
        }
    }
}

__device__ __forceinline__ floatx16 multiply(float x, float w, floatx16 acc) { return __builtin_amdgcn_mfma_f32_32x32x2f32(x, w, acc, 0, 0, 0); }
__device__ __forceinline__ floatx4 multiply(float x, float w, floatx4 acc) { return __builtin_amdgcn_mfma_f32_16x16x4f32(x, w, acc, 0, 0, 0); }

constexpr int kShare = 4;               // waves of a tile
template <int BITS, int R, int MB> __global__ __launch_bounds__(64 * kShare) void k_gated_tiles_f32(const TilesArgs a)
{
    typedef std::conditional_t<R == 32, floatx16, floatx4> Acc;
    constexpr int kEach = R / 2, kSums = R * R / 64;         // inputs of a segment to a lane; sums of a block to a lane
    __shared__ float sums[kShare][2][R][R + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane % R, q = lane / R, n_segs = a.I >> 5;
    const int tiles_f = (a.F + R - 1) / R, tile_m = quotient((int)blockIdx.x, tiles_f), f0 = ((int)blockIdx.x - tile_m * tiles_f) * R, m0 = tile_m * (R * MB);
    struct Segment { floatx4 x[MB][kEach / 4]; Codes w[2]; uint32_t z[2][2]; float s[2]; int j; };
    const float *x_at[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) x_at[i] = a.X + (size_t)min(m0 + R * i + r, a.T - 1) * a.I + kEach * q;      // (rows that are none: the last one again)
    const int row0 = min(f0 + r, a.F - 1);
    auto load = [&](int seg, const Segment &before) {
        Segment v;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int e = 0; e < kEach / 4; ++e) v.x[i][e] = *reinterpret_cast<const floatx4 *>(x_at[i] + seg * 32 + 4 * e);
#pragma unroll
        for (int b = 0; b < 2; ++b) v.w[b] = lane_codes<BITS, R>(a.codes + ((size_t)(row0 + b * a.F) * n_segs + seg) * BITS, q);
        v.j = __builtin_amdgcn_readfirstlane(quotient(seg, a.segs_per_group));
#pragma unroll
        for (int b = 0; b < 2; ++b) { v.s[b] = before.s[b]; v.z[b][0] = before.z[b][0]; v.z[b][1] = before.z[b][1]; }
        if (v.j != before.j) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const size_t row = (size_t)(row0 + b * a.F);
                v.s[b] = a.s[row * a.G + v.j];
                if (a.zp == nullptr) {
                    v.z[b][0] = __float_as_uint(a.zf[row * a.G + v.j]);
                } else {
                    const uint32_t bit = (uint32_t)v.j * BITS, *const zw = a.zp + row * a.z_row_words + (bit >> 5);
                    v.z[b][0] = zw[0];
                    if (BITS == 3) v.z[b][1] = zw[(bit & 31u) > 29u ? 1 : 0];
                }
            }
        }
        return v;
    };
    Acc acc[MB][2];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < kSums; ++e) acc[i][b][e] = 0.0f;
    const int first_seg = (int)((int64_t)n_segs * wave / kShare), end_seg = (int)((int64_t)n_segs * (wave + 1) / kShare);
    Segment now;
    now.j = -1;
#pragma unroll
    for (int b = 0; b < 2; ++b) { now.s[b] = 0.0f; now.z[b][0] = now.z[b][1] = 0; }
    now = load(min(first_seg, n_segs - 1), now);
    for (int seg = first_seg; seg < end_seg; ++seg) {
        const Segment next = load(min(seg + 1, n_segs - 1), now);
        __builtin_amdgcn_sched_barrier(0);             // (left to itself the compiler moves these loads behind the products)
        float w[2][kEach];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float z = __uint_as_float(now.z[b][0]);
            if (a.zp != nullptr) {
                const uint32_t at = ((uint32_t)now.j * BITS) & 31u, word = BITS == 3 ? __builtin_amdgcn_alignbit(now.z[b][1], now.z[b][0], at) : now.z[b][0] >> at;
                z = (float)(word & ((1u << BITS) - 1u));
            }
            uint32_t four[kEach / 4];
            lane_fours<BITS, R>(now.w[b], q, four);
#pragma unroll
            for (int k = 0; k < kEach / 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[b][place_in<BITS, R>(k, e)] = (byte_to_float(four[k], e) - z) * now.s[b];
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[i][b] = multiply(now.x[i][e / 4][e % 4], w[b][e], acc[i][b]);
        __builtin_amdgcn_sched_barrier(0);
        now = next;
    }
    // acc[..][e] of a lane: token 8 (e / 4) + 4 q + e % 4 of 32, or 4 q + e of 16, row r
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        if (i > 0) __syncthreads();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < kSums; ++e) sums[wave][b][8 * (e >> 2) + 4 * q + (e & 3)][r] = acc[i][b][e];
        __syncthreads();
        constexpr int N = kSums / kShare;
        int t[N];
        float g[N], u[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int in = (k * kShare + wave) * (64 / R) + q;
            t[k] = m0 + R * i + in;
            g[k] = u[k] = 0.0f;
#pragma unroll
            for (int v = 0; v < kShare; ++v) { g[k] += sums[v][0][in][r]; u[k] += sums[v][1][in][r]; }
        }
        leave(a, t, f0 + r, g, u);
    }
}

size_t lds_bytes(const Problem &p, int tt) { return ((size_t)tt * (p.I / 32) * kApart + kWaves * kRows * tt) * sizeof(float); }

// tokens of a workgroup
int few_at_once(const Problem &p) { return p.T >= 3 && lds_bytes(p, 4) <= 80 * 1024 ? 4 : p.T >= 2 && lds_bytes(p, 2) <= 80 * 1024 ? 2 : 1; }

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

// Which of the kernels, by what they are estimated to take, us: with a few tokens (one token's inputs have to fit LDS) 7 and 0.12, 0.25 or 0.36 for every million weights and one, two or four tokens; or rounds of one workgroup a
// compute unit, so much for every segment of each.  Measured, few tokens / 16 x 16 tiles: 4096 -> 2 x 11008, 2 bit, one token 18 / 51, 4 40 / 55, 16 131 / 66; 4 tokens, 1024 -> 2 x 2752 9.8 / 8.5.  Tiles of
// 16 x 16, 32 x 16, 32 x 32, 64 x 32 (tokens x rows): 33 tokens, 8192 -> 2 x 512 40 / 55 / 95 / 147; 17 tokens, 4096 -> 2 x 11008 99 / 70 / 86 / 148; 64 tokens 221 / 168 / 127 / 152; 512 tokens 1700 / 1166 / 813 / 763.
enum F32Kernel { kFewTokens, kTiles16x16, kTiles32x16, kTiles32x32, kTiles64x32 };
static F32Kernel f32_kernel(const Problem &p)
{
    static const struct { int tokens, rows; double first, each; } tiles[4] = {{16, 16, 4.5, 0.135}, {32, 16, 5.0, 0.195}, {32, 32, 6.0, 0.315}, {64, 32, 6.0, 0.57}};
    const double millions = (double)p.O * (double)p.I * 1e-6;
    const int few = few_at_once(p);
    double best = p.T <= 16 && lds_bytes(p, 1) <= 160 * 1024 ? 7.0 + millions * (double)((p.T + few - 1) / few) * (few == 4 ? 0.36 : few == 2 ? 0.25 : 0.12) : 1e30;
    F32Kernel k = kFewTokens;
    for (int t = 0; t < 4; ++t) {
        const int64_t n = ((p.T + tiles[t].tokens - 1) / tiles[t].tokens) * ((p.O / 2 + tiles[t].rows - 1) / tiles[t].rows);
        const double us = tiles[t].first + (double)((n + 255) / 256) * (double)(p.I / 32) * tiles[t].each;
        if (us < best) { best = us; k = (F32Kernel)(kTiles16x16 + t); }
    }
    return k;
}

// zpacked, or zero points as floats (a prepared layer's)
static void launch_few(const Problem &p, const GatedOut &out, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, hipStream_t st)
{
    FewArgs a{};
    a.X = (const float *)X; a.codes = (const uint32_t *)codes; a.s = s; a.zp = (const uint32_t *)zpacked; a.zf = z; a.dH = (const float *)out.dH; a.H = (float *)out.H; a.dY = (float *)out.dY;
    a.T = (int)p.T; a.I = (int)p.I; a.F = (int)(p.O / 2); a.G = (int)p.G; a.segs_per_group = (int)(p.g / 32); a.kind = out.kind;
    a.codes_bytes = (uint32_t)(p.O * p.I * p.bits / 8);
    a.z_row_words = (uint32_t)((p.G * p.bits + 31) / 32);
    const int tt = few_at_once(p);
#define EQAT_FEW_T(B, FZ) do { if (tt == 4) launch_tt<B, FZ, 4>(p, a, st); else if (tt == 2) launch_tt<B, FZ, 2>(p, a, st); else launch_tt<B, FZ, 1>(p, a, st); } while (0)
#define EQAT_FEW(B) do { if (zpacked != nullptr) EQAT_FEW_T(B, false); else EQAT_FEW_T(B, true); } while (0)
    if (p.bits == 2) EQAT_FEW(2); else if (p.bits == 3) EQAT_FEW(3); else EQAT_FEW(4);
#undef EQAT_FEW_T
#undef EQAT_FEW
}

template <int BITS> static void launch_tiles(F32Kernel k, const TilesArgs &a, hipStream_t st)
{
    auto go = [&](auto kern, int tokens, int rows) { kern<<<dim3((unsigned)((a.F + rows - 1) / rows) * (unsigned)((a.T + tokens - 1) / tokens)), 64 * kShare, 0, st>>>(a); };
    if (k == kTiles16x16) go(k_gated_tiles_f32<BITS, 16, 1>, 16, 16);
    else if (k == kTiles32x16) go(k_gated_tiles_f32<BITS, 16, 2>, 32, 16);
    else if (k == kTiles32x32) go(k_gated_tiles_f32<BITS, 32, 1>, 32, 32);
    else go(k_gated_tiles_f32<BITS, 32, 2>, 64, 32);
}

void launch_gated_f32(const Problem &p, const GatedOut &out, const void *X, const void *codes, const float *s, const void *zpacked, const float *z, hipStream_t st)
{
    const F32Kernel k = f32_kernel(p);
    if (k == kFewTokens) { launch_few(p, out, X, codes, s, zpacked, z, st); return; }
    TilesArgs a{};
    a.X = (const float *)X; a.codes = (const uint32_t *)codes; a.s = s; a.zp = (const uint32_t *)zpacked; a.zf = z; a.dH = (const float *)out.dH; a.H = (float *)out.H; a.dY = (float *)out.dY;
    a.T = (int)p.T; a.I = (int)p.I; a.F = (int)(p.O / 2); a.G = (int)p.G; a.segs_per_group = (int)(p.g / 32); a.kind = out.kind;
    a.z_row_words = (int)((p.G * p.bits + 31) / 32);
    if (p.bits == 2) launch_tiles<2>(k, a, st); else if (p.bits == 3) launch_tiles<3>(k, a, st); else launch_tiles<4>(k, a, st);
}

}  // namespace eqat
