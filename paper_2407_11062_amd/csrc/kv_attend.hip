// Attention over the 4-bit cache, streamed: a wave takes whole records of 32 tokens, for up to 16 rows (query, head) that share a head of the cache.
//
// Bound by the bytes of the cache.  The records that a head of the cache holds for all rows of a call are one row of work, cut into equal shares, one for a workgroup and as
// many as are resident: a share may end within a unit (16 rows of a sequence) and begin in the next, so lengths that differ leave nobody waiting.  Records come by
// direct-to-LDS loads into a ring of each wave's own, so that two are on their way while one is worked on, without a register.
//
// With x^ = m + s c (kv.h) the sums over elements and tokens part into sums over codes, which are exact in binary16, and sums over the steps:
//   q . k^_t   = sum over groups g of  s_tg (q_g . c_tg) + m_tg sum(q_g)
//   sum_t p_t v^_td = sum_t (p_t s_tg) c_td  +  sum_t p_t m_tg
// The products with codes run on the matrix cores, everything else in binary32; no key or value is ever rebuilt.  q and p s are binary16 there: q of bf16 exactly
// (scaled by a power of two per row; elements 2^26 below its largest to what that leaves), p s to 11 bits, and with fp32 activations both as the sum of two such numbers
// (22 bits).  The values' steps say by what power of two p is held, so that p s keeps its bits far below the largest p and however small the values are.
// A matrix instruction drops what lies 2^-26 below its largest term, its addend among them.  With fp32 activations the two parts and the records are therefore added
// up outside, and codes are taken as c - 8 about m + 8 s, which leaves less to cancel between the two sums.  The softmax keeps a running maximum
// and sum; the maximum moves only when a score passes it by 2 in log2, so that most records rescale nothing (p <= 4).
//
// 32 sequences of 32768 tokens, 64 heads on 8 of 128: 145 us, 5.3 TB/s (a large copy: 4.8).  A token at 515, 32 heads of 128: 8.4 us, of which the way to the first
// record (lengths, pages and queries, the record itself) takes 3 and the launch as much.  16 sequences of up to 4096, 64 heads on 8: 17.7 us for 44 MB.
#include "kv_work.h"

#include <algorithm>
#include <cmath>

namespace eqat {
namespace {

constexpr int waves_of(int head_dim) { return head_dim > 128 ? 4 : 8; }         // of a workgroup, one on each compute unit (heads of 256 take 250 to 490 registers: one wave a SIMD)
constexpr int kRowsOfUnit = 16;                    // rows (query, head of the group) of a unit
constexpr int kFewestRecords = 32;                 // of a share: a join with another workgroup costs about as much (one token at 515: 32 8.4 us, 16 9.7, 8 9.5)
constexpr int kFewParts = 4;                       // parts of a unit that are fetched together
constexpr int kResident = 256;                     // compute units
constexpr int workgroups_of(int head_dim, int groups, bool bf16) { return head_dim == 64 && (bf16 || groups == 1) ? 2 : 1; }          // that registers and LDS of a compute unit hold
// Records of a wave's ring.  Heads of 256: 2 and 3 are alike (32 sequences of 16000, 8 heads, one group 189 and 191 us, groups of 32 271 and 267; one of 515 13.6 and 13.8).
constexpr int depth_of(int head_dim) { return head_dim > 128 ? 2 : 3; }

// f16(a * s.lo), f16(b * t.lo) in the halves of a register, s, t words whose low half is a binary16 number: the form that the compiler makes v_fma_mixlo_f16 and
// v_fma_mixhi_f16 of, with the wait states that those owe
__device__ __forceinline__ uint32_t scaled_pair(float a, uint32_t s, float b, uint32_t t)
{
    const half2v r = {(_Float16)__builtin_fmaf(a, (float)__builtin_bit_cast(half2v, s)[0], 0.0f), (_Float16)__builtin_fmaf(b, (float)__builtin_bit_cast(half2v, t)[0], 0.0f)};
    return __builtin_bit_cast(uint32_t, r);
}
// Two codes of a word (kv.h) as binary16: products 0 .. 3 of a value chunk, or the four pairs of a key word.
// CENTRED (fp32): c - 8, times 16 in the odd pairs: 1024 + c or 1024 + 16 c by the bits, less 1032 or 1152.  Else c 2^-24 or c 2^-20, as the bits are.
template <bool CENTRED> __device__ __forceinline__ uint32_t pick(uint32_t w, int p)
{
    const uint32_t c = (p >= 2 ? w >> 8 : w) & (p & 1 ? 0x00F000F0u : 0x000F000Fu);
    if constexpr (!CENTRED) return c;
    const _Float16 off = p & 1 ? -1152.0f : -1032.0f;
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, c | 0x64006400u) + half2v{off, off});
}
template <bool CENTRED> __device__ __forceinline__ float middle(uint32_t step)          // what a code of 0 stands for
{
    return CENTRED ? __builtin_fmaf(8.0f, low_half(step), high_half(step)) : high_half(step);
}
template <int NS, int SG, bool F32> __global__ __launch_bounds__(waves_of(32 * NS) * 64, workgroups_of(32 * NS, NS / SG, !F32) * waves_of(32 * NS) / 4) void k_kv_attend(const AttendArgs a)
{
    using R = KvRecord<NS, SG>;
    using T = typename std::conditional<F32, float, bf16_t>::type;
    constexpr int D = R::D, G = R::G, kChunks = NS / 2, kPad = D + 4, kWaves = waves_of(D), kDepth = depth_of(D), kStepLoads = (G + 3) / 4, kLoads = 2 * kChunks + kStepLoads, kStepWords = (G + 1) / 2;
    constexpr float kUnit = F32 ? 1.0f : 0x1p24f;          // what a code's binary16 form is divided by
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];              // the waves' rings; then the waves' sums [wave][row][kPad]
    __shared__ float s_ml[kWaves][kRowsOfUnit][2];
    __shared__ uint32_t s_last;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int head = blockIdx.x % a.heads, slot = blockIdx.x / a.heads;
    uint8_t *ring = lds + wave * kDepth * R::kBytes;
    const uint32_t ring_at = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_addr_of(ring));
    const Lane sequences = lane_of(a, 0);
    const Share mine = share_of(a, slot, sequences);
    Segment w{};
    for (int at = mine.first; at < mine.last; at = w.to) {
        w = segment_of(a, mine, at, sequences);
        if (!w.any) return;
        if (w.to <= w.unit_from) continue;                        // the unit's records are the next workgroup's
        // ---- this lane's row of the queries -----------------------------------------------------------
        const int row = w.unit * kRowsOfUnit + r, query = quotient(row, a.ratio), of_group = row - query * a.ratio;
        const bool is_row = query < w.s.n;
        const int pos = w.s.pos + query;
        const int seen_to = is_row && a.causal ? min(w.s.len, pos + 1) : w.s.len;             // positions seen_from .. seen_to - 1 (a row that is none restricts nothing)
        const int seen_from = is_row ? window_from(pos, a.window) : 0;
        // Records w.rec + wave, + kWaves, ...: lane i looks up the number in the pool of the i-th of 64 of them (-1: its page is not there).  Without a branch: lanes past the
        // last record read beyond the table's buffer.
        const __amdgpu_buffer_rsrc_t table = make_rsrc(a.b.table + (int64_t)w.b * a.b.table_stride, (uint32_t)min(a.b.table_stride, 1 << 28) * 4u);
        int numbers = -1;
        auto look_up = [&](int from) {
            const int rec = from + lane * kWaves, of_seq = quotient(rec, a.page_records);
            const bool is = rec < w.rec_to;
            const int page = __builtin_amdgcn_raw_buffer_load_b32(table, is ? of_seq * 4 : (int)kOobOffset, 0, 0);
            numbers = (is & (page >= 0) & (page < (int)a.pages)) ? (page * a.heads + head) * a.page_records + (rec - of_seq * a.page_records) : -1;
        };
        const int first_rec = w.rec + wave, records = max(0, (w.rec_to - first_rec + kWaves - 1) / kWaves);
        look_up(first_rec);
        T loaded[NS][8];
        {
            // (a row that is none has one of the last query's)
            const T *q = static_cast<const T *>(a.q.p) + (int64_t)(w.s.first + min(query, w.s.n - 1)) * a.q.token_stride + (int64_t)(head * a.ratio + of_group) * a.q.head_stride;
#pragma unroll
            for (int j = 0; j < NS; ++j) __builtin_memcpy(loaded[j], __builtin_assume_aligned(q + 32 * j + 8 * c, 16), sizeof(loaded[j]));
        }
        // The i-th record of this wave into the ring.  The loads are assembly, so nothing but the waits below counts them; a record that is not there is fetched from
        // the pool's first bytes and not looked at, so that every record counts as many.
        uint64_t gone = 0;                                     // bit i & 63: the i-th record is not there
        auto fetch = [&](int i) {
            if (i > 0 && (i & 63) == 0) look_up(first_rec + i * kWaves);
            const int number = __builtin_amdgcn_readlane(numbers, i & 63);
            gone = number < 0 ? gone | (uint64_t)1 << (i & 63) : gone & ~((uint64_t)1 << (i & 63));
            const RawRsrc src = make_raw_rsrc(a.pool + (int64_t)max(number, 0) * R::kBytes, R::kBytes);
            const uint32_t to = ring_at + (uint32_t)(i % kDepth) * R::kBytes;
#pragma unroll
            for (int k = 0; k < 2 * kChunks; ++k) load_to_lds16_at(src, to + k * 1024, (uint32_t)(k * 1024 + lane * 16));
#pragma unroll
            for (int k = 0; k < kStepLoads; ++k)
                if (G >= 4 || lane < 16 * G) load_to_lds16_at(src, to + R::kKeySteps + k * 1024, (uint32_t)(R::kKeySteps + k * 1024 + lane * 16));
        };
        // the queries' loads and the look-up are complete before the first record's are issued: a wait for them would wait for those too
        __builtin_amdgcn_s_waitcnt(0x0F70);
#pragma unroll
        for (int i = 0; i < kDepth - 1; ++i) if (i < records) fetch(i);
        half8 qh[NS], ql[F32 ? NS : 1];
        float sums[G], k_scale;
        {
            float x[NS][8], top = 0.0f;
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) { x[j][e] = (float)loaded[j][e]; top = fmaxf(top, fabsf(x[j][e])); }
            // the row scaled by a power of two to a largest element in [2^13, 2^14): code products are sums of q c 2^-24 or, for the pairs in bits 4 - 7, of (q 2^-4) c 2^-20
            top = chunks_max(top);
            const int up = min(140 - (int)(__float_as_uint(top) >> 23), 126);
            const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] *= scale;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < SG; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s += x[g * SG + j][e];
                sums[g] = chunks_sum(s) * (1.0f / kUnit);
            }
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = x[j][e], f = (e >> 1) & 1 ? 0x1p-4f : 1.0f;
                    const _Float16 h = (_Float16)(y * f);
                    qh[j][e] = h;
                    if constexpr (F32) ql[j][e] = (_Float16)(y * f - (float)h);
                }
            // The scale of the scores, all powers of two taken back, as a normal binary32 number.  Beyond 2^126 a row has one key, or some that are alike, whatever the power:
            // what is left off here comes back with the maximum.  Below 2^-126 all scores are nothing, but a hidden one has to stay -inf.
            const int back = (F32 ? 0 : 24) - up, lowered = max(a.scale_exponent + back - 126, 0);
            k_scale = fmaxf(__builtin_amdgcn_ldexpf(a.scale, back - lowered), 0x1p-126f);
            s_ml[wave][r][0] = __builtin_amdgcn_ldexpf(1.0f, lowered);
        }
        // ---- the records of this wave -----------------------------------------------------------------
        floatx4 o[2 * NS];
        // Running maximum (rounded up to a whole number, so that powers of two are exact), what scores have taken off them, sum of p, sum of p m.  p is held times 2^bias, and so
        // are the sums: the largest value step so far is below 2^(13 - bias), so p s (p at most 4) stays in binary16, and one that lies 2^25 below the largest is normal there.
        float top = -3.0e38f, off = top, total = 0.0f, even[G];
        int bias = 0;
        uint32_t steps_to = 0;                                  // the last binary16 number, as bits, that `bias` was made for
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) o[n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int g = 0; g < G; ++g) even[g] = 0.0f;
        // a maximum of 2^22 and more has no room for a bias in binary32: p s stays in binary16 without
        auto settle = [&](float next) {
            const float next_off = fabsf(next) < 4194304.0f ? next - (float)bias : next, down = exp2_of(off - next_off);
            top = next; off = next_off;
            total *= down;
#pragma unroll
            for (int g = 0; g < G; ++g) even[g] *= down;
#pragma unroll
            for (int n = 0; n < 2 * NS; ++n) o[n] *= down;
        };
        // records that every row of the unit sees in full need no mask
        int all_from = seen_from, all_to = seen_to;
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) { all_from = max(all_from, __shfl_xor(all_from, d)); all_to = min(all_to, __shfl_xor(all_to, d)); }
        all_from = __builtin_amdgcn_readfirstlane(all_from); all_to = __builtin_amdgcn_readfirstlane(all_to);
        // what some row sees: from the first row's beginning to the last one's end
        const int any_from = __builtin_amdgcn_readfirstlane(seen_from), any_to = __builtin_amdgcn_readlane(seen_to, min(kRowsOfUnit, w.s.n * a.ratio - w.unit * kRowsOfUnit) - 1);

        for (int i = 0; i < records; ++i) {
            const int rec = first_rec + i * kWaves;
            if (i + kDepth - 1 < records) {
                __builtin_amdgcn_s_waitcnt(0xC07F);               // the reads of the record before this one, into whose place goes
                fetch(i + kDepth - 1);
                __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0((kDepth - 1) * kLoads));
            } else {
                __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
            }
            asm volatile("" ::: "memory");
            if (gone >> (i & 63) & 1) continue;
            const uint8_t *at = ring + (i % kDepth) * R::kBytes;
            const bool edge = rec * kKvRecord < all_from || (rec + 1) * kKvRecord > all_to;
            // the values' steps, each in one lane (NaN is above every number)
            auto step = [&](int k) { return (uint32_t)*reinterpret_cast<const uint16_t *>(at + R::kValueSteps + k * 256 + (lane & (G > 1 ? 63 : 31)) * 4); };
            uint32_t steps = 0;
#pragma unroll
            for (int k = 0; k < kStepWords; ++k) steps = max(steps, step(k));
            uintx4 kc[kChunks], vc[kChunks], ks[G][2], vs[G][2];
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                kc[k] = *reinterpret_cast<const uintx4 *>(at + R::kKeys + k * 1024 + lane * 16);
                vc[k] = *reinterpret_cast<const uintx4 *>(at + R::kValues + k * 1024 + lane * 16);
            }
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    ks[g][h] = *reinterpret_cast<const uintx4 *>(at + R::kKeySteps + g * 128 + h * 64 + c * 16);
                    vs[g][h] = *reinterpret_cast<const uintx4 *>(at + R::kValueSteps + g * 128 + h * 64 + c * 16);
                }
            if (__any(steps > steps_to)) {
                // of those that are numbers and that some row sees
                const int t = rec * kKvRecord + (lane & 31);
                uint32_t big = 0;
#pragma unroll
                for (int k = 0; k < kStepWords; ++k) { const uint32_t u = step(k); big = max(big, u < 0x7C00u ? u : 0u); }
                big = lanes_greatest(t >= any_from && t < any_to ? big : 0u);
                if (big > steps_to) {
                    steps_to = big < 0x400u ? 0xFFFFFFFFu >> __builtin_clz(big) : big | 0x3FFu;
                    bias = 139 - (int)(__float_as_uint(low_half(big)) >> 23);
                    settle(top);
                }
            }
            float s[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f}, low = acc;
#pragma unroll
                    for (int j = g * SG; j < (g + 1) * SG; ++j) {
                        const uint32_t word = kc[(h * NS + j) >> 2][(h * NS + j) & 3];
                        uintx4 codes;
#pragma unroll
                        for (int p = 0; p < 4; ++p) codes[p] = pick<F32>(word, p);
                        acc = mfma(codes, qh[j], acc);
                        if constexpr (F32) low = mfma(codes, ql[j], low);
                    }
                    if constexpr (F32) acc += low;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float t = __builtin_fmaf(middle<F32>(ks[g][h][i]), sums[g], g == 0 ? 0.0f : s[h][i]);
                        s[h][i] = __builtin_fmaf(low_half(ks[g][h][i]), acc[i], t);
                    }
                }
            if (edge) {
                // what a row does not see must not reach it, NaN among it: neither its score nor, by way of 0 * NaN, its value
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = rec * kKvRecord + h * 16 + c * 4 + i;
                        const bool seen = t >= seen_from && t < seen_to;
                        s[h][i] = seen ? s[h][i] : -__builtin_inff();
#pragma unroll
                        for (int g = 0; g < G; ++g) vs[g][h][i] = seen ? vs[g][h][i] : 0u;
                    }
            }
            // (rounded before the maximum is taken off: what one rounding of both would leave of large scores is no small number)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[h][i] *= k_scale;
            float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            most = chunks_max(most);
            if (__any(most > top + 2.0f)) settle(fmaxf(top, __builtin_ceilf(most)));
            float p[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[h][i] = exp2_of(s[h][i] - off);
                    total += p[h][i];
                }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uintx4 ph, pl;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) even[g] = __builtin_fmaf(middle<F32>(vs[g][h][i]), p[h][i], even[g]);
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        if constexpr (F32) {
                            float x = p[h][i] * low_half(vs[g][h][i]), y = p[h][i + 1] * low_half(vs[g][h][i + 1]);
                            asm("" : "+v"(x), "+v"(y));          // both uses below round the binary32 product (a mixed-precision product rounds once, and not to the same number)
                            const half2v hi = {(_Float16)x, (_Float16)y}, lo = {(_Float16)((x - (float)hi[0]) * 0x1p11f), (_Float16)((y - (float)hi[1]) * 0x1p11f)};
                            ph[h * 2 + i / 2] = __builtin_bit_cast(uint32_t, hi);
                            pl[h * 2 + i / 2] = __builtin_bit_cast(uint32_t, lo);
                        } else {
                            ph[h * 2 + i / 2] = scaled_pair(p[h][i], vs[g][h][i], p[h][i + 1], vs[g][h][i + 1]);
                        }
                    }
                }
#pragma unroll
                for (int n = 2 * g * SG; n < 2 * (g + 1) * SG; ++n) {
                    uintx4 codes;
#pragma unroll
                    for (int q = 0; q < 4; ++q) codes[q] = pick<F32>(vc[n >> 2][q], n & 3);
                    if constexpr (F32) {
                        const floatx4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                        const floatx4 low = mfma(codes, __builtin_bit_cast(half8, pl), zero), down = {0x1p-11f, 0x1p-11f, 0x1p-11f, 0x1p-11f};
                        o[n] += __builtin_elementwise_fma(low, down, mfma(codes, __builtin_bit_cast(half8, ph), zero));
                    } else {
                        o[n] = mfma(codes, __builtin_bit_cast(half8, ph), o[n]);
                    }
                }
            }
            asm volatile("" ::: "memory");
        }
        // ---- the waves' sums joined ---------------------------------------------------------------------
        float (*s_o)[kRowsOfUnit][kPad] = reinterpret_cast<float (*)[kRowsOfUnit][kPad]>(lds);
        __syncthreads();                                          // the rings have been read
        const float unit = exp2_of(off - top);                    // 2^-bias
        total = chunks_sum(total) * unit;
#pragma unroll
        for (int g = 0; g < G; ++g) even[g] = chunks_sum(even[g]) * unit;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            // products 2 j and 2 j + 1: elements 32 j + 8 c + 0 .. 7
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int n = 2 * j + (i & 1);
                x[i] = __builtin_fmaf(o[n][i >> 1], (n & 1 ? kUnit / 16.0f : kUnit) * unit, even[j / SG]);
            }
            *reinterpret_cast<floatx4 *>(&s_o[wave][r][32 * j + 8 * c]) = floatx4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<floatx4 *>(&s_o[wave][r][32 * j + 8 * c + 4]) = floatx4{x[4], x[5], x[6], x[7]};
        }
        if (c == 0) { s_ml[wave][r][0] = fmaxf(top * s_ml[wave][r][0], -3.0e38f); s_ml[wave][r][1] = total; }
        __syncthreads();
        constexpr int kOut = kWaves == 8 && D == 128 ? 4 : D / 16, kOfRow = D / kOut;      // elements of a row that a thread takes, threads of a row
        const bool joins = tid < kRowsOfUnit * kOfRow;
        const int orow = joins ? tid / kOfRow : 0, d0 = (tid % kOfRow) * kOut;
        float m = s_ml[0][orow][0], l = 0.0f, x[kOut] = {};
#pragma unroll
        for (int i = 1; i < kWaves; ++i) m = fmaxf(m, s_ml[i][orow][0]);
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const float f = exp2_of(s_ml[i][orow][0] - m);
            l = __builtin_fmaf(s_ml[i][orow][1], f, l);
#pragma unroll
            for (int e = 0; e < kOut; ++e) x[e] = __builtin_fmaf(s_o[i][orow][d0 + e], f, x[e]);
        }
        const bool whole = w.unit_from >= mine.first && w.unit_to <= mine.last;
        bool answers = true;
        if (!whole) {
            // Parts and counter are written and read at device scope (the workgroups sit on different XCDs): every wave waits for its stores, the workgroup meets, one
            // lane counts it in, and the last to arrive adds up all parts in their order.  A workgroup has at most two parts: of the unit that it finds begun, and of the one
            // that it leaves unfinished.
            constexpr uint32_t kPart = kRowsOfUnit * D * 4, kStats = kRowsOfUnit * 8;
            uint8_t *base = reinterpret_cast<uint8_t *>(a.parts), *stats = base + 2 * (int64_t)a.slots * a.heads * kPart;
            const int from = w.unit_from / mine.size, arrivals = (w.unit_to - 1) / mine.size - from + 1;
            auto part = [&](int k) { return ((int64_t)(from + k) * 2 + (k == 0 ? 1 : 0)) * a.heads + head; };          // of the k-th workgroup of the unit
            {
                const int64_t to = part(slot - from);
                const __amdgpu_buffer_rsrc_t dst = make_rsrc(base + to * kPart, kPart), st = make_rsrc(stats + to * kStats, kStats);
#pragma unroll
                for (int e = 0; e < kOut; e += 4) {
                    if (!joins) break;
                    const intx4 v = {__float_as_int(x[e]), __float_as_int(x[e + 1]), __float_as_int(x[e + 2]), __float_as_int(x[e + 3])};
                    __builtin_amdgcn_raw_buffer_store_b128(v, dst, (orow * D + d0 + e) * 4, 0, kAuxDeviceScope);
                }
                const intx2 v = {__float_as_int(m), __float_as_int(l)};
                if (joins && d0 == 0) __builtin_amdgcn_raw_buffer_store_b64(v, st, orow * 8, 0, kAuxDeviceScope);
            }
            wait_all_and_barrier();
            uint32_t *counter = a.counters + (int64_t)from * a.heads + head;
            if (tid == 0) {
                const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = before == (uint32_t)(arrivals - 1) ? 1u : 0u;
                if (s_last != 0u) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            answers = s_last != 0u;
            if (answers) {
                m = -3.0e38f; l = 0.0f;
#pragma unroll
                for (int e = 0; e < kOut; ++e) x[e] = 0.0f;
                for (int k0 = 0; k0 < arrivals; k0 += kFewParts) {
                    intx2 ml[kFewParts];
                    intx4 v[kFewParts][kOut / 4];
#pragma unroll
                    for (int k = 0; k < kFewParts; ++k) {                // past the last part: an empty buffer, zeros
                        const bool is = k0 + k < arrivals;
                        const int64_t of = part(is ? k0 + k : 0);
                        const __amdgpu_buffer_rsrc_t src = make_rsrc(base + of * kPart, is ? kPart : 0u), st = make_rsrc(stats + of * kStats, is ? kStats : 0u);
                        ml[k] = __builtin_amdgcn_raw_buffer_load_b64(st, orow * 8, 0, kAuxDeviceScope);
#pragma unroll
                        for (int e = 0; e < kOut; e += 4) v[k][e / 4] = __builtin_amdgcn_raw_buffer_load_b128(src, (orow * D + d0 + e) * 4, 0, kAuxDeviceScope);
                    }
#pragma unroll
                    for (int k = 0; k < kFewParts; ++k) {
                        const float other = k0 + k < arrivals ? __int_as_float(ml[k][0]) : -3.0e38f;
                        const float next = fmaxf(m, other), f = exp2_of(m - next), g = exp2_of(other - next);
                        m = next;
                        l = __builtin_fmaf(__int_as_float(ml[k][1]), g, l * f);
#pragma unroll
                        for (int e = 0; e < kOut; ++e) x[e] = __builtin_fmaf(__int_as_float(v[k][e / 4][e % 4]), g, x[e] * f);
                    }
                }
            }
        }
        const int orow_all = w.unit * kRowsOfUnit + orow, oquery = quotient(orow_all, a.ratio), oh = head * a.ratio + (orow_all - oquery * a.ratio);
        if (answers && joins && oquery < w.s.n) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;        // a row that sees nothing: zeros
            T *out = static_cast<T *>(a.out.p) + (int64_t)(w.s.first + oquery) * a.out.token_stride + (int64_t)oh * a.out.head_stride + d0;
#pragma unroll
            for (int e = 0; e < kOut; e += 4) {
                if constexpr (F32) {
                    *reinterpret_cast<floatx4 *>(out + e) = floatx4{x[e] * inv, x[e + 1] * inv, x[e + 2] * inv, x[e + 3] * inv};
                } else {
                    bf16x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (bf16_t)(x[e + i] * inv);
                    *reinterpret_cast<bf16x4 *>(out + e) = v;
                }
            }
            if (a.lse != nullptr && d0 == 0)
                a.lse[(int64_t)(w.s.first + oquery) * ((int64_t)a.heads * a.ratio) + oh] = l == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(l)) * 0.6931471805599453f;
        }
        __syncthreads();                                          // the sums have been read: the rings may fill again
    }
}

// Shares of the work of a head of the cache: no more workgroups than are resident (a second round of a few took as long as the first: 40 heads, 16 sequences of 8000
// 126 us, with 7 shares a head for 6 198), and two a compute unit only where that leaves shares of 64 records (heads of 64 on 40, 8 sequences of 8000 46 us one, 42 two;
// 32 in fp32, 32 sequences of 2000 60 and 51; on 8, where it leaves 31, 15.3 and 17.2).
int most_shares_of(const KvShape &s, int workgroups) { return std::max(1, workgroups * kResident / s.heads); }
int shares_of(const KvShape &s, const KvBatch &b, int ratio)
{
    const int workgroups = workgroups_of(s.head_dim, s.groups, s.act_bf16);
    const bool large = (double)units_at_most(b, ratio, kRowsOfUnit) * s.heads * (b.max_len / 32) >= 64.0 * workgroups * kResident;
    return most_shares_of(s, large ? workgroups : 1);
}

// Sequences of more rows than this go to the kernel that rebuilds keys and values (bf16): for 64 rows this one takes 14.6 us and that one 26 (8000 tokens, 8 heads of
// the cache), 8.7 and 16.8 us (500 tokens).
constexpr int kStreamedRows = 64;
// Where a call's units of 16 rows are no more than two for every compute unit, and its caches long, no sequence does: 256 rows of four sequences at 2100 tokens 28 us and 38,
// 800 rows at 4000 42 and 48, but 2700 rows at 333 tokens 37 and 18.5.
bool has_prompts(const KvShape &s, const KvBatch &b, int ratio)
{
    if (!s.act_bf16 || (int64_t)b.max_new * ratio <= kStreamedRows) return false;
    const int units = units_at_most(b, ratio, kRowsOfUnit);
    return b.max_len < 2048 || (int64_t)units * s.heads > 2 * kResident || units * (b.max_len / 32 + 1.0 + kKvBeginning) > kKvMostPlaces;
}

// The workspace does not depend on which kernels a batch takes: what serves a batch serves every smaller one.
struct WsLayout { Scratch streamed, prompts; };
WsLayout ws_layout(const KvShape &s, const KvBatch &b, int ratio)
{
    WsLayout l;
    l.streamed = scratch_of(0, (size_t)most_shares_of(s, workgroups_of(s.head_dim, s.groups, s.act_bf16)) * s.heads, true, kRowsOfUnit, s.head_dim);
    l.prompts = Scratch{l.streamed.end, l.streamed.end, l.streamed.end};
    if (s.act_bf16 && (int64_t)b.max_new * ratio > kStreamedRows) l.prompts = prompt_scratch(s, (l.streamed.end + 255) / 256 * 256);
    return l;
}

template <int NS, int SG, bool F32> void launch_t(const AttendArgs &a, hipStream_t st)
{
    constexpr int D = 32 * NS, kWaves = waves_of(D), rings = kWaves * depth_of(D) * KvRecord<NS, SG>::kBytes, sums = kWaves * kRowsOfUnit * (D + 4) * 4, smem = rings > sums ? rings : sums;
    static std::atomic<uint64_t> asked{0};
    allow_lds(asked, reinterpret_cast<const void *>(&k_kv_attend<NS, SG, F32>), smem);
    k_kv_attend<NS, SG, F32><<<dim3((unsigned)a.slots * (unsigned)a.heads), kWaves * 64, smem, st>>>(a);
}
template <int NS, int SG> void launch(const KvShape &s, const AttendArgs &a, hipStream_t st)
{
    if (s.act_bf16) launch_t<NS, SG, false>(a, st);
    else launch_t<NS, SG, true>(a, st);
}

}  // namespace

size_t kv_attend_ws_bytes(const KvShape &s, const KvBatch &b, int q_heads) { return ws_layout(s, b, q_heads / s.heads).prompts.end; }

void launch_kv_attend(const KvShape &s, const KvBatch &b, const KvAttend &t, const void *pool, void *ws, hipStream_t st)
{
    const WsLayout l = ws_layout(s, b, t.q_heads / s.heads);
    AttendArgs a;
    a.b = b; a.q = t.q; a.out = t.out; a.lse = t.lse;
    a.pool = static_cast<const uint8_t *>(pool);
    a.pages = s.pages; a.heads = s.heads; a.ratio = t.q_heads / s.heads; a.page_records = s.page_records; a.window = t.window; a.causal = t.causal;
    a.scale = t.scale * 1.4426950408889634f;
    a.scale_exponent = std::ilogb(a.scale);
    auto scratch = [&](const Scratch &x) {
        a.counters = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(ws) + x.counters);
        a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + x.parts);
    };
    const bool prompts = has_prompts(s, b, a.ratio);
    if (prompts) {
        // Where all sequences have as many new tokens as any may, one launch takes them all, and so it does where the arrays have changed since and some have fewer.
        const bool all = b.tokens == (int64_t)b.sequences * b.max_new;
        a.from_rows = all ? 1 : kStreamedRows + 1; a.to_rows = INT32_MAX;
        scratch(l.prompts);
        launch_kv_prompt(s, a, st);
        if (all) return;
    }
    a.from_rows = 1; a.to_rows = prompts ? kStreamedRows + 1 : INT32_MAX;
    scratch(l.streamed);
    a.unit_bits = __builtin_ctz(kRowsOfUnit);
    a.fewest = kFewestRecords;
    a.slots = shares_of(s, b, a.ratio);
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(s, a, st); else launch<2, 2>(s, a, st); break;
    case 128: if (sg == 1) launch<4, 1>(s, a, st); else if (sg == 2) launch<4, 2>(s, a, st); else launch<4, 4>(s, a, st); break;
    default:
        if (sg == 1) launch<8, 1>(s, a, st); else if (sg == 2) launch<8, 2>(s, a, st); else if (sg == 4) launch<8, 4>(s, a, st); else launch<8, 8>(s, a, st);
    }
}

}  // namespace eqat
