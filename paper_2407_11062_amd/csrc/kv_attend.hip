// Attention over the 4-bit cache, streamed: every wave takes whole records of 32 tokens straight from memory into registers, for up to 16 rows (query, head) that
// share a head of the cache.
//
// With x^ = m + s c (kv.h) the sums over elements and tokens part into sums over codes, which are exact in binary16, and sums over the steps:
//   q . k^_t   = sum over groups g of  s_tg (q_g . c_tg) + m_tg sum(q_g)
//   sum_t p_t v^_td = sum_t (p_t s_tg) c_td  +  sum_t p_t m_tg
// The products with codes run on the matrix cores, everything else in binary32; no key or value is ever rebuilt.  q and p s are binary16 there: q of bf16 exactly
// (scaled by a power of two per row), p s to 11 bits, and with fp32 activations both as the sum of two such numbers (22 bits).
// A matrix instruction drops what lies 2^-26 below its largest term, its addend among them.  With fp32 activations the two parts and the records are therefore added
// up outside, and codes are taken as c - 8 about m + 8 s, which leaves less to cancel between the two sums.  The softmax keeps a running maximum
// and sum; the maximum moves only when a score passes it by 2 in log2, so that most records rescale nothing (p <= 4, and s < 2^14, so p s stays in binary16).
#include "kv_work.h"

namespace eqat {
namespace {

constexpr int kWaves = 4;
constexpr int kRowsOfUnit = 16;                    // rows (query, head of the group) of a unit
constexpr int kWorkgroups = 1024;                  // what the division of the work aims at: four workgroups on each of 256 compute units
constexpr int kFewestRecords = 2 * kWaves;         // of a chunk

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
template <int NS, int SG, bool F32> __global__ __launch_bounds__(kWaves * 64) void k_kv_attend(const AttendArgs a)
{
    using R = KvRecord<NS, SG>;
    using T = typename std::conditional<F32, float, bf16_t>::type;
    constexpr int D = R::D, G = R::G, kChunks = NS / 2, kPad = D + 4;
    constexpr float kUnit = F32 ? 1.0f : 0x1p24f;          // what a code's binary16 form is divided by
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int head = blockIdx.x % a.heads;
    const Work w = work_of(a, blockIdx.x / a.heads);
    if (!w.any) return;
    // ---- this lane's row of the queries -----------------------------------------------------------
    const int row = w.unit * kRowsOfUnit + r, query = row / a.ratio, of_group = row - query * a.ratio;
    const bool is_row = query < w.s.n;
    const int pos = w.s.len - w.s.n + query;
    const int seen_to = is_row && a.causal ? min(w.s.len, pos + 1) : w.s.len;             // positions seen_from .. seen_to - 1 (a row that is none restricts nothing)
    const int seen_from = is_row && a.window > 0 ? max(0, pos - a.window + 1) : 0;
    half8 qh[NS], ql[F32 ? NS : 1];
    float sums[G], k_scale;
    {
        const T *q = static_cast<const T *>(a.q.p) + (int64_t)(w.s.first + query) * a.q.token_stride + (int64_t)(head * a.ratio + of_group) * a.q.head_stride;
        float x[NS][8], top = 0.0f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[j][e] = 0.0f;
            if (is_row) {
                if constexpr (F32) {
                    const floatx4 u = *reinterpret_cast<const floatx4 *>(q + 32 * j + 8 * c), v = *reinterpret_cast<const floatx4 *>(q + 32 * j + 8 * c + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { x[j][e] = u[e]; x[j][4 + e] = v[e]; }
                } else {
                    const bf16x8 u = *reinterpret_cast<const bf16x8 *>(q + 32 * j + 8 * c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[j][e] = (float)u[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
        }
        // the row scaled by a power of two to a largest element in [2^13, 2^14): code products are sums of q c 2^-24 or, for the pairs in bits 4 - 7, of (q 2^-4) c 2^-20
        top = chunks_max(top);
        const int up = min(max(140 - (int)(__float_as_uint(top) >> 23), -100), 100);
        const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < SG; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += x[g * SG + j][e];
            sums[g] = chunks_sum(s) * scale * (1.0f / kUnit);
        }
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[j][e] * scale, f = (e >> 1) & 1 ? 0x1p-4f : 1.0f;
                const _Float16 h = (_Float16)(y * f);
                qh[j][e] = h;
                if constexpr (F32) ql[j][e] = (_Float16)(y * f - (float)h);
            }
        k_scale = a.scale * __uint_as_float((uint32_t)(127 - up) << 23) * kUnit;
    }
    // ---- the records of this wave -----------------------------------------------------------------
    floatx4 o[2 * NS];
    float top = -3.0e38f, total = 0.0f, even[G];            // running maximum, sum of p, sum of p m
    float v_scale = 1.0f;                                   // fp32: what the accumulators are scaled by
#pragma unroll
    for (int n = 0; n < 2 * NS; ++n) o[n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < G; ++g) even[g] = 0.0f;
    // records that every row of the unit sees in full need no mask
    int all_from = seen_from, all_to = seen_to;
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) { all_from = max(all_from, __shfl_xor(all_from, d)); all_to = min(all_to, __shfl_xor(all_to, d)); }
    all_from = __builtin_amdgcn_readfirstlane(all_from); all_to = __builtin_amdgcn_readfirstlane(all_to);

    const int32_t *table = a.b.table + (int64_t)w.b * a.b.table_stride;
    for (int rec = w.first + wave; rec < w.last; rec += kWaves) {
        const int page_of_seq = rec / a.page_records, page = __builtin_amdgcn_readfirstlane(table[page_of_seq]);
        if (page < 0 || page >= a.pages) continue;           // not there
        const uint8_t *at = a.pool + (((int64_t)page * a.heads + head) * a.page_records + (rec - page_of_seq * a.page_records)) * R::kBytes;
        uintx4 kc[kChunks], vc[kChunks], ks[G][2], vs[G][2];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            kc[i] = *reinterpret_cast<const uintx4 *>(at + R::kKeys + i * 1024 + lane * 16);
            vc[i] = *reinterpret_cast<const uintx4 *>(at + R::kValues + i * 1024 + lane * 16);
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ks[g][h] = *reinterpret_cast<const uintx4 *>(at + R::kKeySteps + g * 128 + h * 64 + c * 16);
                vs[g][h] = *reinterpret_cast<const uintx4 *>(at + R::kValueSteps + g * 128 + h * 64 + c * 16);
            }
        const bool edge = rec * kKvRecord < all_from || (rec + 1) * kKvRecord > all_to;
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
        float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        most = chunks_max(most) * k_scale;
        if (__any(most > top + 2.0f)) {
            const float next = fmaxf(top, most), down = exp2_of(top - next);
            top = next;
            total *= down;
#pragma unroll
            for (int g = 0; g < G; ++g) even[g] *= down;
#pragma unroll
            for (int n = 0; n < 2 * NS; ++n) o[n] *= down;
        }
        float p[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[h][i] = exp2_of(__builtin_fmaf(s[h][i], k_scale, -top));
                total += p[h][i];
            }
        if constexpr (F32) {
            // two binary16 numbers hold 22 bits of p s only where its low part does not run into denormals: values' steps are brought to about 2^11 by a power of two
            uint32_t big = 0;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) { const float v = low_half(vs[g][h][i]); big = max(big, v < 65536.0f ? __float_as_uint(v) : 0u); }
            if (edge) {                      // rows see different tokens
#pragma unroll
                for (int d = 8; d >= 1; d >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d));
            }
            const float most_step = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(chunks_max(__uint_as_float(big)))));
            if (most_step * v_scale >= 4096.0f || (v_scale == 1.0f && most_step > 0.0f)) {
                const float next = __uint_as_float((uint32_t)(127 + 138 - (int)(__float_as_uint(most_step) >> 23)) << 23);
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) o[n] *= next / v_scale;
                v_scale = next;
            }
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
                        float x = p[h][i] * v_scale * low_half(vs[g][h][i]), y = p[h][i + 1] * v_scale * low_half(vs[g][h][i + 1]);
                        asm("" : "+v"(x), "+v"(y));          // both uses below round the binary32 product (a mixed-precision product rounds once, and not to the same number)
                        const half2v hi = {(_Float16)x, (_Float16)y}, lo = {(_Float16)(x - (float)hi[0]), (_Float16)(y - (float)hi[1])};
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
                    o[n] += mfma(codes, __builtin_bit_cast(half8, ph), zero) + mfma(codes, __builtin_bit_cast(half8, pl), zero);
                } else {
                    o[n] = mfma(codes, __builtin_bit_cast(half8, ph), o[n]);
                }
            }
        }
    }
    // ---- the waves' sums joined ---------------------------------------------------------------------
    __shared__ __attribute__((aligned(16))) float s_o[kWaves][kRowsOfUnit][kPad];
    __shared__ float s_ml[kWaves][kRowsOfUnit][2];
    total = chunks_sum(total);
#pragma unroll
    for (int g = 0; g < G; ++g) even[g] = chunks_sum(even[g]);
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        // products 2 j and 2 j + 1: elements 32 j + 8 c + 0 .. 7
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int n = 2 * j + (i & 1);
            x[i] = __builtin_fmaf(o[n][i >> 1], (n & 1 ? kUnit / 16.0f : kUnit) / v_scale, even[j / SG]);
        }
        *reinterpret_cast<floatx4 *>(&s_o[wave][r][32 * j + 8 * c]) = floatx4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<floatx4 *>(&s_o[wave][r][32 * j + 8 * c + 4]) = floatx4{x[4], x[5], x[6], x[7]};
    }
    if (c == 0) { s_ml[wave][r][0] = top; s_ml[wave][r][1] = total; }
    __syncthreads();
    constexpr int kOut = D / 16;                              // elements of a row that a thread takes
    const int orow = tid >> 4, d0 = (tid & 15) * kOut;
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
    if (w.chunks > 1) {
        // Parts and counter are written and read at device scope (the workgroups sit on different XCDs): every wave waits for its stores, the workgroup meets, one
        // lane counts it in, and the last to arrive adds up all parts in their order.
        __shared__ uint32_t s_last;
        constexpr uint32_t kPart = kRowsOfUnit * D * 4, kStats = kRowsOfUnit * 8;
        const int64_t parts = 2 * (int64_t)a.target * a.heads;
        uint8_t *base = reinterpret_cast<uint8_t *>(a.parts), *stats = base + parts * kPart;
        const int64_t mine = (int64_t)w.part * a.heads + head;
        {
            const __amdgpu_buffer_rsrc_t dst = make_rsrc(base + mine * kPart, kPart), st = make_rsrc(stats + mine * kStats, kStats);
#pragma unroll
            for (int e = 0; e < kOut; e += 4) {
                const intx4 v = {__float_as_int(x[e]), __float_as_int(x[e + 1]), __float_as_int(x[e + 2]), __float_as_int(x[e + 3])};
                __builtin_amdgcn_raw_buffer_store_b128(v, dst, (orow * D + d0 + e) * 4, 0, kAuxDeviceScope);
            }
            const intx2 v = {__float_as_int(m), __float_as_int(l)};
            if ((tid & 15) == 0) __builtin_amdgcn_raw_buffer_store_b64(v, st, orow * 8, 0, kAuxDeviceScope);
        }
        wait_all_and_barrier();
        uint32_t *counter = a.counters + (int64_t)w.counter * a.heads + head;
        if (tid == 0) {
            const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)(w.chunks - 1) ? 1u : 0u;
            if (s_last != 0u) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (s_last == 0u) return;
        m = -3.0e38f; l = 0.0f;
#pragma unroll
        for (int e = 0; e < kOut; ++e) x[e] = 0.0f;
        for (int k = 0; k < w.chunks; ++k) {
            const int64_t from = (int64_t)(w.part - w.chunk + k) * a.heads + head;
            const __amdgpu_buffer_rsrc_t src = make_rsrc(base + from * kPart, kPart), st = make_rsrc(stats + from * kStats, kStats);
            const intx2 ml = __builtin_amdgcn_raw_buffer_load_b64(st, orow * 8, 0, kAuxDeviceScope);
            intx4 v[kOut / 4];
#pragma unroll
            for (int e = 0; e < kOut; e += 4) v[e / 4] = __builtin_amdgcn_raw_buffer_load_b128(src, (orow * D + d0 + e) * 4, 0, kAuxDeviceScope);
            const float next = fmaxf(m, __int_as_float(ml[0])), f = exp2_of(m - next), g = exp2_of(__int_as_float(ml[0]) - next);
            m = next;
            l = __builtin_fmaf(__int_as_float(ml[1]), g, l * f);
#pragma unroll
            for (int e = 0; e < kOut; ++e) x[e] = __builtin_fmaf(__int_as_float(v[e / 4][e % 4]), g, x[e] * f);
        }
    }
    const int orow_all = w.unit * kRowsOfUnit + orow, oquery = orow_all / a.ratio, oh = head * a.ratio + (orow_all - oquery * a.ratio);
    if (oquery >= w.s.n) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;            // a row that sees nothing: zeros
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
    if (a.lse != nullptr && (tid & 15) == 0)
        a.lse[(int64_t)(w.s.first + oquery) * ((int64_t)a.heads * a.ratio) + oh] = l == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

// chunks that the division aims at, for every head of the cache
int chunks_aimed_at(const KvShape &s) { return (kWorkgroups + s.heads - 1) / s.heads; }

// Sequences with more rows than this go to the kernel that rebuilds keys and values (bf16).
constexpr int kStreamedRows = 64;

struct WsLayout { Scratch streamed, prompts; };
WsLayout ws_layout(const KvShape &s, const KvBatch &b, int q_heads)
{
    WsLayout l;
    l.streamed = scratch_of(0, chunks_aimed_at(s), s.heads, kRowsOfUnit, s.head_dim);
    l.prompts = Scratch{l.streamed.end, l.streamed.end, l.streamed.end};
    if (s.act_bf16 && (int64_t)b.max_new * (q_heads / s.heads) > kStreamedRows)
        l.prompts = scratch_of((l.streamed.end + 255) / 256 * 256, prompt_target(s), s.heads, prompt_unit_rows(s), s.head_dim);
    return l;
}

template <int NS, int SG> void launch(const KvShape &s, const AttendArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)a.slots * (unsigned)a.heads);
    if (s.act_bf16) k_kv_attend<NS, SG, false><<<grid, kWaves * 64, 0, st>>>(a);
    else k_kv_attend<NS, SG, true><<<grid, kWaves * 64, 0, st>>>(a);
}

}  // namespace

size_t kv_attend_ws_bytes(const KvShape &s, const KvBatch &b, int q_heads) { return ws_layout(s, b, q_heads).prompts.end; }

void launch_kv_attend(const KvShape &s, const KvBatch &b, const KvAttend &t, const void *pool, void *ws, hipStream_t st)
{
    const WsLayout l = ws_layout(s, b, t.q_heads);
    AttendArgs a;
    a.b = b; a.q = t.q; a.out = t.out; a.lse = t.lse;
    a.pool = static_cast<const uint8_t *>(pool);
    a.pages = s.pages; a.heads = s.heads; a.ratio = t.q_heads / s.heads; a.page_records = s.page_records; a.window = t.window; a.causal = t.causal;
    a.scale = t.scale * 1.4426950408889634f;
    auto scratch = [&](const Scratch &x) {
        a.counters = reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(ws) + x.counters);
        a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + x.parts);
    };
    const bool prompts = s.act_bf16 && (int64_t)b.max_new * a.ratio > kStreamedRows;
    if (prompts) {
        a.from_rows = kStreamedRows + 1; a.to_rows = INT32_MAX;
        scratch(l.prompts);
        launch_kv_prompt(s, a, st);
        if (b.tokens == (int64_t)b.sequences * b.max_new) return;        // all sequences have as many new tokens
    }
    a.from_rows = 1; a.to_rows = prompts ? kStreamedRows + 1 : INT32_MAX;
    scratch(l.streamed);
    a.unit_rows = kRowsOfUnit;
    a.fewest = kFewestRecords;
    a.target = chunks_aimed_at(s);
    KvBatch few = b;
    if (prompts) few.max_new = kStreamedRows / a.ratio;
    a.slots = a.target + units_at_most(few, a.ratio, kRowsOfUnit);
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(s, a, st); else launch<2, 2>(s, a, st); break;
    case 128: if (sg == 1) launch<4, 1>(s, a, st); else if (sg == 2) launch<4, 2>(s, a, st); else launch<4, 4>(s, a, st); break;
    default:
        if (sg == 1) launch<8, 1>(s, a, st); else if (sg == 2) launch<8, 2>(s, a, st); else if (sg == 4) launch<8, 4>(s, a, st); else launch<8, 8>(s, a, st);
    }
}

}  // namespace eqat
