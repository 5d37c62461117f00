// Writing keys and values into the 4-bit cache, and reading them back.
//
// Both move bytes: a token and head of 128 elements is 512 bytes of bf16 and 136 (one group) to 160 (four) in the cache.  A wave takes the keys or the values of a record of 32 tokens and one
// head, sixteen tokens at a time, four lanes to a token: lane c of them has the elements 32 j + 8 c .. + 7 of every j, which are one word of the cache each for a key, and for
// a value eight half words (kv.h says where they stand).  A lane then stores a key's words of four j as they lie, 16 neighbouring bytes, and a group's least and
// greatest element are found in a lane and two exchanges.  Half words of values go through LDS into the order of the record where all of it is written, and singly where not.
//
// 8192 tokens of 32 heads of 128, one group, bf16: a write takes 40 us for its 170 MB (4.2 TB/s), bound by arithmetic (18 instructions an element, 33 us of a SIMD's
// issue), a read 28 us (6.1 TB/s; a large copy 4.8).  A token of 32 heads: 4.3 and 3.6 us, the launch.  Half words in banks of their own, stored by LDS instructions
// rather than by flat ones: 42 and 29.
//
// eqat_kv_rotary_write is the same launch with the keys turned on their way in (rounded to the activations' type, as eqat_rotary leaves them, so that what is written is
// bitwise what the two calls write) and workgroups beside it that turn the queries.  A workgroup makes the cosines and sines of its record's tokens in LDS first.
// us of a graph's step, one launch / the two: 16 sequences, 64 heads on 8 of 128, 6.0 / 8.5; one token of 32 heads 5.7 / 7.8; 333 tokens of 32 heads 11.3 / 12.0; 8192 79 / 87; 8192 of 64 heads on 8
// 69 / 67; fp32, 4 x 2000 of 40 heads, 176 / 182.
#include "layer.h"
#include "turn.h"

#include <algorithm>

namespace eqat {
namespace {

constexpr int kCacheWaves = 4;

struct CacheArgs {
    KvBatch b;
    KvRows k, v;
    uint8_t *pool;
    int64_t pages;
    int heads, page_records;
};

// of the four lanes of a token; NaN wins (v_minimum3_f32, v_maximum3_f32)
__device__ __forceinline__ float greater(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float least_of(float a, float b) { return __builtin_elementwise_minimum(a, b); }
template <int CTRL> __device__ __forceinline__ float of_quad(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ float quad_greatest(float v) { v = greater(v, of_quad<0xB1>(v)); return greater(v, of_quad<0x4E>(v)); }
__device__ __forceinline__ float quad_least(float v) { v = least_of(v, of_quad<0xB1>(v)); return least_of(v, of_quad<0x4E>(v)); }

// A group's step and least element, as they stand in the cache: NaN where an element is not finite or beyond binary16 (so no step passes 131008 / 15, and what a kernel
// makes of codes and steps stays within binary16 or a rounding of it).
struct Step { float s, m; uint32_t word; };
__device__ __forceinline__ Step step_of(float least, float greatest)
{
    _Float16 m = (_Float16)least, s = (_Float16)fmaxf((greatest - least) / 15.0f, 0x1p-24f);
    if (!(fabsf((float)m) + fabsf((float)(_Float16)greatest) < __builtin_inff())) { m = (_Float16)__builtin_nanf(""); s = m; }
    Step r;
    r.s = (float)s; r.m = (float)m;
    r.word = (uint32_t)__builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
    return r;
}

// Codes round((x - m) / s) of a lane's eight elements, of the correctly rounded quotients, element e in bits sh(e).  A multiply-add that adds 1.5 2^23 rounds a product
// to a whole number; with the reciprocal of s once 2^-21 too small and once as much too large the two numbers bracket the quotient's, and where they are the same they
// are it.  Where any is not (ties and beside them) the lane divides.
template <typename SH> __device__ __forceinline__ uint32_t codes_of(const float *x, const Step &t, SH sh)
{
    constexpr float kWhole = 12582912.0f;
    const float r = __builtin_amdgcn_rcpf(t.s), below = r * (1.0f - 0x1p-21f), above = r * (1.0f + 0x1p-21f);
    uint32_t word = 0, whole = 0;
    bool unsure = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = x[e] - t.m, a = __builtin_fmaf(d, below, kWhole), b = __builtin_fmaf(d, above, kWhole);
        unsure |= !(a == b);
        word += __float_as_uint(__builtin_amdgcn_fmed3f(a, kWhole, kWhole + 15.0f)) << sh(e);
        whole += 0x4B400000u << sh(e);
    }
    word -= whole;
    if (unsure) {
        word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) word |= (uint32_t)fminf(fmaxf(__builtin_rintf((x[e] - t.m) / t.s), 0.0f), 15.0f) << sh(e);          // (NaN: 0)
    }
    return word;
}

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    } else {
        const floatx4 a = *reinterpret_cast<const floatx4 *>(p), b = *reinterpret_cast<const floatx4 *>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (bf16_t)x[e];
        *reinterpret_cast<bf16x8 *>(p) = v;
    } else {
        floatx4 a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) { a[e] = x[e]; b[e] = x[4 + e]; }
        *reinterpret_cast<floatx4 *>(p) = a; *reinterpret_cast<floatx4 *>(p + 4) = b;
    }
}

// The record of a wave: the `index`-th of those that the newest tokens of the sequences touch, and one head.  Positions from .. to - 1 of the record are the call's,
// position from + i in row `row` + i; those from `held` on are not there, nor is any where the record is not.
struct Place { bool any, there; int token0, row, from, to, held; uint8_t *record; };
__device__ __forceinline__ Place place_of(const CacheArgs &a, int index, int head, int64_t record_bytes)
{
    Place p{};
    int before = 0;
    for (int base = 0; base < a.b.sequences && !p.any; base += 64) {
        const int b = base + (threadIdx.x & 63);
        KvSeq s{};
        if (b < a.b.sequences) s = kv_seq(a.b, a.page_records * kKvRecord, b);
        const int rec0 = s.pos >> 5, mine = s.n > 0 ? ((s.pos + s.n - 1) >> 5) - rec0 + 1 : 0, x = lane_sums(mine), at = index - before - (x - mine);
        const uint64_t has = __ballot(at >= 0 && at < mine);
        if (has != 0) {
            const int src = __ffsll((unsigned long long)has) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            const int rec = of(rec0) + of(at), pos = of(s.pos), end = pos + of(s.n) - 1;
            p.any = true;
            p.token0 = rec * kKvRecord;
            p.from = max(p.token0, pos);
            p.to = min(p.token0 + kKvRecord - 1, end) + 1;
            p.row = of(s.first) + (p.from - pos);
            p.held = of(s.len);
            if (rec >= 0 && p.token0 < p.held) {
                const int of_seq = quotient(rec, a.page_records), page = __builtin_amdgcn_readfirstlane(a.b.table[(int64_t)(base + src) * a.b.table_stride + of_seq]);
                p.there = page >= 0 && page < a.pages;
                p.record = a.pool + (((int64_t)(p.there ? page : 0) * a.heads + head) * a.page_records + (rec - of_seq * a.page_records)) * record_bytes;
            }
        }
        before += __builtin_amdgcn_readlane(x, 63);
    }
    return p;
}

// half word of a value: token slot, products 4 a ..
__device__ __forceinline__ uint32_t value_at(int slot, int a, int r)
{
    return (uint32_t)(a * 1024 + (((slot & 15) >> 2) * 16 + r) * 16 + ((slot >> 4) * 2 + ((slot & 3) >> 1)) * 4 + (slot & 1) * 2);
}
// word of a key: tokens 16 h + t, of lane c of the token; the NS words of it from j = 0 on are neighbours in pieces of four (two, where NS = 2)
template <int NS> __device__ __forceinline__ uint32_t key_at(int h, int t, int c, int j)
{
    const int w = h * NS + j;
    return (uint32_t)((w >> 2) * 1024 + (c * 16 + t) * 16 + (w & 3) * 4);
}

// the lanes of a wave see each other's writes to LDS behind this
__device__ __forceinline__ void wave_meets() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// the elements of the lane's token `pos`, zeros where it is none of the call's
template <int NS, typename T> __device__ __forceinline__ void load_token(const KvRows &rows, const Place &at, int pos, int head, int c, float (&x)[NS][8])
{
    if (pos >= at.from && pos < at.to) {
        const T *p = static_cast<const T *>(rows.p) + (int64_t)(at.row + (pos - at.from)) * rows.token_stride + head * rows.head_stride + 8 * c;
#pragma unroll
        for (int j = 0; j < NS; ++j) load8(p + 32 * j, x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[j][e] = 0.0f;
    }
}

// f(IC<0>{}) ... f(IC<N - 1>{})
template <int N, int I = 0, typename F> __device__ __forceinline__ void static_for_heads(F &&f)
{
    if constexpr (I < N) { f(IC<I>{}); static_for_heads<N, I + 1>(f); }
}

// What the turned write has beside it.  blockIdx.y from kv_blocks on: queries, `block_heads` heads each.
struct TurnArgs {
    const float *freq;
    KvRows q, q_out;
    float amplitude;
    int half, part, interleaved, q_heads, block_heads, kv_blocks, once;
};
__device__ __forceinline__ void turn(float &x, float &y, floatx2 cs)
{
    const float u = __builtin_fmaf(x, cs[0], -(y * cs[1]));
    y = __builtin_fmaf(y, cs[0], x * cs[1]);
    x = u;
}

// A token's key, lane c of its four: elements 32 j + 8 c ..; `turns` of its token; `from` its first element in memory, which nothing writes.  All lanes come here, with a token's
// turns and memory where theirs is none: nothing but scalar branches, so that no register is parked while lanes are off.
template <int NS, typename T> __device__ __forceinline__ void turn_key(const TurnArgs &r, const floatx2 *turns, const T *from, int c, float (&x)[NS][8])
{
    if (r.interleaved) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const int p = 16 * j + 4 * c + e / 2;
                const floatx2 cs = turns[min(p, r.half - 1)];
                float u = x[j][e], v = x[j][e + 1];
                turn(u, v, cs);
                x[j][e] = p < r.half ? u : x[j][e];
                x[j][e + 1] = p < r.half ? v : x[j][e + 1];
            }
    } else if (r.half % 32 == 0) {                            // the partner is the lane's own
        const int apart = r.half / 32;
        static_for_heads<NS / 2>([&](auto h) {
            constexpr int H = decltype(h)::value + 1;
            if (apart != H) return;
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) turn(x[j][e], x[j + H][e], turns[32 * j + 8 * c + e]);
        });
    } else {                                                  // it is another lane's: from memory
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = 32 * j + 8 * c + e, p = i < r.half ? i : min(i - r.half, r.half - 1);
                const floatx2 cs = turns[p];
                const float other = to_float(from[i < r.half ? i + r.half : p]);
                float u = i < r.half ? x[j][e] : other, v = i < r.half ? other : x[j][e];
                turn(u, v, cs);
                x[j][e] = i < r.half ? u : i < r.part ? v : x[j][e];
            }
    }
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = to_float((T)x[j][e]);
}

// The queries of a record's rows, heads head0 ..: a unit of work is eight neighbouring elements, or two times eight that are partners, two units on their way at a time; pairs and single
// elements where eight do not divide half of what is turned.  Both of a pair are read before either is written.
template <int NS, typename T, bool ONCE> __device__ __forceinline__ void turn_queries(const TurnArgs &r, const floatx2 *turns, const Place &at, int head0)
{
    constexpr int D = 32 * NS, kThreads = kCacheWaves * 64;
    const int heads = min(r.block_heads, r.q_heads - head0), tokens = at.to - at.from;
    const bool by_eight = r.interleaved || r.half % 8 == 0;
    const int turned = r.interleaved ? D / 8 : by_eight ? r.half / 8 : r.half, units = r.interleaved ? D / 8 : by_eight ? (D - r.half) / 8 : D - r.half, n = tokens * heads * units;
    struct Unit { const T *from; T *to; const floatx2 *cs; int p; Eight<T> x, y; };
    auto place = [&](int u) {
        Unit w;
        const int th = quotient(u, units), t = quotient(th, heads), h = head0 + (th - t * heads);
        const int64_t row = at.row + t;
        w.p = u - th * units;
        w.from = static_cast<const T *>(r.q.p) + row * r.q.token_stride + h * r.q.head_stride;
        w.to = static_cast<T *>(r.q_out.p) + row * r.q_out.token_stride + h * r.q_out.head_stride;
        w.cs = turns + t * r.half;
        return w;
    };
    if (!by_eight) {
        for (int u = threadIdx.x; u < n; u += kThreads) {
            const Unit w = place(u);
            if (w.p < turned) {
                float x = to_float(w.from[w.p]), y = to_float(w.from[w.p + r.half]);
                turn(x, y, w.cs[w.p]);
                w.to[w.p] = (T)x; w.to[w.p + r.half] = (T)y;
            } else {
                w.to[w.p + r.half] = w.from[w.p + r.half];
            }
        }
        return;
    }
    auto take = [&](int u) {
        Unit w = place(min(u, n - 1));
        const bool two = !r.interleaved && w.p < turned;
        const T *from = w.from + 8 * w.p;
        w.x.template load<ONCE>(r.interleaved || two ? from : from + r.half);
        if (two) w.y.template load<ONCE>(from + r.half);
        return w;
    };
    auto put = [&](Unit &w) {
        float x[8], y[8];
        T *to = w.to + 8 * w.p;
        if (r.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = w.x.get(e);
#pragma unroll
            for (int e = 0; e < 8; e += 2) if (8 * w.p + e < r.part) turn(x[e], x[e + 1], w.cs[4 * w.p + e / 2]);
            w.x.set(x);
        } else if (w.p < turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = w.x.get(e); y[e] = w.y.get(e); turn(x[e], y[e], w.cs[8 * w.p + e]); }
            w.x.set(x);
            w.y.set(y);
            w.y.template store<ONCE>(to + r.half);
        } else {
            to += r.half;
        }
        w.x.template store<ONCE>(to);
    };
    for (int u = threadIdx.x; u < n; u += 2 * kThreads) {
        Unit v = take(u), w = take(u + kThreads);
        put(v);
        if (u + kThreads < n) put(w);
    }
}

template <int NS, int SG, typename T, bool TURN> __device__ __forceinline__ void kv_write_body(const CacheArgs &a, const TurnArgs &turned)
{
    using R = KvRecord<NS, SG>;
    extern __shared__ __attribute__((aligned(16))) floatx2 turns[];           // [tokens of the record][half]
    Place all{};
    if constexpr (TURN) {
        all = place_of(a, blockIdx.x, 0, R::kBytes);
        if (!all.any) return;                                 // (the same in all waves)
        for (int e = threadIdx.x; e < (all.to - all.from) * turned.half; e += kCacheWaves * 64) {
            const int t = quotient(e, turned.half);
            float cs, sn;
            cos_sin(all.from + t, turned.freq[e - t * turned.half], cs, sn);
            turns[e] = floatx2{cs * turned.amplitude, sn * turned.amplitude};
        }
        __syncthreads();
        if ((int)blockIdx.y >= turned.kv_blocks) {
            const int head0 = ((int)blockIdx.y - turned.kv_blocks) * turned.block_heads;
            if (turned.once) turn_queries<NS, T, true>(turned, turns, all, head0); else turn_queries<NS, T, false>(turned, turns, all, head0);
            return;
        }
    }
    __shared__ __attribute__((aligned(16))) uint8_t lds[kCacheWaves / 2][16 * R::D];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, t = lane >> 2, c = lane & 3;
    const int head = blockIdx.y * (kCacheWaves / 2) + (wave >> 1);
    const bool values = (wave & 1) != 0;                      // this wave's part of the record
    if (head >= a.heads) return;
    Place at = all;
    if constexpr (TURN) at.record += (int64_t)head * a.page_records * R::kBytes;
    else at = place_of(a, blockIdx.x, head, R::kBytes);
    if (!at.any || !at.there) return;
    at.to = min(at.to, at.held);
    const bool full = at.to - at.from == kKvRecord;
    const KvRows rows = values ? a.v : a.k;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int pos = at.token0 + h * 16 + t;
        const bool is = pos >= at.from && pos < at.to;
        if (!__any(is)) continue;
        float x[NS][8];
        load_token<NS, T>(rows, at, pos, head, c, x);
        if constexpr (TURN) {
            if (!values) {
                const int row = is ? pos - at.from : 0;
                turn_key<NS, T>(turned, turns + row * turned.half, static_cast<const T *>(rows.p) + (int64_t)(at.row + row) * rows.token_stride + head * rows.head_stride, c, x);
            }
        }
        Step steps[R::G];
#pragma unroll
        for (int g = 0; g < R::G; ++g) {
            float lo = x[g * SG][0], hi = lo;
#pragma unroll
            for (int j = g * SG; j < (g + 1) * SG; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) { lo = least_of(lo, x[j][e]); hi = greater(hi, x[j][e]); }
            steps[g] = step_of(quad_least(lo), quad_greatest(hi));
            if (is && c == 0) *reinterpret_cast<uint32_t *>(at.record + (values ? R::kValueSteps : R::kKeySteps) + g * 128 + (h * 16 + t) * 4) = steps[g].word;
        }
        if (!values) {
            uint32_t words[NS];
#pragma unroll
            for (int j = 0; j < NS; ++j) words[j] = codes_of(x[j], steps[j / SG], [](int e) { return 16 * (e & 1) + 4 * (e >> 1); });
            if (is) {
                uint8_t *to = at.record + R::kKeys;
                if constexpr (NS == 2) *reinterpret_cast<uintx2 *>(to + key_at<NS>(h, t, c, 0)) = uintx2{words[0], words[1]};
                else
#pragma unroll
                    for (int j = 0; j < NS; j += 4) *reinterpret_cast<uintx4 *>(to + key_at<NS>(h, t, c, j)) = uintx4{words[j], words[j + 1], words[j + 2], words[j + 3]};
            }
        } else {
            uint32_t pairs[NS];                               // byte i: the elements 2 i and 2 i + 1
#pragma unroll
            for (int j = 0; j < NS; ++j) pairs[j] = codes_of(x[j], steps[j / SG], [](int e) { return 4 * e; });
            uint8_t *to = full ? lds[wave >> 1] : at.record + R::kValues;
#pragma unroll
            for (int n = 0; n < NS / 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {                 // row 4 c + i of products 4 n ..: a pair of j = 2 n and one of 2 n + 1
                    const uint32_t half = (pairs[2 * n] >> (8 * i) & 0xFFu) | (pairs[2 * n + 1] >> (8 * i) & 0xFFu) << 8;
                    if (is) *reinterpret_cast<uint16_t *>(to + value_at(h * 16 + t, n, 4 * c + i)) = (uint16_t)half;
                }
        }
    }
    if (values && full) {
        wave_meets();
#pragma unroll
        for (int n = 0; n < NS / 2; ++n)
            *reinterpret_cast<uintx4 *>(at.record + R::kValues + n * 1024 + lane * 16) = *reinterpret_cast<const uintx4 *>(lds[wave >> 1] + n * 1024 + lane * 16);
    }
}

template <int NS, int SG, typename T> __global__ __launch_bounds__(kCacheWaves * 64) void k_kv_write(const CacheArgs a) { kv_write_body<NS, SG, T, false>(a, TurnArgs{}); }
template <int NS, int SG, typename T> __global__ __launch_bounds__(kCacheWaves * 64) void k_kv_rotary_write(const CacheArgs a, const TurnArgs r) { kv_write_body<NS, SG, T, true>(a, r); }

__device__ __forceinline__ float stands_for(uint32_t code, uint32_t step)
{
    const half2v sm = __builtin_bit_cast(half2v, step);
    return __builtin_fmaf((float)sm[0], (float)code, (float)sm[1]);
}

template <int NS, int SG, typename T> __global__ __launch_bounds__(kCacheWaves * 64) void k_kv_read(const CacheArgs a)
{
    using R = KvRecord<NS, SG>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kCacheWaves / 2][16 * R::D];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, t = lane >> 2, c = lane & 3;
    const int head = blockIdx.y * (kCacheWaves / 2) + (wave >> 1);
    const bool values = (wave & 1) != 0;                      // this wave's part of the record
    const KvRows rows = values ? a.v : a.k;
    if (head >= a.heads || rows.p == nullptr) return;
    const Place at = place_of(a, blockIdx.x, head, R::kBytes);
    if (!at.any) return;
    uint32_t steps[2][R::G], words[2][NS];                    // of a key
    if (at.there) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < R::G; ++g) steps[h][g] = *reinterpret_cast<const uint32_t *>(at.record + (values ? R::kValueSteps : R::kKeySteps) + g * 128 + (h * 16 + t) * 4);
        if (values) {
            uintx4 v[NS / 2];
#pragma unroll
            for (int n = 0; n < NS / 2; ++n) v[n] = *reinterpret_cast<const uintx4 *>(at.record + R::kValues + n * 1024 + lane * 16);
#pragma unroll
            for (int n = 0; n < NS / 2; ++n) *reinterpret_cast<uintx4 *>(lds[wave >> 1] + n * 1024 + lane * 16) = v[n];
            wave_meets();
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t *from = at.record + R::kKeys;
                if constexpr (NS == 2) { const uintx2 v = *reinterpret_cast<const uintx2 *>(from + key_at<NS>(h, t, c, 0)); words[h][0] = v[0]; words[h][1] = v[1]; }
                else
#pragma unroll
                    for (int j = 0; j < NS; j += 4) {
                        const uintx4 v = *reinterpret_cast<const uintx4 *>(from + key_at<NS>(h, t, c, j));
#pragma unroll
                        for (int i = 0; i < 4; ++i) words[h][j + i] = v[i];
                    }
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int pos = at.token0 + h * 16 + t;
        if (pos < at.from || pos >= at.to) continue;
        const bool there = at.there && pos < at.held;
        T *to = static_cast<T *>(rows.p) + (int64_t)(at.row + (pos - at.from)) * rows.token_stride + head * rows.head_stride + 8 * c;
        float x[NS][8] = {};
        if (there && !values) {
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][e] = stands_for((words[h][j] >> (16 * (e & 1) + 4 * (e >> 1))) & 15u, steps[h][j / SG]);
        } else if (there) {
#pragma unroll
            for (int n = 0; n < NS / 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t half = *reinterpret_cast<const uint16_t *>(lds[wave >> 1] + value_at(h * 16 + t, n, 4 * c + i));
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const int j = 2 * n + (e >> 1); x[j][2 * i + (e & 1)] = stands_for((half >> (4 * e)) & 15u, steps[h][j / SG]); }
                }
        }
#pragma unroll
        for (int j = 0; j < NS; ++j) store8(to + 32 * j, x[j]);
    }
}

template <int NS, int SG> void launch(const KvShape &s, const CacheArgs &a, int records, bool write, const TurnArgs *turned, hipStream_t st)
{
    dim3 grid((unsigned)records, (unsigned)(s.heads + kCacheWaves / 2 - 1) / (kCacheWaves / 2));
    if (turned != nullptr) {
        TurnArgs r = *turned;
        r.kv_blocks = (int)grid.y;
        // Queries of `block_heads` heads to a workgroup, or of as few as four where that leaves compute units idle
        r.block_heads = std::min(r.block_heads, std::max(4, (int)((int64_t)r.q_heads * records / 512)));
        r.block_heads = std::max(r.block_heads, (r.q_heads + 16383) / 16384);
        grid.y += (unsigned)((r.q_heads + r.block_heads - 1) / r.block_heads);
        const size_t lds = (size_t)std::min(a.b.max_new, kKvRecord) * r.half * sizeof(floatx2);
        if (s.act_bf16) k_kv_rotary_write<NS, SG, bf16_t><<<grid, kCacheWaves * 64, lds, st>>>(a, r);
        else k_kv_rotary_write<NS, SG, float><<<grid, kCacheWaves * 64, lds, st>>>(a, r);
    } else if (write) {
        if (s.act_bf16) k_kv_write<NS, SG, bf16_t><<<grid, kCacheWaves * 64, 0, st>>>(a);
        else k_kv_write<NS, SG, float><<<grid, kCacheWaves * 64, 0, st>>>(a);
    } else {
        if (s.act_bf16) k_kv_read<NS, SG, bf16_t><<<grid, kCacheWaves * 64, 0, st>>>(a);
        else k_kv_read<NS, SG, float><<<grid, kCacheWaves * 64, 0, st>>>(a);
    }
}

void launch_any(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, void *pool, bool write, const TurnArgs *turned, hipStream_t st)
{
    const CacheArgs a{b, k, v, static_cast<uint8_t *>(pool), s.pages, s.heads, s.page_records};
    // n newest tokens touch at most (n + 30) / 32 + 1 records
    const int64_t each = (int64_t)b.sequences * (((int64_t)b.max_new + 30) / 32 + 1), all = b.tokens / 32 + 2 * (int64_t)b.sequences;
    const int records = (int)(each < all ? each : all);
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(s, a, records, write, turned, st); else launch<2, 2>(s, a, records, write, turned, st); break;
    case 128:
        if (sg == 1) launch<4, 1>(s, a, records, write, turned, st); else if (sg == 2) launch<4, 2>(s, a, records, write, turned, st); else launch<4, 4>(s, a, records, write, turned, st);
        break;
    default:
        if (sg == 1) launch<8, 1>(s, a, records, write, turned, st); else if (sg == 2) launch<8, 2>(s, a, records, write, turned, st);
        else if (sg == 4) launch<8, 4>(s, a, records, write, turned, st); else launch<8, 8>(s, a, records, write, turned, st);
    }
}

}  // namespace

void launch_kv_write(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, void *pool, hipStream_t st) { launch_any(s, b, k, v, pool, true, nullptr, st); }
void launch_kv_read(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, const void *pool, hipStream_t st)
{
    launch_any(s, b, k, v, const_cast<void *>(pool), false, nullptr, st);
}

void launch_kv_rotary_write(const KvShape &s, const KvBatch &b, const Rotary &turned, const KvRows &q, const KvRows &q_out, int q_heads, const KvRows &k, const KvRows &v, void *pool,
                            hipStream_t st)
{
    TurnArgs r{};
    r.freq = turned.freq; r.q = q; r.q_out = q_out; r.amplitude = turned.amplitude; r.half = turned.part / 2; r.part = turned.part; r.interleaved = turned.interleaved;
    r.q_heads = q_heads;
    // A record's tokens of 16 heads, so that a prompt's cosines and sines are a fraction of the work; where a sequence has a token or a few, all the heads that 256 lanes turn at once
    r.block_heads = std::max(16, 512 / (std::max(1, std::min(b.max_new, kKvRecord)) * s.head_dim / 8));
    r.once = 2 * b.tokens * q_heads * s.head_dim * (s.act_bf16 ? 2 : 4) > (int64_t)96 << 20;          // (see launch_rotary)
    launch_any(s, b, k, v, pool, true, &r, st);
}

}  // namespace eqat
