// Writing keys and values into the 4-bit cache, and reading them back.
//
// Both move bytes: a token and head of 128 elements is 512 bytes of bf16 and 136 (one group) to 160 (four) in the cache.  A row of 16 lanes takes one token and
// head.  Of the key it takes eight neighbouring elements a lane, one word of the cache; of the value, two neighbouring elements of every 32, one half word of the
// cache for every 64 (kv.h says why they stand there).
#include "kv.h"

namespace eqat {
namespace {

struct CacheArgs {
    KvBatch b;
    KvRows k, v;
    uint8_t *pool;
    int64_t pages, rows;
    int heads, page_records;
};

// maximum over the LANES lanes around this one (a power of two, at most 16)
template <int LANES> __device__ __forceinline__ float row_max(float v)
{
    if constexpr (LANES > 1) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true)));        // quad_perm 1 0 3 2
    if constexpr (LANES > 2) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true)));        // quad_perm 2 3 0 1
    if constexpr (LANES > 4) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, true)));       // the half row mirrored
    if constexpr (LANES > 8) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, true)));       // the row mirrored
    return v;
}

// A group's step and least element, as they stand in the cache.  `odd` is 0, or NaN where an element is not finite: the whole group then stands as NaN,
// as one with an element beyond binary16 does (so no step passes 131008 / 15, and what a kernel makes of codes and steps stays within binary16 or a rounding of it).
struct Step { float s, m; uint32_t word; };
__device__ __forceinline__ Step step_of(float least, float greatest, float odd)
{
    _Float16 m = (_Float16)least, s = (_Float16)fmaxf((greatest - least) / 15.0f, 0x1p-24f);
    if (!(fabsf((float)m) + fabsf((float)(_Float16)greatest) + odd < __builtin_inff())) { m = (_Float16)__builtin_nanf(""); s = m; }
    Step r;
    r.s = (float)s; r.m = (float)m;
    r.word = (uint32_t)__builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, m) << 16;
    return r;
}
// round((x - m) / s) within 0 .. 15 (0 where that is NaN), of the correctly rounded quotient
__device__ __forceinline__ uint32_t code_of(float x, const Step &t)
{
    return (uint32_t)fminf(fmaxf(__builtin_rintf((x - t.m) / t.s), 0.0f), 15.0f);
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
template <typename T> struct Two { T v[2]; };

// Where the token of row `row` of the launch stands.  valid: it has a position, on a page of the pool.
struct Place { bool valid; int head; int64_t token; int slot; int64_t record; };
__device__ __forceinline__ Place place_of(const CacheArgs &a, int64_t row)
{
    Place p{};
    p.token = row / a.heads;
    p.head = (int)(row - p.token * a.heads);
    if (row >= a.rows) return p;
    const int b = kv_seq_of(a.b, (int)p.token);
    const KvSeq s = kv_seq(a.b, a.page_records * kKvRecord, b);
    const int i = (int)p.token - s.first, pos = s.len - s.n + i;
    if (i < 0 || i >= s.n || pos < 0) return p;
    const int rec = pos >> 5, page_of_seq = rec / a.page_records;
    const int page = a.b.table[(int64_t)b * a.b.table_stride + page_of_seq];
    p.slot = pos & 31;
    p.valid = page >= 0 && page < a.pages;
    p.record = ((int64_t)page * a.heads + p.head) * a.page_records + (rec - page_of_seq * a.page_records);
    return p;
}

// byte of key word (step j, chunk c) and of value half (products 4 a ..) of a token
template <int NS> __device__ __forceinline__ uint32_t key_at(int slot, int j, int c)
{
    const int w = (slot >> 4) * NS + j;
    return (uint32_t)((w >> 2) * 1024 + (c * 16 + (slot & 15)) * 16 + (w & 3) * 4);
}
__device__ __forceinline__ uint32_t value_at(int slot, int a, int r)
{
    return (uint32_t)(a * 1024 + (((slot & 15) >> 2) * 16 + r) * 16 + ((slot >> 4) * 2 + ((slot & 3) >> 1)) * 4 + (slot & 1) * 2);
}

template <int NS, int SG, typename T> __global__ __launch_bounds__(256) void k_kv_write(const CacheArgs a)
{
    using R = KvRecord<NS, SG>;
    const int i = threadIdx.x & 15;
    const Place at = place_of(a, (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4));
    if (!at.valid) return;
    uint8_t *rec = a.pool + at.record * R::kBytes;
    const T *key = static_cast<const T *>(a.k.p) + at.token * a.k.token_stride + at.head * a.k.head_stride;
    const T *value = static_cast<const T *>(a.v.p) + at.token * a.v.token_stride + at.head * a.v.head_stride;
    constexpr int kWords = (NS + 3) / 4;               // words of the key that a lane takes: i, i + 16
    float x[kWords][8], y[NS][2];
    if (i < 4 * NS) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) load8(key + (w * 16 + i) * 8, x[w]);
    }
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        const Two<T> t = *reinterpret_cast<const Two<T> *>(value + 32 * j + 2 * i);
        y[j][0] = (float)t.v[0]; y[j][1] = (float)t.v[1];
    }
    if (i < 4 * NS) {
        float lo[kWords], hi[kWords], odd[kWords];
        constexpr int kLanes = SG < 4 ? 4 * SG : 16;   // lanes of a group
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            float l = x[w][0], h = x[w][0], o = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) { l = fminf(l, x[w][e]); h = fmaxf(h, x[w][e]); o += x[w][e] * 0.0f; }
            lo[w] = -row_max<kLanes>(-l); hi[w] = row_max<kLanes>(h); odd[w] = row_max<kLanes>(o != o ? 1.0f : 0.0f);
        }
        if constexpr (SG == 8) {
            lo[0] = lo[1] = fminf(lo[0], lo[1]); hi[0] = hi[1] = fmaxf(hi[0], hi[1]); odd[0] = odd[1] = fmaxf(odd[0], odd[1]);
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const Step t = step_of(lo[w], hi[w], odd[w] != 0.0f ? __builtin_nanf("") : 0.0f);
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) word |= code_of(x[w][e], t) << (16 * (e & 1) + 4 * (e >> 1));
            const int j = (w * 16 + i) >> 2;
            *reinterpret_cast<uint32_t *>(rec + R::kKeys + key_at<NS>(at.slot, j, i & 3)) = word;
            if ((w * 16 + i) % (4 * SG) == 0) *reinterpret_cast<uint32_t *>(rec + R::kKeySteps + (j / SG) * 128 + at.slot * 4) = t.word;
        }
    }
    uint32_t half[NS / 2] = {};
#pragma unroll
    for (int g = 0; g < R::G; ++g) {
        float l = y[g * SG][0], h = l, o = 0.0f;
#pragma unroll
        for (int j = 0; j < SG; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) { l = fminf(l, y[g * SG + j][e]); h = fmaxf(h, y[g * SG + j][e]); o += y[g * SG + j][e] * 0.0f; }
        const Step t = step_of(-row_max<16>(-l), row_max<16>(h), row_max<16>(o != o ? 1.0f : 0.0f) != 0.0f ? __builtin_nanf("") : 0.0f);
#pragma unroll
        for (int j = 0; j < SG; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) { const int n = 2 * (g * SG + j) + e; half[n >> 2] |= code_of(y[g * SG + j][e], t) << (4 * (n & 3)); }
        if (i == 0) *reinterpret_cast<uint32_t *>(rec + R::kValueSteps + g * 128 + at.slot * 4) = t.word;
    }
#pragma unroll
    for (int n = 0; n < NS / 2; ++n) *reinterpret_cast<uint16_t *>(rec + R::kValues + value_at(at.slot, n, i)) = (uint16_t)half[n];
}

__device__ __forceinline__ float stands_for(uint32_t code, uint32_t step)
{
    const float s = (float)__builtin_bit_cast(_Float16, (uint16_t)step), m = (float)__builtin_bit_cast(_Float16, (uint16_t)(step >> 16));
    return __builtin_fmaf(s, (float)code, m);
}

template <int NS, int SG, typename T> __global__ __launch_bounds__(256) void k_kv_read(const CacheArgs a)
{
    using R = KvRecord<NS, SG>;
    const int i = threadIdx.x & 15;
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= a.rows) return;
    const Place at = place_of(a, row);
    const uint8_t *rec = a.pool + (at.valid ? at.record * R::kBytes : 0);
    if (a.k.p != nullptr && i < 4 * NS) {
        T *key = static_cast<T *>(a.k.p) + at.token * a.k.token_stride + at.head * a.k.head_stride;
#pragma unroll
        for (int w = 0; w < (NS + 3) / 4; ++w) {
            const int j = (w * 16 + i) >> 2;
            float x[8] = {};
            if (at.valid) {
                const uint32_t word = *reinterpret_cast<const uint32_t *>(rec + R::kKeys + key_at<NS>(at.slot, j, i & 3));
                const uint32_t step = *reinterpret_cast<const uint32_t *>(rec + R::kKeySteps + (j / SG) * 128 + at.slot * 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = stands_for((word >> (16 * (e & 1) + 4 * (e >> 1))) & 15u, step);
            }
            store8(key + (w * 16 + i) * 8, x);
        }
    }
    if (a.v.p != nullptr) {
        T *value = static_cast<T *>(a.v.p) + at.token * a.v.token_stride + at.head * a.v.head_stride;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            Two<T> t{};
            if (at.valid) {
                const uint32_t half = *reinterpret_cast<const uint16_t *>(rec + R::kValues + value_at(at.slot, j >> 1, i));
                const uint32_t step = *reinterpret_cast<const uint32_t *>(rec + R::kValueSteps + (j / SG) * 128 + at.slot * 4);
#pragma unroll
                for (int e = 0; e < 2; ++e) t.v[e] = (T)stands_for((half >> (8 * (j & 1) + 4 * e)) & 15u, step);
            }
            *reinterpret_cast<Two<T> *>(value + 32 * j + 2 * i) = t;
        }
    }
}

template <int NS, int SG> void launch(const KvShape &s, const CacheArgs &a, bool write, hipStream_t st)
{
    const dim3 grid((unsigned)((a.rows + 15) / 16));
    if (write) {
        if (s.act_bf16) k_kv_write<NS, SG, bf16_t><<<grid, 256, 0, st>>>(a);
        else k_kv_write<NS, SG, float><<<grid, 256, 0, st>>>(a);
    } else {
        if (s.act_bf16) k_kv_read<NS, SG, bf16_t><<<grid, 256, 0, st>>>(a);
        else k_kv_read<NS, SG, float><<<grid, 256, 0, st>>>(a);
    }
}

void launch_any(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, void *pool, bool write, hipStream_t st)
{
    const CacheArgs a{b, k, v, static_cast<uint8_t *>(pool), s.pages, b.tokens * s.heads, s.heads, s.page_records};
    if (a.rows == 0) return;
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(s, a, write, st); else launch<2, 2>(s, a, write, st); break;
    case 128: if (sg == 1) launch<4, 1>(s, a, write, st); else if (sg == 2) launch<4, 2>(s, a, write, st); else launch<4, 4>(s, a, write, st); break;
    default:
        if (sg == 1) launch<8, 1>(s, a, write, st); else if (sg == 2) launch<8, 2>(s, a, write, st);
        else if (sg == 4) launch<8, 4>(s, a, write, st); else launch<8, 8>(s, a, write, st);
    }
}

}  // namespace

void launch_kv_write(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, void *pool, hipStream_t st) { launch_any(s, b, k, v, pool, true, st); }
void launch_kv_read(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, const void *pool, hipStream_t st)
{
    launch_any(s, b, k, v, const_cast<void *>(pool), false, st);
}

}  // namespace eqat
