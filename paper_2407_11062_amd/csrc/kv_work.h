// What the two attention kernels share: arguments, the division of the work, joining.
#pragma once
#include "gemm_tiles.h"
#include "kv.h"

namespace eqat {

struct AttendArgs {
    KvBatch b;
    KvRows q, out;
    float *lse, *parts;                            // parts: [chunk][head][unit_rows][D] sums, then [chunk][head][unit_rows][2] maxima and totals
    uint32_t *counters;                            // [unit][head], zero before and after every launch
    const uint8_t *pool;
    int64_t pages;
    int heads, ratio, page_records, window, target, slots;
    int unit_rows, fewest;                         // rows (query, head of the group) of a unit; records of a chunk at the least
    int from_rows, to_rows;                        // the launch takes the sequences with from_rows <= rows < to_rows
    bool causal;
    float scale;                                   // times log2(e)
};

namespace {

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float low_half(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)w); }
__device__ __forceinline__ float high_half(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }

// over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float chunks_max(float v)
{
    const uint32_t a = __float_as_uint(v);
    const uintx2 p = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const float w = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const uint32_t b = __float_as_uint(w);
    const uintx2 q = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float chunks_sum(float v)
{
    const uint32_t a = __float_as_uint(v);
    const uintx2 p = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const float w = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const uint32_t b = __float_as_uint(w);
    const uintx2 q = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

__device__ __forceinline__ floatx4 mfma(const uintx4 &a, const half8 &b, const floatx4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), b, c, 0, 0, 0); }

// How the work of a call is divided: a unit is up to unit_rows rows of a sequence (times every head of the cache), its records are cut into chunks of C, and a workgroup
// takes a chunk.  C follows from the lengths as they are on the device, so that the chunks of all sequences are about `target` in all, however their lengths differ.
struct Work { int b, unit, chunk, chunks, first, last, part, counter; KvSeq s; bool any; };

struct Extent { int units, lo, hi; };
__device__ __forceinline__ Extent extent_of(const AttendArgs &a, const KvSeq &s)
{
    Extent e;
    const int rows = s.n * a.ratio;
    e.units = rows >= a.from_rows && rows < a.to_rows ? (rows + a.unit_rows - 1) / a.unit_rows : 0;
    e.lo = a.window > 0 ? max(0, s.len - s.n - a.window + 1) >> 5 : 0;
    e.hi = (s.len + 31) >> 5;
    return e;
}

__device__ __forceinline__ Work work_of(const AttendArgs &a, int slot)
{
    const int lane = threadIdx.x & 63, page_tokens = a.page_records * kKvRecord;
    uint64_t records = 0;
    for (int base = 0; base < a.b.sequences; base += 64) {
        const int b = base + lane;
        if (b < a.b.sequences) {
            const Extent e = extent_of(a, kv_seq(a.b, page_tokens, b));
            records += (uint64_t)e.units * (uint64_t)(e.hi - e.lo);
        }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) records += __shfl_xor(records, d);
    const int C = max((int)((records + a.target - 1) / a.target), a.fewest);
    Work w{};
    int before = 0, parts = 0, counters = 0;
    bool found = false;
    for (int base = 0; base < a.b.sequences; base += 64) {
        const int b = base + lane;
        KvSeq s{};
        Extent e{};
        if (b < a.b.sequences) { s = kv_seq(a.b, page_tokens, b); e = extent_of(a, s); }
        const int chunks = e.units > 0 ? max(1, (e.hi - e.lo + C - 1) / C) : 0, mine = e.units * chunks, cut = chunks > 1 ? e.units : 0;
        int x = mine, y = cut * chunks, z = cut;         // inclusive sums over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int xx = __shfl_up(x, d), yy = __shfl_up(y, d), zz = __shfl_up(z, d);
            if (lane >= d) { x += xx; y += yy; z += zz; }
        }
        const int at = slot - before - (x - mine);       // this slot within the sequence of the lane
        const uint64_t has = __ballot(at >= 0 && at < mine);
        if (has != 0 && !found) {
            const int src = __ffsll((unsigned long long)has) - 1;
            found = true;
            const int i = __shfl(at, src);
            w.b = base + src;
            w.chunks = __shfl(chunks, src);
            w.unit = i / w.chunks;
            w.chunk = i - w.unit * w.chunks;
            w.s.first = __shfl(s.first, src); w.s.n = __shfl(s.n, src); w.s.len = __shfl(s.len, src);
            const int lo = __shfl(e.lo, src), hi = __shfl(e.hi, src);
            w.first = lo + w.chunk * C;
            w.last = min(hi, w.first + C);
            w.part = parts + __shfl(y - cut * chunks, src) + i;
            w.counter = counters + __shfl(z - cut, src) + w.unit;
        }
        before += __shfl(x, 63); parts += __shfl(y, 63); counters += __shfl(z, 63);
    }
    w.any = found && before <= a.slots;                  // more than the host was told of: nothing is computed
    return w;
}

// a launch has a slot for every chunk aimed at and for every unit there can be
int units_at_most(const KvBatch &b, int ratio, int unit_rows)
{
    const int64_t each = (int64_t)b.sequences * (((int64_t)b.max_new * ratio + unit_rows - 1) / unit_rows);
    const int64_t all = (b.tokens * ratio + unit_rows - 1) / unit_rows + b.sequences;
    return (int)(each < all ? each : all);
}

// Where a launch's counters and parts lie in the workspace.  There is at most one cut unit per chunk aimed at, and a cut unit has fewer than twice its share of them.
struct Scratch { size_t counters, parts, end; };
Scratch scratch_of(size_t at, int target, int heads, int unit_rows, int head_dim)
{
    const size_t chunks = (size_t)target * heads;
    Scratch l;
    l.counters = at;
    l.parts = at + (chunks * 4 + 255) / 256 * 256;
    l.end = l.parts + 2 * chunks * (size_t)unit_rows * (size_t)(head_dim * 4 + 8);
    return l;
}

}  // namespace

// ---- kv_prompt.hip ---------------------------------------------------------------------------
int prompt_target(const KvShape &s);
int prompt_unit_rows(const KvShape &s);
void launch_kv_prompt(const KvShape &s, AttendArgs a, hipStream_t st);

}  // namespace eqat
