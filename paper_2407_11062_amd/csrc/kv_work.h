// What the two attention kernels share: arguments, the division of the work, joining.
#pragma once
#include "gemm_tiles.h"
#include "kv.h"

#include <atomic>

namespace eqat {

struct AttendArgs {
    KvBatch b;
    KvRows q, out;
    float *lse, *parts;                            // parts: [chunk, or two of a workgroup][head][rows of a unit][D] sums, then [..][head][rows of a unit][2] maxima and totals
    uint32_t *counters;                            // streamed: [workgroup that a unit begins in][head], zero before and after every launch
    const uint8_t *pool;
    int64_t pages;
    int heads, ratio, page_records, window, target, slots;
    int unit_bits, fewest;                         // log2 of the rows (query, head of the group) of a unit; records of a chunk or share at the least
    int from_rows, to_rows;                        // the launch takes the sequences with from_rows <= rows < to_rows
    bool causal;
    float scale;                                   // times log2(e)
    int scale_exponent;                            // 2^scale_exponent <= scale < 2^(scale_exponent + 1)
};

// Where a launch's counters and parts lie in the workspace: two parts for each of the streamed kernel's workgroups, and for each chunk that prompts are cut into (a cut
// unit has fewer than twice its share of them).
struct Scratch { size_t counters, parts, end; };
inline Scratch scratch_of(size_t at, size_t chunks, bool counted, int unit_rows, int head_dim)
{
    Scratch l;
    l.counters = at;
    l.parts = at + (counted ? (chunks * 4 + 255) / 256 * 256 : 0);
    l.end = l.parts + 2 * chunks * (size_t)unit_rows * (size_t)(head_dim * 4 + 8);
    return l;
}

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

// How the work of a call is divided: a unit is up to 2^unit_bits rows of a sequence (times every head of the cache), its records are cut into chunks of C, and a workgroup
// takes a chunk.  C follows from the lengths as they are on the device, so that the chunks of all sequences are about `target` in all, however their lengths differ.
struct Work { int b, unit, chunk, chunks, first, last, part; KvSeq s; bool any; };

struct Extent { int units, lo, hi; };
__device__ __forceinline__ Extent extent_of(const AttendArgs &a, const KvSeq &s)
{
    Extent e;
    const int rows = s.n * a.ratio;
    e.units = rows >= a.from_rows && rows < a.to_rows ? (rows + (1 << a.unit_bits) - 1) >> a.unit_bits : 0;
    e.hi = (s.len + 31) >> 5;
    e.lo = a.window > 0 ? min(window_from(s.pos, a.window) >> 5, e.hi) : 0;
    return e;
}

// CUT: units may be cut.  UNITS: the unit with number `slot` as a whole; else the chunk
template <bool CUT, bool UNITS> __device__ __forceinline__ Work work_of(const AttendArgs &a, int slot)
{
    const int lane = threadIdx.x & 63, page_tokens = a.page_records * kKvRecord;
    KvSeq s{};
    Extent e{};
    auto look = [&](int base) {
        const int b = base + lane;
        s = KvSeq{}; e = Extent{};
        if (b < a.b.sequences) { s = kv_seq(a.b, page_tokens, b); e = extent_of(a, s); }
    };
    int C = 1 << 30;
    if constexpr (CUT) {
        float records = 0.0f;                            // in all, up to rounding: every workgroup adds them up in the same order
        int units = 0;
        for (int base = 0; base < a.b.sequences; base += 64) { look(base); records += (float)e.units * (float)(e.hi - e.lo); units += e.units; }
        records = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lane_sums(records)), 63));
        units = __builtin_amdgcn_readlane(lane_sums(units), 63);
        // every unit has one chunk that may be a small one; at least records / target whatever the rounding: the room for parts depends on it
        C = max((int)fminf(records / (float)max(a.target - units, a.target / 2) * 1.00001f, 1.0e9f) + 1, a.fewest);
    }
    Work w{};
    int before = 0, parts = 0;
    for (int base = 0; base < a.b.sequences; base += 64) {
        if (!CUT || a.b.sequences > 64) look(base);
        const int recs = e.hi - e.lo, chunks = !CUT ? min(e.units, 1) : e.units > 0 ? max(1, quotient(recs + C - 1, C)) : 0;
        const int mine = UNITS ? e.units : e.units * chunks, x = lane_sums(mine), y = CUT ? lane_sums(chunks > 1 ? e.units * chunks : 0) : 0;
        const int at = slot - before - (x - mine);       // this slot within the sequence of the lane
        const uint64_t has = __ballot(at >= 0 && at < mine);
        if (has != 0) {
            const int src = __ffsll((unsigned long long)has) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            const int i = of(at), each = quotient(of(recs) + of(chunks) - 1, of(chunks));
            w.any = true;
            w.b = base + src;
            w.chunks = of(chunks);
            w.unit = UNITS || w.chunks == 1 ? i : quotient(i, w.chunks);
            w.chunk = UNITS ? 0 : i - w.unit * w.chunks;
            w.s.first = of(s.first); w.s.n = of(s.n); w.s.len = of(s.len); w.s.pos = of(s.pos);
            w.first = of(e.lo) + w.chunk * each;
            w.last = min(of(e.hi), w.first + each);
            if constexpr (CUT) w.part = parts + of(y - (chunks > 1 ? mine * (UNITS ? chunks : 1) : 0)) + w.unit * w.chunks + w.chunk;
        }
        before += __builtin_amdgcn_readlane(x, 63); parts += __builtin_amdgcn_readlane(y, 63);
    }
    w.any = w.any && before <= a.slots;                  // more than the host was told of: nothing is computed
    return w;
}

// The other division, for rows few enough that what counts is the bytes of the cache: the records of all units, one after the other, in equal shares, one for each of
// the workgroups that are resident.  A share may end within a unit and begin in the next; each stretch of a unit costs a beginning and a join with the others.  Where
// shares that end with the units (`whole`: units take a whole number of them) are not more than kSpare records larger, it is those.  Else each unit's records follow
// kKvBeginning places that are none, for the time that a stretch's beginning and end take (about 4 us): shares of short units are of as many units, not of as many records.
constexpr int kSpare = 20;
struct Share { int first, last, size; bool whole; };
// A stretch of one unit: records rec .. rec_to - 1 (none: rec_to < rec), the unit's records and the stretch's end within the row of work.
struct Segment { int b, unit, rec, rec_to, unit_from, unit_to, to; KvSeq s; bool any; };
struct Lane { KvSeq s; Extent e; };                          // the sequence of a lane

__device__ __forceinline__ Lane lane_of(const AttendArgs &a, int base)
{
    Lane l{};
    const int b = base + (threadIdx.x & 63);
    if (b < a.b.sequences) { l.s = kv_seq(a.b, a.page_records * kKvRecord, b); l.e = extent_of(a, l.s); }
    return l;
}

// l: the lane's sequence of the first 64
__device__ __forceinline__ Share share_of(const AttendArgs &a, int slot, Lane l)
{
    int records = 0, units = 0;
    float about = 0.0f;
    for (int base = 0; base < a.b.sequences; base += 64) {
        if (base > 0) l = lane_of(a, base);
        records += l.e.units * max(1, l.e.hi - l.e.lo);
        units += l.e.units;
        about += (float)l.e.units * (float)(kKvBeginning + max(1, l.e.hi - l.e.lo));
    }
    records = __builtin_amdgcn_readlane(lane_sums(records), 63);
    units = __builtin_amdgcn_readlane(lane_sums(units), 63);
    about = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lane_sums(about)), 63));
    if (records == 0 || about > 2.1e9f) return Share{0, 0, 1, true};          // (more than the host was told of: nothing is computed)
    const int size = max(quotient(records + a.slots - 1, a.slots), a.fewest);
    // the smallest such size: `size`, or by halves where size + kSpare is one (a larger size never has more shares).  One body: code that runs once comes from far.
    int low = size, high = size + kSpare + 1, at = size, shares = 0;
    while (low < high) {
        int of_at = 0;
        for (int base = 0; base < a.b.sequences; base += 64) {
            if (a.b.sequences > 64) l = lane_of(a, base);
            of_at += l.e.units * max(1, quotient(l.e.hi - l.e.lo + at - 1, at));
        }
        of_at = __builtin_amdgcn_readlane(lane_sums(of_at), 63);
        if (of_at <= a.slots) { high = at; shares = of_at; } else { low = at + 1; }
        at = shares == 0 ? size + kSpare : (low + high) >> 1;
    }
    if (shares > 0) return slot < shares ? Share{slot * high, (slot + 1) * high, high, true} : Share{0, 0, 1, true};
    const int places = records + units * kKvBeginning, each = quotient(places + a.slots - 1, a.slots);
    return Share{(int)min((int64_t)slot * each, (int64_t)places), (int)min((int64_t)(slot + 1) * each, (int64_t)places), each, false};
}

__device__ __forceinline__ Segment segment_of(const AttendArgs &a, const Share &share, int pos, Lane l)
{
    Segment w{};
    int before = 0;
    for (int base = 0; base < a.b.sequences && !w.any; base += 64) {
        if (a.b.sequences > 64) l = lane_of(a, base);
        const int recs = l.e.hi - l.e.lo, shares = share.whole ? max(1, quotient(recs + share.size - 1, share.size)) : 1, each = share.whole ? shares * share.size : kKvBeginning + max(1, recs);
        const int mine = l.e.units * each, x = lane_sums(mine), at = pos - before - (x - mine);
        const uint64_t has = __ballot(at >= 0 && at < mine);
        if (has != 0) {
            const int src = __ffsll((unsigned long long)has) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            const int i = of(at), n = of(each), lo = of(l.e.lo), hi = of(l.e.hi);
            w.any = true;
            w.b = base + src;
            w.unit = i < n ? 0 : quotient(i, n);
            w.s.first = of(l.s.first); w.s.n = of(l.s.n); w.s.len = of(l.s.len); w.s.pos = of(l.s.pos);
            const int start = pos - (i - w.unit * n);
            w.unit_from = share.whole ? start : start + kKvBeginning;
            w.unit_to = start + n;
            w.to = min(share.last, w.unit_to);
            if (share.whole) {                               // a unit's shares are alike
                const int parts = of(shares), k = quotient(i - w.unit * n, share.size), each_part = quotient(hi - lo + parts - 1, parts);
                w.rec = lo + k * each_part;
                w.rec_to = min(hi, w.rec + each_part);
            } else {
                w.rec = lo + max(0, pos - w.unit_from);
                w.rec_to = min(hi, lo + (w.to - w.unit_from));     // a sequence that holds nothing has one record to itself that is none
            }
        }
        before += __builtin_amdgcn_readlane(x, 63);
    }
    return w;
}

// a launch has a slot for every chunk aimed at and for every unit there can be
int units_at_most(const KvBatch &b, int ratio, int unit_rows)
{
    const int64_t each = (int64_t)b.sequences * (((int64_t)b.max_new * ratio + unit_rows - 1) / unit_rows);
    const int64_t all = (b.tokens * ratio + unit_rows - 1) / unit_rows + b.sequences;
    return (int)(each < all ? each : all);
}

// more LDS than the default has to be asked for, once on every device; `asked`: a bit per device, of the kernel
inline void allow_lds(std::atomic<uint64_t> &asked, const void *kernel, int bytes)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if ((asked.load(std::memory_order_relaxed) & bit) != 0) return;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess) asked.fetch_or(bit, std::memory_order_relaxed);
}

}  // namespace

// ---- kv_prompt.hip ---------------------------------------------------------------------------
Scratch prompt_scratch(const KvShape &s, size_t at);
void launch_kv_prompt(const KvShape &s, AttendArgs a, hipStream_t st);

}  // namespace eqat
