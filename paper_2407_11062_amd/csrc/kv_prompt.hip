// Attention over the 4-bit cache for many rows: a workgroup takes 16 or 32 rows (query, head that shares a head of the cache) a wave, rebuilds 64 tokens at a time as
// binary16 in LDS, where all its waves read them, and runs both products on the matrix cores.
//
// Bound by the matrix cores, by the exponentials and by the reads of LDS, about evenly, so a key or value is rebuilt once for the rows of the workgroup, and the products
// for the scores of one tile stand between the exponentials of the one before it.  It lies in LDS in the order in which the matrix instructions' lanes take it (kv.h), which
// is the order of the cache: writes and reads are 1 KB of neighbouring bytes.
// Keys and values are halved on their way (m + s c may pass 65504 by a rounding), and held to 11 bits (2^-24 below 2^-13: of the cache's smallest steps that is one), as are
// queries with the scale of the scores in them, and p.  The running maximum is the products' addend, so that a score is an exponent as it comes, and the sum of p is one
// product more, with ones.  Scores and sums are binary32.
//
// 8192 tokens, 64 heads on 8 of 128: 1150 to 1160 us, 950 TFLOP/s where a product of 8192^3 reaches 1207.  333 tokens, 32 heads of 128: 15.9 us, of which the first tile of a
// workgroup takes 7 (launch, lengths, pages, records, each known only after the one before) and a tile 1.2.
#include "kv_work.h"

namespace eqat {
namespace {

constexpr int kTile = 64;                          // tokens in LDS at a time, two records; two tiles of keys and two of values
// p is held times 2^kRaised: up to four times the maximum stays in binary16, and what lies 2^27 below it is still rounded to all of its bits.
constexpr float kRaised = 13.0f;
// Rows of a workgroup: 256, or 64 where that leaves compute units without one; for heads of 256 it is 128 (two groups of rows a wave do not fit the registers, nor do four
// waves' shares of a tile on its way).
constexpr int kLargeWaves = 8, kSmallWaves = 4;
constexpr int large_columns(int head_dim) { return head_dim > 128 ? 1 : 2; }

__device__ __forceinline__ half2v as_half2(uint32_t w) { return __builtin_bit_cast(half2v, w); }
// two codes of a word (kv.h), pair p, halved: of 1024 + c, or 1024 + 16 c, as the bits are
__device__ __forceinline__ half2v halves_of(uint32_t w, int p)
{
    const half2v x = as_half2(((p >= 2 ? w >> 8 : w) & (p & 1 ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u);
    const _Float16 by = p & 1 ? 0.03125f : 0.5f, off = p & 1 ? -32.0f : -512.0f;
    return __builtin_elementwise_fma(x, half2v{by, by}, half2v{off, off});
}

// TEAMS of kPromptWaves waves each take the same rows and their own stretch of the tokens, in tiles of their own, and the first joins what they have.
template <int NS, int SG, int kPromptWaves, int kColumns, int TEAMS, bool CUT> __global__ __launch_bounds__(kPromptWaves * 64 * TEAMS, 2) void k_kv_prompt(const AttendArgs a)
{
    using R = KvRecord<NS, SG>;
    constexpr int kUnitRows = kPromptWaves * kColumns * 16;
    constexpr int D = R::D, G = R::G, kChunks = NS / 2, kTileBytes = kTile * D * 2, kStaged = (4 * kChunks + kPromptWaves - 1) / kPromptWaves;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds_all[];         // a team's two tiles of keys, two of values
    __shared__ uint32_t s_odd_all[TEAMS][4];                                  // tile & 3: a value of a token that is there is NaN
    const int tid = threadIdx.x, wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int team = TEAMS > 1 ? wave_all / kPromptWaves : 0, wave = TEAMS > 1 ? wave_all % kPromptWaves : wave_all;
    uint8_t *lds = lds_all + team * 4 * kTileBytes;
    uint32_t *s_odd = s_odd_all[team];
    const int head = blockIdx.x % a.heads;
    const Work w = work_of<CUT, false>(a, blockIdx.x / a.heads);
    if (!w.any) return;
    const int unit = (w.s.n * a.ratio + kUnitRows - 1) / kUnitRows - 1 - w.unit;        // the last rows, which see most, first
    // ---- this lane's rows -------------------------------------------------------------------------
    half8 q[kColumns][NS];
    float back[kColumns];
    bool fits = false;
    int seen_from[kColumns], seen_to[kColumns], query[kColumns], of_group[kColumns];
    int least_to = 0x7FFFFFFF, most_from = 0;
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        const int row = unit * kUnitRows + (wave * kColumns + t) * 16 + r;
        query[t] = quotient(row, a.ratio); of_group[t] = row - query[t] * a.ratio;
        const bool is_row = query[t] < w.s.n;
        const int pos = w.s.pos + query[t];
        seen_to[t] = !is_row ? 0 : a.causal ? min(w.s.len, pos + 1) : w.s.len;
        seen_from[t] = is_row ? window_from(pos, a.window) : 0;
        if (is_row) { least_to = min(least_to, seen_to[t]); most_from = max(most_from, seen_from[t]); }
        const bf16_t *src = static_cast<const bf16_t *>(a.q.p) + (int64_t)(w.s.first + query[t]) * a.q.token_stride + (int64_t)(head * a.ratio + of_group[t]) * a.q.head_stride;
        float top = 0.0f;
        bf16x8 x[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            x[j] = bf16x8{};
            if (is_row) x[j] = *reinterpret_cast<const bf16x8 *>(src + 32 * j + 8 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)x[j][e]));
        }
        // The row with the scale of the scores in it, 2 for the halved keys and log2(e); a power of two more, taken back from the scores, where binary16 would not hold
        // it well: in rows far larger or smaller than those of a model.
        const float scale = a.scale * 2.0f, most = chunks_max(top) * scale;
        const int fit = most > 32768.0f || (most > 0.0f && most < 0x1p-8f) ? min(max(127 - (int)(__float_as_uint(most) >> 23), -126), 100) : 0;
        const float fitted = __uint_as_float((uint32_t)(127 + fit) << 23);
        back[t] = __uint_as_float((uint32_t)(127 - fit) << 23);
        fits |= fit != 0;
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[t][j][e] = (_Float16)((float)x[j][e] * scale * fitted);
    }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) {
        least_to = min(least_to, __shfl_xor(least_to, d));
        most_from = max(most_from, __shfl_xor(most_from, d));
    }
    const bool any_fits = __any(fits);
    least_to = __builtin_amdgcn_readfirstlane(least_to);
    most_from = __builtin_amdgcn_readfirstlane(most_from);
    // ---- the records of the workgroup ---------------------------------------------------------------
    int first = w.first, last = w.last;
    {
        const int row1 = min((unit + 1) * kUnitRows, w.s.n * a.ratio) - 1;
        if (a.causal) last = min(last, ((w.s.pos + row1 / a.ratio) >> 5) + 1);
        first = max(first, window_from(w.s.pos + unit * kUnitRows / a.ratio, a.window) >> 5);
    }
    int tiles = max(0, (last - first + 1) >> 1);
    if constexpr (TEAMS > 1) {                               // as many tiles each, past the last one none that is there
        tiles = (tiles + TEAMS - 1) / TEAMS;
        first += 2 * tiles * team;
        last = min(last, first + 2 * tiles);
    }
    const int32_t *table = a.b.table + (int64_t)w.b * a.b.table_stride;
    // the next record's number in the pool; -1 where it is past the end or its page is not there.  Lane i has looked up the i-th of 64 of them.
    int ahead = 0, looked_up = -1;
    auto next_record = [&]() __attribute__((always_inline)) {
        if ((ahead & 63) == 0) {
            const int rec = first + ahead + lane, of_seq = quotient(rec, a.page_records);
            const int page = rec < last ? table[of_seq] : -1;
            looked_up = page >= 0 && page < a.pages ? (page * a.heads + head) * a.page_records + (rec - of_seq * a.page_records) : -1;
        }
        return __builtin_amdgcn_readlane(looked_up, ahead++ & 63);
    };
    // Chunks of a tile, kStaged a wave: of two records, keys' and values' chunks.  Keys are fetched for two tiles on, values for the next.  All waves issue the same loads,
    // whichever they have use for, from the pool's first record where there is none: loads under a branch would be waited for where it ends.
    constexpr int kShared = SG < 4 ? SG : 4;                 // words of a chunk of keys that share their step
    constexpr int kGroups = SG == 1 ? 2 : 1;                 // groups of a chunk of values
    uintx4 raw[kStaged], value_steps[kStaged][2 * kGroups];
    uint32_t key_steps[kStaged][4 / kShared];
    int here0 = -1, here1 = -1, next0 = -1, next1 = -1, after0 = -1, after1 = -1;            // the records of this tile, the next, the one after
    auto turn = [&]() __attribute__((always_inline)) {
        here0 = next0; here1 = next1; next0 = after0; next1 = after1;
        after0 = next_record(); after1 = next_record();
    };
    auto of = [](int a, int b, bool second) __attribute__((always_inline)) { return second ? b : a; };          // (by value: a choice of variables would put them in memory)
    // chunk k of this wave: waves that share a SIMD (w, w + 4) take one of keys and one of values where there are eight
    struct Chunk { bool is, key; int rec, i; };
    auto chunk = [&](int k) __attribute__((always_inline)) {
        const int id = (kPromptWaves == 8 && kChunks == 2 && wave >= 4 ? wave ^ 2 : wave) + k * kPromptWaves, part = id % (2 * kChunks);
        return Chunk{id < 4 * kChunks, part < kChunks, id / (2 * kChunks) & 1, part % kChunks};
    };
    auto fetch = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kStaged; ++k) {
            const Chunk x = chunk(k);
            const uint8_t *at = a.pool + (int64_t)max(of(of(next0, next1, x.rec != 0), of(after0, after1, x.rec != 0), x.key), 0) * R::kBytes;
            raw[k] = *reinterpret_cast<const uintx4 *>(at + (x.key ? R::kKeys : R::kValues) + x.i * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; e += kShared) {
                const int word = x.i * 4 + e, sub = (word / NS) & 1, j = word % NS;
                key_steps[k][e / kShared] = *reinterpret_cast<const uint32_t *>(at + R::kKeySteps + (j / SG) * 128 + (sub * 16 + r) * 4);
            }
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int h = 0; h < 2; ++h) value_steps[k][2 * g + h] = *reinterpret_cast<const uintx4 *>(at + R::kValueSteps + ((2 * x.i + g) / SG) * 128 + h * 64 + c * 16);
        }
    };
    const half2v halved = {(_Float16)0.5f, (_Float16)0.5f};
    // into LDS, keys as those of tile key_tile, values as those of value_tile
    auto rebuild = [&](int key_tile, int value_tile, bool do_keys, bool do_values) __attribute__((always_inline)) {
        uint8_t *keys = lds + (key_tile & 1) * kTileBytes, *values = lds + (2 + (value_tile & 1)) * kTileBytes;
#pragma unroll
        for (int k = 0; k < kStaged; ++k) {
            const Chunk x = chunk(k);
            if (!x.is) continue;
            if (x.key) {
                if (!do_keys || of(after0, after1, x.rec != 0) < 0) continue;          // (not there: masked, whatever stands in LDS)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int word = x.i * 4 + e, sub = word / NS, j = word % NS;
                    const half2v sm = as_half2(key_steps[k][e / kShared]), m = sm * halved;
                    uintx4 y;
#pragma unroll
                    for (int p = 0; p < 4; ++p) y[p] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(halves_of(raw[k][e], p), half2v{sm[0], sm[0]}, half2v{m[1], m[1]}));
                    *reinterpret_cast<uintx4 *>(keys + ((x.rec * 2 + sub) * NS + j) * 1024 + lane * 16) = y;
                }
            } else if (do_values) {
                // What no row sees must be a number: 0 p = 0.  A NaN that some row may see is put aside and dealt with apart.
                const int token = (first + 2 * value_tile + x.rec) * kKvRecord;
                const bool there = of(next0, next1, x.rec != 0) >= 0;
                uint32_t most = 0;                            // of the steps in the low halves: NaN is above every number
#pragma unroll
                for (int g = 0; g < 2 * kGroups; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = max(most, value_steps[k][g][e] & 0xFFFFu);
                if (__any(most >= 0x7C00u) || !there || token + kKvRecord > w.s.len) {
                    bool odd = false;
#pragma unroll
                    for (int g = 0; g < 2 * kGroups; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool is = there && token + (g & 1) * 16 + c * 4 + e < w.s.len, nan = (value_steps[k][g][e] & 0x7C00u) == 0x7C00u;
                            odd |= is && nan;
                            value_steps[k][g][e] = is && !nan ? value_steps[k][g][e] : 0u;
                        }
                    if (__any(odd) && lane == 0) s_odd[value_tile & 3] = 1u;
                }
                half2v s[kGroups][4], m[kGroups][4];
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t u = value_steps[k][2 * g + (e >> 1)][(e & 1) * 2], v = value_steps[k][2 * g + (e >> 1)][(e & 1) * 2 + 1];
                        s[g][e] = as_half2(__builtin_amdgcn_perm(v, u, 0x05040100u));
                        m[g][e] = as_half2(__builtin_amdgcn_perm(v, u, 0x07060302u)) * halved;
                    }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int n = 4 * x.i + p, g = kGroups == 2 ? p >> 1 : 0;
                    uintx4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(halves_of(raw[k][e], p), s[g][e], m[g][e]));
                    *reinterpret_cast<uintx4 *>(values + (x.rec * 2 * NS + n) * 1024 + lane * 16) = y;
                }
            }
        }
    };
    floatx4 o[kColumns][2 * NS], sum[kColumns], s[4][kColumns];
    float top[kColumns];                                     // what a score has had taken off it, in its own fitted units
    float limit[kColumns];                                   // above which a score moves it: kRaised + 2, or anything before the row has seen something
    const floatx4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const uintx4 ones = {0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        top[t] = 0.0f; limit[t] = -__builtin_inff(); sum[t] = zero;
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) o[t][n] = zero;
    }
    // the scores of 16 tokens, less top
    auto key_parts = [&](int tile, int h, uintx4 (&k)[NS]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NS; ++j) k[j] = *reinterpret_cast<const uintx4 *>(lds + (tile & 1) * kTileBytes + (h * NS + j) * 1024 + lane * 16);
    };
    auto scores = [&](int h, const uintx4 (&k)[NS]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < kColumns; ++t) s[h][t] = mfma(k[0], q[t][0], floatx4{-top[t], -top[t], -top[t], -top[t]});
#pragma unroll
        for (int j = 1; j < NS; ++j)
#pragma unroll
            for (int t = 0; t < kColumns; ++t) s[h][t] = mfma(k[j], q[t][j], s[h][t]);
    };
    if (tid < 4 * TEAMS) s_odd_all[tid >> 2][tid & 3] = 0u;
    __syncthreads();
    if (tiles > 0) {
        turn(); fetch(); rebuild(0, 0, true, false);
        turn(); fetch(); rebuild(1, 0, true, true);
        turn();                                              // this tile, the next, the one after
    }
    __syncthreads();
    if (tiles > 0) {
#pragma unroll
        for (int h = 0; h < 4; ++h) { uintx4 k[NS]; key_parts(0, h, k); scores(h, k); }
        __syncthreads();                                     // all waves have read the first tile's keys: the loop's first rebuild puts the third tile's there
    }
    // A tile's turn reads the keys of the next tile and its own values, and writes the keys of the one after into the place of its own, which nobody reads any more
    // since the barrier before (here, or at the turn's end), and the next tile's values into that of the last tile's.
    for (int tile = 0; tile < tiles; ++tile) {
        fetch();                                              // keys of tile + 2, values of tile + 1
        const int token0 = (first + 2 * tile) * kKvRecord;
        const uint32_t odd = s_odd[tile & 3];
        const bool absent0 = here0 < 0, absent1 = here1 < 0;
        uintx4 k_now[NS], k_next[NS];
        key_parts(tile + 1, 0, k_now);
        if (any_fits || token0 < most_from || token0 + kTile > least_to || absent0 || absent1) {
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int t = 0; t < kColumns; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = token0 + h * 16 + c * 4 + i;
                        const bool seen = at >= seen_from[t] && at < seen_to[t] && !(h < 2 ? absent0 : absent1);
                        s[h][t][i] = seen ? s[h][t][i] * back[t] : -__builtin_inff();
                    }
        }
        bool move = false;
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
            float most = s[0][t][0];
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s[h][t][i]);
            move |= most > limit[t];
        }
        if (__any(move)) {
            // the maximum moves: always to the first tile's, later where a score passes it by 2.  (Scores of 2^22 and more have no room for kRaised in binary32.)
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                float most = s[0][t][0];
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most = fmaxf(most, s[h][t][i]);
                most = chunks_max(most);
                const bool moves = most > limit[t];
                const float by = moves ? fabsf(most) < 4194304.0f ? most - kRaised : most : 0.0f, down = limit[t] > 0.0f ? exp2_of(-by) : 0.0f;
                top[t] += by / back[t];
                limit[t] = moves ? kRaised + 2.0f : limit[t];
                sum[t] *= down;
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) o[t][n] *= down;
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[h][t][i] -= by;
            }
        }
        // Exponentials of 16 tokens beside the products for the 16 before them of the next tile (past the last tile: of whatever stands there, not looked at), each
        // step's parts of keys, then of values, read a step ahead
        uint32_t p[kColumns][2][4];
        auto exponentials = [&](int h) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = exp2_of(s[h][t][i]);
                p[t][h >> 1][(h & 1) * 2] = __builtin_bit_cast(uint32_t, half2v{(_Float16)e[0], (_Float16)e[1]});
                p[t][h >> 1][(h & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, half2v{(_Float16)e[2], (_Float16)e[3]});
            }
        };
        constexpr int kAhead = NS < 4 || (SG == 1 && kColumns == 2) ? 2 : 4;             // parts of values read ahead: as many as the registers hold
        const uint8_t *values = lds + (2 + (tile & 1)) * kTileBytes;
        uintx4 v_now[kAhead], v_next[kAhead];
        auto value_parts = [&](int n, uintx4 (&v)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) v[i] = *reinterpret_cast<const uintx4 *>(values + (n + i) * 1024 + lane * 16);
        };
        __builtin_amdgcn_s_setprio(1);                        // of the two waves of a SIMD the one at its products goes first (1.2 ms -> 1.18 at 8192 tokens)
        exponentials(0);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            __builtin_amdgcn_sched_barrier(0);
            if (h < 3) { key_parts(tile + 1, h + 1, k_next); exponentials(h + 1); }
            else value_parts(0, v_now);
            scores(h, k_now);
#pragma unroll
            for (int j = 0; j < NS; ++j) k_now[j] = k_next[j];
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < NS * kColumns; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 4 / NS > 0 ? 4 / NS : 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
            }
        }
        half8 ph[kColumns][2];
#pragma unroll
        for (int t = 0; t < kColumns; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ph[t][h] = __builtin_bit_cast(half8, uintx4{p[t][h][0], p[t][h][1], p[t][h][2], p[t][h][3]});
                sum[t] = mfma(ones, ph[t][h], sum[t]);
            }
#pragma unroll
        for (int n = 0; n < 4 * NS; n += kAhead) {
            __builtin_amdgcn_sched_barrier(0);
            if (n + kAhead < 4 * NS) value_parts(n + kAhead, v_next);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int t = 0; t < kColumns; ++t) o[t][(n + i) % (2 * NS)] = mfma(v_now[i], ph[t][(n + i) / (2 * NS)], o[t][(n + i) % (2 * NS)]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) v_now[i] = v_next[i];
            __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (__builtin_amdgcn_readfirstlane(odd) != 0u) {
            // NaN among the values: it reaches the rows that see its token, in the elements of its group
            for (int t64 = 0; t64 < kTile; ++t64) {
                const int at = token0 + t64;
                const int rec = of(here0, here1, t64 >= kKvRecord);
                if (rec < 0 || at >= w.s.len) continue;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t step = *reinterpret_cast<const uint32_t *>(a.pool + (int64_t)rec * R::kBytes + R::kValueSteps + g * 128 + (t64 & 31) * 4);
                    if ((step & 0x7C00u) != 0x7C00u) continue;
#pragma unroll
                    for (int t = 0; t < kColumns; ++t)
#pragma unroll
                        for (int n = 2 * g * SG; n < 2 * (g + 1) * SG; ++n)
                            if (at >= seen_from[t] && at < seen_to[t]) o[t][n] = floatx4{1.0f, 1.0f, 1.0f, 1.0f} * __builtin_nanf("");
                }
            }
        }
        if (wave == 0 && lane == 0) s_odd[(tile + 3) & 3] = 0u;             // read a tile ago, set again two tiles on
        rebuild(tile + 2, tile + 1, true, true);
        turn();
        __syncthreads();
    }
    // ---- results --------------------------------------------------------------------------------------
    float total[kColumns];
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        total[t] = sum[t][0];
        top[t] = limit[t] > 0.0f ? top[t] * back[t] : -3.0e38f;
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) o[t][n] *= 2.0f;
    }
    if constexpr (TEAMS > 1) {
        // the other team's through its tiles, lane by lane: rows and elements are the same
        static_assert(TEAMS == 2 && kPromptWaves * kColumns * (2 * NS + 1) * 1024 <= 4 * kTileBytes, "the team's sums and results fit its tiles");
        floatx4 *theirs = reinterpret_cast<floatx4 *>(lds_all + 4 * kTileBytes) + wave * kColumns * (2 * NS + 1) * 64 + lane;
        if (team == 1) {
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) theirs[(t * (2 * NS + 1) + n) * 64] = o[t][n];
                theirs[(t * (2 * NS + 1) + 2 * NS) * 64] = floatx4{top[t], total[t], 0.0f, 0.0f};
            }
        }
        __syncthreads();
        if (team == 1) return;
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
            const floatx4 stats = theirs[(t * (2 * NS + 1) + 2 * NS) * 64];
            const float next = fmaxf(top[t], stats[0]), f = exp2_of(top[t] - next), g = exp2_of(stats[0] - next);
            top[t] = next;
            total[t] = __builtin_fmaf(stats[1], g, total[t] * f);
#pragma unroll
            for (int n = 0; n < 2 * NS; ++n) {
                const floatx4 x = theirs[(t * (2 * NS + 1) + n) * 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[t][n][i] = __builtin_fmaf(x[i], g, o[t][n][i] * f);
            }
        }
    }
    if constexpr (CUT) {
        if (w.chunks > 1) {                                  // the join is a launch of its own: its bytes (a part is 32 KB and more) are too many for one workgroup
            constexpr uint32_t kPart = kUnitRows * D * 4, kStats = kUnitRows * 8;
            const int64_t mine = (int64_t)w.part * a.heads + head;
            uint8_t *base = reinterpret_cast<uint8_t *>(a.parts), *stats = base + 2 * (int64_t)a.target * a.heads * kPart + mine * kStats;
            base += mine * kPart;
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                const int row = (wave * kColumns + t) * 16 + r;
#pragma unroll
                for (int j = 0; j < NS; ++j) {
                    float *to = reinterpret_cast<float *>(base) + row * D + 32 * j + 8 * c;
                    *reinterpret_cast<floatx4 *>(to) = floatx4{o[t][2 * j][0], o[t][2 * j + 1][0], o[t][2 * j][1], o[t][2 * j + 1][1]};
                    *reinterpret_cast<floatx4 *>(to + 4) = floatx4{o[t][2 * j][2], o[t][2 * j + 1][2], o[t][2 * j][3], o[t][2 * j + 1][3]};
                }
                if (c == 0) *reinterpret_cast<floatx2 *>(stats + row * 8) = floatx2{top[t], total[t]};
            }
            return;
        }
    }
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        if (query[t] >= w.s.n) continue;
        const int oh = head * a.ratio + of_group[t];
        const float inv = total[t] == 0.0f ? 0.0f : 1.0f / total[t];
        bf16_t *out = static_cast<bf16_t *>(a.out.p) + (int64_t)(w.s.first + query[t]) * a.out.token_stride + (int64_t)oh * a.out.head_stride;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            bf16x8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (bf16_t)(o[t][2 * j + (i & 1)][i >> 1] * inv);
            *reinterpret_cast<bf16x8 *>(out + 32 * j + 8 * c) = v;
        }
        if (a.lse != nullptr && c == 0)
            a.lse[(int64_t)(w.s.first + query[t]) * ((int64_t)a.heads * a.ratio) + oh] = total[t] == 0.0f ? -__builtin_inff() : (top[t] + __builtin_log2f(total[t])) * 0.6931471805599453f;
    }
}

// Sixteen rows of a unit that was cut, from its parts.
template <int D> __global__ __launch_bounds__(256) void k_kv_join(const AttendArgs a)
{
    constexpr int kOut = D / 16;                             // elements of a thread
    const int groups = 1 << (a.unit_bits - 4), head = blockIdx.x % a.heads, group = blockIdx.x / a.heads % groups, rows = 1 << a.unit_bits;
    const Work w = work_of<true, true>(a, blockIdx.x / (a.heads * groups));
    if (!w.any || w.chunks < 2) return;
    const int unit = ((w.s.n * a.ratio + rows - 1) >> a.unit_bits) - 1 - w.unit;        // as in the kernel above
    const int row = group * 16 + (threadIdx.x >> 4), d0 = (threadIdx.x & 15) * kOut;
    const int row_all = unit * rows + row, query = quotient(row_all, a.ratio), oh = head * a.ratio + (row_all - query * a.ratio);
    if (query >= w.s.n) return;
    const float *parts = a.parts + row * D + d0, *stats = a.parts + 2 * (int64_t)a.target * a.heads * rows * D + row * 2;
    float m = -3.0e38f, l = 0.0f, x[kOut] = {};
#pragma unroll 4
    for (int k = 0; k < w.chunks; ++k) {
        const int64_t from = (int64_t)(w.part + k) * a.heads + head;
        const floatx2 ml = *reinterpret_cast<const floatx2 *>(stats + from * rows * 2);
        floatx4 v[kOut / 4];
#pragma unroll
        for (int e = 0; e < kOut / 4; ++e) v[e] = *reinterpret_cast<const floatx4 *>(parts + from * rows * D + 4 * e);
        const float next = fmaxf(m, ml[0]), f = exp2_of(m - next), g = exp2_of(ml[0] - next);
        m = next;
        l = __builtin_fmaf(ml[1], g, l * f);
#pragma unroll
        for (int e = 0; e < kOut; ++e) x[e] = __builtin_fmaf(v[e / 4][e % 4], g, x[e] * f);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bf16_t *out = static_cast<bf16_t *>(a.out.p) + (int64_t)(w.s.first + query) * a.out.token_stride + (int64_t)oh * a.out.head_stride + d0;
#pragma unroll
    for (int e = 0; e < kOut; e += 4) {
        bf16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (bf16_t)(x[e + i] * inv);
        *reinterpret_cast<bf16x4 *>(out + e) = v;
    }
    if (a.lse != nullptr && d0 == 0)
        a.lse[(int64_t)(w.s.first + query) * ((int64_t)a.heads * a.ratio) + oh] = l == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

struct PromptPlan { int rows, target; bool small, cut, teams; };    // rows of a unit; chunks aimed at for a head of the cache; workgroups of few rows; units may be cut; two teams

template <int NS, int SG, int W, int C, int TEAMS, bool CUT> void launch_t(const AttendArgs &a, bool join, int units, hipStream_t st)
{
    constexpr int smem = TEAMS * 4 * kTile * 32 * NS * 2;
    static std::atomic<uint64_t> asked{0};
    allow_lds(asked, reinterpret_cast<const void *>(&k_kv_prompt<NS, SG, W, C, TEAMS, CUT>), smem);
    k_kv_prompt<NS, SG, W, C, TEAMS, CUT><<<dim3((unsigned)a.slots * (unsigned)a.heads), W * 64 * TEAMS, smem, st>>>(a);
    if (join) k_kv_join<32 * NS><<<dim3((unsigned)units * (W * C) * (unsigned)a.heads), 256, 0, st>>>(a);
}
template <int NS, int SG> void launch(const AttendArgs &a, const PromptPlan &p, int units, hipStream_t st)
{
    constexpr int kColumns = large_columns(32 * NS);
    if (!p.small) return launch_t<NS, SG, kLargeWaves, kColumns, 1, false>(a, false, units, st);
    if constexpr (NS < 8)
        if (p.teams) return launch_t<NS, SG, kSmallWaves, 1, 2, false>(a, false, units, st);
    launch_t<NS, SG, NS == 8 ? kLargeWaves : kSmallWaves, 1, 1, true>(a, p.cut, units, st);
}

// Workgroups of 256 rows where there is one for every compute unit, else of 64, two to a compute unit.  Where even those do not take half the places, sequences of more than
// kFewest records are cut, and joined in a launch of its own (3 us).  Where caches are shorter and there is no more than one workgroup for a compute unit, it is two teams
// (333 tokens, 32 heads 16.1 us for 16.8, 100 rows behind 411 tokens 17.2 for 20.4; one tile, 11.0 for 9.2, is one team's).  Heads of 256: two teams' tiles do not fit LDS.
constexpr int kFewest = 16;
PromptPlan prompt_plan(const KvShape &s, const KvBatch &b, int ratio)
{
    const int large = kLargeWaves * large_columns(s.head_dim) * 16;
    PromptPlan p;
    p.small = (int64_t)units_at_most(b, ratio, large) * s.heads < 256;
    p.rows = p.small && s.head_dim <= 128 ? kSmallWaves * 16 : large;
    p.target = ((s.head_dim <= 128 ? 512 : 256) + s.heads - 1) / s.heads;
    p.cut = p.small && units_at_most(b, ratio, p.rows) < p.target / 2 && b.max_len > kFewest * kKvRecord;
    p.teams = p.small && !p.cut && s.head_dim <= 128 && b.max_len > kTile && (int64_t)units_at_most(b, ratio, p.rows) * s.heads <= 256;
    return p;
}
}  // namespace

Scratch prompt_scratch(const KvShape &s, size_t at)
{
    const KvBatch none{};                                     // no units: the plan of the most that is cut
    const PromptPlan p = prompt_plan(s, none, 1);
    return scratch_of(at, (size_t)p.target * s.heads, false, p.rows, s.head_dim);
}

void launch_kv_prompt(const KvShape &s, AttendArgs a, hipStream_t st)
{
    const PromptPlan p = prompt_plan(s, a.b, a.ratio);
    const int units = units_at_most(a.b, a.ratio, p.rows);
    a.unit_bits = __builtin_ctz(p.rows);
    a.fewest = p.cut ? kFewest : 1 << 30;
    a.target = p.target;
    a.slots = (p.cut ? p.target : 0) + units;
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(a, p, units, st); else launch<2, 2>(a, p, units, st); break;
    case 128: if (sg == 1) launch<4, 1>(a, p, units, st); else if (sg == 2) launch<4, 2>(a, p, units, st); else launch<4, 4>(a, p, units, st); break;
    default:
        if (sg == 1) launch<8, 1>(a, p, units, st); else if (sg == 2) launch<8, 2>(a, p, units, st);
        else if (sg == 4) launch<8, 4>(a, p, units, st); else launch<8, 8>(a, p, units, st);
    }
}

}  // namespace eqat
