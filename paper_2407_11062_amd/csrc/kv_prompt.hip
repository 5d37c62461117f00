// Attention over the 4-bit cache for many rows: a workgroup takes 32 rows (query, head that shares a head of the cache) a wave, rebuilds 64 tokens at a time as binary16
// in LDS, where all its waves read them, and runs both products on the matrix cores.
//
// Bound by the matrix cores and by the exponentials beside them, so a key or value is rebuilt once for the 256 rows of the workgroup: three instructions for two elements.
// It lies in LDS in the order in which the matrix instructions' lanes take it (kv.h), which is the order of the cache: writes and reads are 1 KB of neighbouring bytes.
// Keys and values are halved on their way (m + s c may pass 65504 by a rounding), and held to 11 bits; scores, softmax and sums are binary32, p is binary16.
#include "kv_work.h"

namespace eqat {
namespace {

constexpr int kTile = 64;                          // tokens in LDS at a time, two records; two tiles of them
constexpr int kPromptWaves = 8;
// groups of 16 rows of a wave: heads of 256 leave the registers for one
constexpr int columns_of(int head_dim) { return head_dim > 128 ? 1 : 2; }

__device__ __forceinline__ half2v as_half2(uint32_t w) { return __builtin_bit_cast(half2v, w); }
// two codes of a word (kv.h), pair p, as numbers
__device__ __forceinline__ half2v codes_of(uint32_t w, int p)
{
    const half2v x = as_half2(((p >= 2 ? w >> 8 : w) & (p & 1 ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u);       // 1024 + c, 1024 + 16 c
    const half2v sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f}, off = {(_Float16)-64.0f, (_Float16)-64.0f}, off1 = {(_Float16)-1024.0f, (_Float16)-1024.0f};
    return p & 1 ? __builtin_elementwise_fma(x, sixteenth, off) : x + off1;
}

template <int NS, int SG> __global__ __launch_bounds__(kPromptWaves * 64, 2) void k_kv_prompt(const AttendArgs a)
{
    using R = KvRecord<NS, SG>;
    constexpr int kColumns = columns_of(32 * NS), kUnitRows = kPromptWaves * kColumns * 16;
    constexpr int D = R::D, G = R::G, kChunks = NS / 2, kTileBytes = kTile * D * 2, kStaged = (4 * kChunks + kPromptWaves - 1) / kPromptWaves;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];             // two tiles: keys, values
    __shared__ uint32_t s_odd[4];                                             // tile & 3: a value of a token that is there is NaN
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, c = lane >> 4;
    const int head = blockIdx.x % a.heads;
    const Work w = work_of(a, blockIdx.x / a.heads);
    if (!w.any) return;
    const int unit = (w.s.n * a.ratio + kUnitRows - 1) / kUnitRows - 1 - w.unit;        // the last rows, which see most, first
    // ---- this lane's rows -------------------------------------------------------------------------
    half8 q[kColumns][NS];
    float k_scale[kColumns];
    int seen_from[kColumns], seen_to[kColumns], query[kColumns], of_group[kColumns];
    int most_to = 0, least_to = 0x7FFFFFFF, most_from = 0, least_from = 0x7FFFFFFF;
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        const int row = unit * kUnitRows + (wave * kColumns + t) * 16 + r;
        query[t] = row / a.ratio; of_group[t] = row - query[t] * a.ratio;
        const bool is_row = query[t] < w.s.n;
        const int pos = w.s.len - w.s.n + query[t];
        seen_to[t] = !is_row ? 0 : a.causal ? min(w.s.len, pos + 1) : w.s.len;
        seen_from[t] = is_row && a.window > 0 ? max(0, pos - a.window + 1) : 0;
        if (is_row) {
            most_to = max(most_to, seen_to[t]); least_to = min(least_to, seen_to[t]);
            most_from = max(most_from, seen_from[t]); least_from = min(least_from, seen_from[t]);
        }
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
        const int up = min(max(135 - (int)(__float_as_uint(chunks_max(top)) >> 23), -100), 100);         // the row's largest element in [2^8, 2^9)
        const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[t][j][e] = (_Float16)((float)x[j][e] * scale);
        k_scale[t] = a.scale * 2.0f * __uint_as_float((uint32_t)(127 - up) << 23);
    }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) {
        most_to = max(most_to, __shfl_xor(most_to, d)); least_to = min(least_to, __shfl_xor(least_to, d));
        most_from = max(most_from, __shfl_xor(most_from, d)); least_from = min(least_from, __shfl_xor(least_from, d));
    }
    most_to = __builtin_amdgcn_readfirstlane(most_to); least_to = __builtin_amdgcn_readfirstlane(least_to);
    most_from = __builtin_amdgcn_readfirstlane(most_from); least_from = __builtin_amdgcn_readfirstlane(least_from);
    // ---- the records of the workgroup ---------------------------------------------------------------
    int first = w.first, last = w.last;
    {
        const int row1 = min((unit + 1) * kUnitRows, w.s.n * a.ratio) - 1;
        if (a.causal) last = min(last, (w.s.len - w.s.n + row1 / a.ratio + 32) >> 5);
        if (a.window > 0) first = max(first, max(0, w.s.len - w.s.n + unit * kUnitRows / a.ratio - a.window + 1) >> 5);
    }
    const int tiles = max(0, (last - first + 1) >> 1);
    const int32_t *table = a.b.table + (int64_t)w.b * a.b.table_stride;
    // the next record's place; nullptr where it is past the end or its page is not there
    int next_rec = first, next_page = first / a.page_records, in_page = first - next_page * a.page_records;
    auto next_record = [&]() -> const uint8_t * {
        const uint8_t *at = nullptr;
        if (next_rec < last) {
            const int page = __builtin_amdgcn_readfirstlane(table[next_page]);
            if (page >= 0 && page < a.pages) at = a.pool + (((int64_t)page * a.heads + head) * a.page_records + in_page) * R::kBytes;
        }
        ++next_rec;
        if (++in_page == a.page_records) { in_page = 0; ++next_page; }
        return at;
    };
    // Chunks of a tile, kStaged a wave: of two records, keys' and values' chunks
    constexpr int kShared = SG < 4 ? SG : 4;                 // words of a chunk of keys that share their step
    uintx4 raw[kStaged], steps[kStaged][4];
    const uint8_t *place[2];                                 // of the records of the tile fetched last
    auto fetch = [&]() {
        place[0] = next_record();
        place[1] = next_record();
#pragma unroll
        for (int k = 0; k < kStaged; ++k) {
            const int id = wave + k * kPromptWaves, rec = id / (2 * kChunks), part = id % (2 * kChunks), i = part % kChunks;
            if (id >= 4 * kChunks) continue;
            const uint8_t *at = place[rec];
            if (at == nullptr) continue;
            if (part < kChunks) {
                raw[k] = *reinterpret_cast<const uintx4 *>(at + R::kKeys + i * 1024 + lane * 16);
#pragma unroll
                for (int e = 0; e < 4; e += kShared) {
                    const int word = i * 4 + e, sub = word / NS, j = word % NS;
                    steps[k][0][e] = *reinterpret_cast<const uint32_t *>(at + R::kKeySteps + (j / SG) * 128 + (sub * 16 + r) * 4);
                }
            } else {
                raw[k] = *reinterpret_cast<const uintx4 *>(at + R::kValues + i * 1024 + lane * 16);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    steps[k][h] = *reinterpret_cast<const uintx4 *>(at + R::kValueSteps + (2 * i / SG) * 128 + h * 64 + c * 16);
                    if constexpr (SG == 1) steps[k][2 + h] = *reinterpret_cast<const uintx4 *>(at + R::kValueSteps + (2 * i + 1) * 128 + h * 64 + c * 16);
                }
            }
        }
    };
    const half2v halved = {(_Float16)0.5f, (_Float16)0.5f};
    auto rebuild = [&](int tile) {
        uint8_t *keys = lds + (tile & 1) * 2 * kTileBytes, *values = keys + kTileBytes;
#pragma unroll
        for (int k = 0; k < kStaged; ++k) {
            const int id = wave + k * kPromptWaves, rec = id / (2 * kChunks), part = id % (2 * kChunks), i = part % kChunks;
            if (id >= 4 * kChunks) continue;
            if (part < kChunks) {
                if (place[rec] == nullptr) continue;         // masked, whatever stands there
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int word = i * 4 + e, sub = word / NS, j = word % NS;
                    const half2v sm = as_half2(steps[k][0][e & -kShared]) * halved, s = {sm[0], sm[0]}, m = {sm[1], sm[1]};
                    uintx4 x;
#pragma unroll
                    for (int p = 0; p < 4; ++p) x[p] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(codes_of(raw[k][e], p), s, m));
                    *reinterpret_cast<uintx4 *>(keys + ((rec * 2 + sub) * NS + j) * 1024 + lane * 16) = x;
                }
            } else {
                // what no row sees must be a number: 0 p = 0.  A NaN that some row may see is put aside and dealt with apart.
                const int token = (first + 2 * tile + rec) * kKvRecord + c * 4;
                bool odd = false;
                half2v s[SG == 1 ? 2 : 1][4], m[SG == 1 ? 2 : 1][4];
#pragma unroll
                for (int g = 0; g < (SG == 1 ? 2 : 1); ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t u[2];
#pragma unroll
                        for (int o = 0; o < 2; ++o) {
                            const int at = (e & 1) * 2 + o;
                            u[o] = steps[k][2 * g + (e >> 1)][at];
                            const bool is = place[rec] != nullptr && token + (e >> 1) * 16 + at < w.s.len, nan = (u[o] & 0x7C00u) == 0x7C00u;
                            odd |= is && nan;
                            u[o] = is && !nan ? u[o] : 0u;
                        }
                        s[g][e] = as_half2(__builtin_amdgcn_perm(u[1], u[0], 0x05040100u)) * halved;
                        m[g][e] = as_half2(__builtin_amdgcn_perm(u[1], u[0], 0x07060302u)) * halved;
                    }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const int n = 4 * i + p, g = SG == 1 ? p >> 1 : 0;
                    uintx4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(codes_of(raw[k][e], p), s[g][e], m[g][e]));
                    *reinterpret_cast<uintx4 *>(values + (rec * 2 * NS + n) * 1024 + lane * 16) = x;
                }
                if (__any(odd) && lane == 0) s_odd[tile & 3] = 1u;
            }
        }
    };
    floatx4 o[kColumns][2 * NS];
    float top[kColumns], total[kColumns];
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        top[t] = -3.0e38f; total[t] = 0.0f;
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) o[t][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (tid < 4) s_odd[tid] = 0u;
    __syncthreads();
    bool absent0 = true, absent1 = true;                     // of the tile in LDS
    if (tiles > 0) { fetch(); rebuild(0); absent0 = place[0] == nullptr; absent1 = place[1] == nullptr; }
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) fetch();
        const int token0 = (first + 2 * tile) * kKvRecord;
        const uint8_t *keys = lds + (tile & 1) * 2 * kTileBytes, *values = keys + kTileBytes;
        if (token0 < most_to && token0 + kTile > least_from) {                // some row of the wave sees some of it
            const uint32_t odd = s_odd[tile & 3];
            floatx4 s[4][kColumns];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
#pragma unroll
                for (int t = 0; t < kColumns; ++t) s[h][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < NS; ++j) {
                    const uintx4 k = *reinterpret_cast<const uintx4 *>(keys + (h * NS + j) * 1024 + lane * 16);
#pragma unroll
                    for (int t = 0; t < kColumns; ++t) s[h][t] = mfma(k, q[t][j], s[h][t]);
                }
            }
            if (token0 < most_from || token0 + kTile > least_to || absent0 || absent1) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int t = 0; t < kColumns; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int at = token0 + h * 16 + c * 4 + i;
                            const bool seen = at >= seen_from[t] && at < seen_to[t] && !(h < 2 ? absent0 : absent1);
                            s[h][t][i] = seen ? s[h][t][i] : -__builtin_inff();
                        }
            }
            uint32_t p[kColumns][2][4];
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                float most = s[0][t][0];
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most = fmaxf(most, s[h][t][i]);
                most = chunks_max(most) * k_scale[t];
                if (__any(most > top[t] + 2.0f)) {
                    const float next = fmaxf(top[t], most), down = exp2_of(top[t] - next);
                    top[t] = next;
                    total[t] *= down;
#pragma unroll
                    for (int n = 0; n < 2 * NS; ++n) o[t][n] *= down;
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        e[i] = exp2_of(__builtin_fmaf(s[h][t][i], k_scale[t], -top[t]));
                        total[t] += e[i];
                    }
                    p[t][h >> 1][(h & 1) * 2] = __builtin_bit_cast(uint32_t, half2v{(_Float16)e[0], (_Float16)e[1]});
                    p[t][h >> 1][(h & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, half2v{(_Float16)e[2], (_Float16)e[3]});
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) {
                    const uintx4 v = *reinterpret_cast<const uintx4 *>(values + (h * 2 * NS + n) * 1024 + lane * 16);
#pragma unroll
                    for (int t = 0; t < kColumns; ++t)
                        o[t][n] = mfma(v, __builtin_bit_cast(half8, uintx4{p[t][h][0], p[t][h][1], p[t][h][2], p[t][h][3]}), o[t][n]);
                }
            if (__builtin_amdgcn_readfirstlane(odd) != 0u) {
                // NaN among the values: it reaches the rows that see its token, in the elements of its group
                for (int t64 = 0; t64 < kTile; ++t64) {
                    const int at = token0 + t64;
                    if ((t64 < 32 ? absent0 : absent1) || at >= w.s.len) continue;
                    const int of_seq = (at >> 5) / a.page_records, page = __builtin_amdgcn_readfirstlane(table[of_seq]);
                    const uint8_t *rec = a.pool + (((int64_t)page * a.heads + head) * a.page_records + ((at >> 5) - of_seq * a.page_records)) * R::kBytes;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const uint32_t step = *reinterpret_cast<const uint32_t *>(rec + R::kValueSteps + g * 128 + (t64 & 31) * 4);
                        if ((step & 0x7C00u) != 0x7C00u) continue;
#pragma unroll
                        for (int t = 0; t < kColumns; ++t)
#pragma unroll
                            for (int n = 2 * g * SG; n < 2 * (g + 1) * SG; ++n)
                                if (at >= seen_from[t] && at < seen_to[t]) o[t][n] = floatx4{1.0f, 1.0f, 1.0f, 1.0f} * __builtin_nanf("");
                    }
                }
            }
        }
        if (tid == 0) s_odd[(tile + 3) & 3] = 0u;             // read a tile ago, set again two tiles on
        if (tile + 1 < tiles) { rebuild(tile + 1); absent0 = place[0] == nullptr; absent1 = place[1] == nullptr; }
        __syncthreads();
    }
    // ---- results --------------------------------------------------------------------------------------
#pragma unroll
    for (int t = 0; t < kColumns; ++t) {
        total[t] = chunks_sum(total[t]);
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) o[t][n] *= 2.0f;
    }
    if (w.chunks > 1) {
        // as in the streamed kernel: parts and counter at device scope, the last workgroup to arrive adds up all parts in their order
        __shared__ uint32_t s_last;
        constexpr uint32_t kPart = kUnitRows * D * 4, kStats = kUnitRows * 8;
        uint8_t *base = reinterpret_cast<uint8_t *>(a.parts), *stats = base + 2 * (int64_t)a.target * a.heads * kPart;
        {
            const int64_t mine = (int64_t)w.part * a.heads + head;
            const __amdgpu_buffer_rsrc_t dst = make_rsrc(base + mine * kPart, kPart), st = make_rsrc(stats + mine * kStats, kStats);
#pragma unroll
            for (int t = 0; t < kColumns; ++t) {
                const int row = (wave * kColumns + t) * 16 + r;
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) {
                    intx4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = __float_as_int(o[t][n][i]);
                    __builtin_amdgcn_raw_buffer_store_b128(v, dst, (row * D + n * 16 + c * 4) * 4, 0, kAuxDeviceScope);
                }
                const intx2 v = {__float_as_int(top[t]), __float_as_int(total[t])};
                if (c == 0) __builtin_amdgcn_raw_buffer_store_b64(v, st, row * 8, 0, kAuxDeviceScope);
            }
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
#pragma unroll
        for (int t = 0; t < kColumns; ++t) {
            const int row = (wave * kColumns + t) * 16 + r;
            top[t] = -3.0e38f; total[t] = 0.0f;
#pragma unroll
            for (int n = 0; n < 2 * NS; ++n) o[t][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < w.chunks; ++k) {
                const int64_t from = (int64_t)(w.part - w.chunk + k) * a.heads + head;
                const __amdgpu_buffer_rsrc_t src = make_rsrc(base + from * kPart, kPart), st = make_rsrc(stats + from * kStats, kStats);
                const intx2 ml = __builtin_amdgcn_raw_buffer_load_b64(st, row * 8, 0, kAuxDeviceScope);
                const float next = fmaxf(top[t], __int_as_float(ml[0])), f = exp2_of(top[t] - next), g = exp2_of(__int_as_float(ml[0]) - next);
                top[t] = next;
                total[t] = __builtin_fmaf(__int_as_float(ml[1]), g, total[t] * f);
#pragma unroll
                for (int n = 0; n < 2 * NS; ++n) {
                    const intx4 v = __builtin_amdgcn_raw_buffer_load_b128(src, (row * D + n * 16 + c * 4) * 4, 0, kAuxDeviceScope);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][n][i] = __builtin_fmaf(__int_as_float(v[i]), g, o[t][n][i] * f);
                }
            }
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

template <int NS, int SG> void launch(const AttendArgs &a, hipStream_t st)
{
    constexpr int smem = 2 * 2 * kTile * 32 * NS * 2;
    allow_lds(reinterpret_cast<const void *>(&k_kv_prompt<NS, SG>), smem);
    k_kv_prompt<NS, SG><<<dim3((unsigned)a.slots * (unsigned)a.heads), kPromptWaves * 64, smem, st>>>(a);
}

}  // namespace

int prompt_target(const KvShape &s) { return (256 + s.heads - 1) / s.heads; }        // a workgroup on every compute unit
int prompt_unit_rows(const KvShape &s) { return kPromptWaves * columns_of(s.head_dim) * 16; }

void launch_kv_prompt(const KvShape &s, AttendArgs a, hipStream_t st)
{
    const int rows = prompt_unit_rows(s);
    a.unit_bits = __builtin_ctz(rows);
    a.fewest = 8;
    a.target = prompt_target(s);
    a.slots = a.target + units_at_most(a.b, a.ratio, rows);
    const int sg = s.group / 32;
    switch (s.head_dim) {
    case 64: if (sg == 1) launch<2, 1>(a, st); else launch<2, 2>(a, st); break;
    case 128: if (sg == 1) launch<4, 1>(a, st); else if (sg == 2) launch<4, 2>(a, st); else launch<4, 4>(a, st); break;
    default:
        if (sg == 1) launch<8, 1>(a, st); else if (sg == 2) launch<8, 2>(a, st); else if (sg == 4) launch<8, 4>(a, st); else launch<8, 8>(a, st);
    }
}

}  // namespace eqat
