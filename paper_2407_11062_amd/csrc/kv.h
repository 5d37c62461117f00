// The key-value cache in 4 bits: what its kernels share.
//
// A pool holds pages; a page holds, head after head, records of 32 tokens (a multiple of them makes a page).  A record is what one wave takes in one step:
//   keys' codes, values' codes    16 D bytes each, in the order in which the matrix instructions' lanes take them (below)
//   keys' steps, values' steps    [G][32] words each: s in the low half of a word, m in the high half, both binary16, of (group, token)
// A wave's lane l is (r, c) = (l % 16, l / 16).  v_mfma_f32_16x16x32_f16 takes eight k-elements of row (or column) r from every lane, those of chunk c; sums come back
// as column r, rows 4 c .. 4 c + 3.
//   Keys are the rows of S^T = K^ Q^T: lane (r, c) takes tokens r and 16 + r, and of 32-element step j the elements 32 j + 8 c .. + 7: one word, element e in
//     half e & 1, nibble e >> 1.
//   Values are transposed for O^T = V^T P^T: S^T left lane (r, c) the tokens 4 c .. 4 c + 3 and 16 + 4 c .. + 3 of column r, so those are its eight k-elements, and
//     as row r of product n it takes element 32 (n / 2) + 2 r + n % 2 (16 elements of one group of 32 or more): a word holds, for two neighbouring tokens, one half
//     each, the elements of products 4 a .. 4 a + 3 in its nibbles.
// Neither scores nor probabilities ever change lanes.
//
// A code is read as a binary16 number without a conversion: the nibble in bits 0 - 3 of a half is c 2^-24, in bits 4 - 7 it is c 2^-20, both denormal, which the
// matrix instructions take exactly.  A word gives its eight codes in one shift and four masks.
#pragma once
#include "common.h"

namespace eqat {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

constexpr int kKvRecord = 32;        // tokens
constexpr int kKvBeginning = 32;     // records' time that the beginning and end of a unit take (kv_work.h)
constexpr double kKvMostPlaces = 2.0e9;   // records and beginnings of all units of a call, counted in 32 bits

struct KvShape {
    int heads, head_dim, group, groups, page_records;
    int64_t pages;
    bool act_bf16;
};
// NS steps of 32 elements to a head, SG of them to a group
template <int NS, int SG> struct KvRecord {
    static constexpr int D = 32 * NS, G = NS / SG;
    static constexpr int kKeys = 0, kValues = 16 * D, kKeySteps = 32 * D, kValueSteps = 32 * D + 128 * G, kBytes = 32 * D + 256 * G;
};
inline int64_t kv_record_bytes(int head_dim, int groups) { return 32 * (int64_t)head_dim + 256 * groups; }

// The sequences of a call (device arrays), and the bounds within which the kernels take what stands in them.
struct KvBatch {
    const int32_t *table, *lens, *starts;
    int sequences, table_stride, max_new, max_len;
    int64_t tokens;
};

struct KvRows { void *p; int64_t token_stride, head_stride; };       // in elements

// ---- kv_cache.hip ----------------------------------------------------------------------------
void launch_kv_write(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, void *pool, hipStream_t st);
void launch_kv_read(const KvShape &s, const KvBatch &b, const KvRows &k, const KvRows &v, const void *pool, hipStream_t st);

// ---- kv_attend.hip ---------------------------------------------------------------------------
struct KvAttend {
    KvRows q, out;
    float *lse;
    int q_heads, window;
    bool causal;
    float scale;
};
size_t kv_attend_ws_bytes(const KvShape &s, const KvBatch &b, int q_heads);
void launch_kv_attend(const KvShape &s, const KvBatch &b, const KvAttend &a, const void *pool, void *ws, hipStream_t st);


// Sequence `b` of a call: rows first .. first + n - 1 of the call's tensors are tokens at positions pos .. pos + n - 1 of it, and positions 0 .. len - 1 may be there.
// n and len are cut to what the host was told of, and rows to those of the tensors; pos is what the arrays say, so a position may be below 0, or be len and more: a token
// that is not there.  No position passes 2^31 - 2 nor lies below 1 - 2^31.
struct KvSeq { int first, n, len, pos; };
__device__ __forceinline__ KvSeq kv_seq(const KvBatch &k, int page_tokens, int b)
{
    const int total = (int)k.tokens;
    KvSeq s;
    const int held = max(k.lens[b], 0), end = k.starts[b + 1];
    s.first = min(max(k.starts[b], 0), total);
    s.n = min(max(min(end, total) - s.first, 0), k.max_new);
    s.pos = (int)((uint32_t)held - (uint32_t)end + (uint32_t)s.first);          // (without rows: any number)
    const int64_t most = min((int64_t)k.table_stride * page_tokens, (int64_t)k.max_len);
    s.len = (int)min((int64_t)held, most);
    return s;
}
// the first position that a query at `pos` sees through a window
__device__ __forceinline__ int window_from(int pos, int window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }

// sums over the lanes up to and with this one (row shifts, then the rows' last lanes to the rows behind them)
template <typename T> __device__ __forceinline__ T lane_sums(T x)
{
    auto from = [](T v, auto ctrl, auto rows) { return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xF, true)); };
    x += from(x, IC<0x111>{}, IC<0xF>{}); x += from(x, IC<0x112>{}, IC<0xF>{}); x += from(x, IC<0x114>{}, IC<0xF>{}); x += from(x, IC<0x118>{}, IC<0xF>{});
    x += from(x, IC<0x142>{}, IC<0xA>{}); x += from(x, IC<0x143>{}, IC<0xC>{});
    return x;
}
// the greatest of the wave, the same way
__device__ __forceinline__ uint32_t lanes_greatest(uint32_t x)
{
    auto from = [](uint32_t v, auto ctrl, auto rows) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, true); };
    x = max(x, from(x, IC<0x111>{}, IC<0xF>{})); x = max(x, from(x, IC<0x112>{}, IC<0xF>{})); x = max(x, from(x, IC<0x114>{}, IC<0xF>{})); x = max(x, from(x, IC<0x118>{}, IC<0xF>{}));
    x = max(x, from(x, IC<0x142>{}, IC<0xA>{})); x = max(x, from(x, IC<0x143>{}, IC<0xC>{}));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

}  // namespace eqat
