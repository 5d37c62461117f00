// C ABI of the 4-bit key-value cache: argument checking on the host, then the kernels.
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_check.h"
#include "prof.h"

#include <cmath>

using eqat::KvBatch;
using eqat::KvRows;
using eqat::KvShape;
using eqat::ProfScope;

namespace {

using namespace eqat::check;

// the bounds of an attention call: rows (query, head) and workgroups are counted in 32 bits
eqat_status check_heads(const KvShape &s, const KvBatch &b, int q_heads)
{
    if (q_heads < s.heads || q_heads % s.heads != 0 || q_heads > 1 << 20) return EQAT_ERR_SHAPE;
    const int64_t ratio = q_heads / s.heads;
    // the streamed kernel counts the places of all units of 16 rows; a bf16 sequence of more than 64 rows is its business only where they fit
    const double units = s.act_bf16 ? 4.0 * b.sequences : (double)(b.tokens * ratio) / 16 + b.sequences;
    if (units * (b.max_len / 32 + 1.0 + eqat::kKvBeginning) > eqat::kKvMostPlaces) return EQAT_ERR_SHAPE;
    if (b.tokens * q_heads >= kMost || (int64_t)b.max_new * ratio >= kMost / 2 || ((int64_t)b.sequences + b.tokens * ratio / 16 + 2048) * s.heads >= kMost) return EQAT_ERR_SHAPE;
    return EQAT_OK;
}

}  // namespace

extern "C" {

size_t eqat_kv_pool_bytes(const eqat_kv_desc *d)
{
    KvShape s;
    if (check_desc(d, &s) != EQAT_OK) return 0;
    return (size_t)(eqat::kv_record_bytes(s.head_dim, s.groups) * s.heads * s.page_records * s.pages);
}

eqat_status eqat_kv_write(const eqat_kv_desc *d, const eqat_kv_batch *b, const void *K, const int64_t *k_strides, const void *V,
                          const int64_t *v_strides, void *pool, void *stream)
{
    KvShape s; KvBatch k; KvRows kr, vr;
    KV_TRY(check_desc(d, &s));
    KV_TRY(check_batch(b, s, &k));
    if (k.tokens == 0) return EQAT_OK;
    KV_TRY(check_rows(K, k_strides, s, &kr));
    KV_TRY(check_rows(V, v_strides, s, &vr));
    KV_TRY(check_pool(pool));
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_KV_WRITE, st); eqat::launch_kv_write(s, k, kr, vr, pool, st); }
    return launch_status();
}

eqat_status eqat_kv_read(const eqat_kv_desc *d, const eqat_kv_batch *b, void *K, const int64_t *k_strides, void *V, const int64_t *v_strides,
                         const void *pool, void *stream)
{
    KvShape s; KvBatch k; KvRows kr{}, vr{};
    KV_TRY(check_desc(d, &s));
    KV_TRY(check_batch(b, s, &k));
    if (k.tokens == 0 || (K == nullptr && V == nullptr)) return EQAT_OK;
    if (K != nullptr) KV_TRY(check_rows(K, k_strides, s, &kr));
    if (V != nullptr) KV_TRY(check_rows(V, v_strides, s, &vr));
    KV_TRY(check_pool(pool));
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_KV_READ, st); eqat::launch_kv_read(s, k, kr, vr, pool, st); }
    return launch_status();
}

size_t eqat_kv_workspace_bytes(const eqat_kv_desc *d, const eqat_kv_batch *b, int q_heads)
{
    KvShape s; KvBatch k;
    if (check_desc(d, &s) != EQAT_OK || b == nullptr) return 0;
    k.tokens = b->tokens; k.sequences = b->sequences; k.max_new = b->max_new; k.max_len = b->max_len;
    if (k.tokens < 0 || k.max_len < 0 || k.sequences < 0 || k.max_new < 0 || check_heads(s, k, q_heads) != EQAT_OK) return 0;
    return eqat::kv_attend_ws_bytes(s, k, q_heads);
}

eqat_status eqat_kv_attention(const eqat_kv_desc *d, const eqat_kv_batch *b, const eqat_kv_attn *a, const void *Q, const int64_t *q_strides,
                              void *out, const int64_t *out_strides, float *lse, const void *pool, void *ws, size_t ws_bytes, void *stream)
{
    KvShape s; KvBatch k; eqat::KvAttend t;
    KV_TRY(check_desc(d, &s));
    KV_TRY(check_batch(b, s, &k));
    if (a == nullptr) return EQAT_ERR_NULL;
    KV_TRY(check_heads(s, k, a->q_heads));
    if (!(a->scale >= 0.0f && a->scale <= 0x1p100f) || a->window < 0) return EQAT_ERR_HYPER;
    if (k.tokens == 0) return EQAT_OK;
    KV_TRY(check_rows(Q, q_strides, s, &t.q));
    KV_TRY(check_rows(out, out_strides, s, &t.out));
    if (!aligned(lse, 4)) return EQAT_ERR_ALIGN;
    KV_TRY(check_pool(pool));
    if (ws == nullptr || ws_bytes < eqat::kv_attend_ws_bytes(s, k, a->q_heads)) return EQAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EQAT_ERR_ALIGN;
    t.lse = lse; t.q_heads = a->q_heads; t.window = a->window; t.causal = a->causal != 0;
    t.scale = a->scale > 0.0f ? a->scale : 1.0f / std::sqrt((float)s.head_dim);
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_KV_ATTEND, st); eqat::launch_kv_attend(s, k, t, pool, ws, st); }
    return launch_status();
}

}  // extern "C"
