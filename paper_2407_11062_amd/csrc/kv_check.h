// Checks of arguments that the entry points of the cache and of what goes into it share.
#pragma once
#include <hip/hip_runtime.h>

#include "kv.h"

namespace eqat {
namespace check {

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline eqat_status launch_status() { return hipGetLastError() == hipSuccess ? EQAT_OK : EQAT_ERR_DEVICE; }
constexpr int64_t kMost = (int64_t)1 << 31;          // rows, pages and workgroups are counted in 32 bits

inline eqat_status check_desc(const eqat_kv_desc *d, KvShape *s)
{
    if (d == nullptr) return EQAT_ERR_NULL;
    if (d->act_dtype != EQAT_F32 && d->act_dtype != EQAT_BF16) return EQAT_ERR_DTYPE;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return EQAT_ERR_SHAPE;
    const int g = d->group == -1 ? d->head_dim : d->group;
    if ((g != 32 && g != 64 && g != 128 && g != 256) || g > d->head_dim) return EQAT_ERR_GROUP;
    if (d->heads < 1 || d->heads > 1 << 16 || d->page_tokens < 32 || d->page_tokens % 32 != 0 || d->pages < 1 || d->pages >= kMost) return EQAT_ERR_SHAPE;
    const int64_t per_page = eqat::kv_record_bytes(d->head_dim, d->head_dim / g) * d->heads * (d->page_tokens / 32);      // below 2^60
    if (d->pages > ((int64_t)1 << 46) / per_page || d->pages * d->heads >= kMost / (d->page_tokens / 32)) return EQAT_ERR_SHAPE;         // records are numbered in 32 bits
    s->heads = d->heads; s->head_dim = d->head_dim; s->group = g; s->groups = d->head_dim / g;
    s->page_records = d->page_tokens / 32; s->pages = d->pages; s->act_bf16 = d->act_dtype == EQAT_BF16;
    return EQAT_OK;
}

inline eqat_status check_batch(const eqat_kv_batch *b, const KvShape &s, KvBatch *k)
{
    if (b == nullptr) return EQAT_ERR_NULL;
    if (b->tokens < 0 || b->sequences < 0 || b->table_stride < 0 || b->max_new < 0 || b->max_len < 0) return EQAT_ERR_SHAPE;
    if (b->tokens >= kMost || b->tokens * s.heads >= kMost / 4 || b->max_len > INT32_MAX - 32) return EQAT_ERR_SHAPE;
    if (b->tokens > 0 && b->sequences == 0) return EQAT_ERR_SHAPE;
    if (b->sequences > 0 && (b->lens == nullptr || b->starts == nullptr || (b->table == nullptr && b->table_stride > 0))) return EQAT_ERR_NULL;
    if (!aligned(b->table, 4) || !aligned(b->lens, 4) || !aligned(b->starts, 4)) return EQAT_ERR_ALIGN;
    k->table = b->table; k->lens = b->lens; k->starts = b->starts; k->tokens = b->tokens;
    k->sequences = b->sequences; k->table_stride = b->table_stride; k->max_new = b->max_new; k->max_len = b->max_len;
    return EQAT_OK;
}

inline eqat_status check_strided(const void *p, const int64_t *strides, bool bf16, KvRows *r)
{
    if (p == nullptr || strides == nullptr) return EQAT_ERR_NULL;
    const int64_t unit = bf16 ? 8 : 4;
    if (!aligned(p, 16) || strides[0] % unit != 0 || strides[1] % unit != 0) return EQAT_ERR_ALIGN;
    r->p = const_cast<void *>(p); r->token_stride = strides[0]; r->head_stride = strides[1];
    return EQAT_OK;
}

inline eqat_status check_rows(const void *p, const int64_t *strides, const KvShape &s, KvRows *r) { return check_strided(p, strides, s.act_bf16, r); }

inline eqat_status check_pool(const void *pool)
{
    if (pool == nullptr) return EQAT_ERR_NULL;
    return aligned(pool, 256) ? EQAT_OK : EQAT_ERR_ALIGN;
}

}  // namespace check
}  // namespace eqat

#define KV_TRY(call) do { if (eqat_status e_ = (call)) return e_; } while (0)
