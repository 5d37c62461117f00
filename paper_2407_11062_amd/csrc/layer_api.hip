// C ABI of the norm, the rotary positions and the gate: argument checking on the host, then the kernels.
#include <hip/hip_runtime.h>

#include "layer.h"
#include "kv_check.h"
#include "prof.h"

#include <cmath>

using eqat::ProfScope;

namespace {

using namespace eqat::check;

bool known(int32_t dtype) { return dtype == EQAT_F32 || dtype == EQAT_BF16; }
#define LAYER_ALIGNED(ptr) do { if (!aligned((ptr), 16)) return EQAT_ERR_ALIGN; } while (0)

eqat_status check_norm(const eqat_norm_desc *d)
{
    if (d == nullptr) return EQAT_ERR_NULL;
    if (!known(d->act_dtype) || !known(d->w_dtype)) return EQAT_ERR_DTYPE;
    if (d->tokens < 0 || d->tokens >= kMost || d->width < 8 || d->width % 8 != 0 || d->width > eqat::kNormMostWidth) return EQAT_ERR_SHAPE;
    if (!(d->eps >= 0.0f && std::isfinite(d->eps))) return EQAT_ERR_HYPER;
    return EQAT_OK;
}

eqat_status check_rotary(const eqat_rotary_desc *d, eqat::Rotary *r)
{
    if (d == nullptr) return EQAT_ERR_NULL;
    if (!known(d->act_dtype)) return EQAT_ERR_DTYPE;
    if (d->head_dim < 8 || d->head_dim % 8 != 0 || d->head_dim > 1024 || d->part < 2 || d->part % 2 != 0 || d->part > d->head_dim) return EQAT_ERR_SHAPE;
    if (!std::isfinite(d->amplitude)) return EQAT_ERR_HYPER;
    if (!aligned(d->frequencies, 4)) return EQAT_ERR_ALIGN;
    r->freq = d->frequencies; r->part = d->part; r->interleaved = d->interleaved != 0; r->amplitude = d->amplitude;
    return EQAT_OK;
}

}  // namespace

extern "C" {

eqat_status eqat_norm_fwd(const eqat_norm_desc *d, const void *X, const void *R, const void *w, void *S, void *Y, uint8_t *codes, float *scales, void *stream)
{
    KV_TRY(check_norm(d));
    if ((codes == nullptr) != (scales == nullptr)) return EQAT_ERR_NULL;
    int group = d->width;
    if (codes != nullptr && d->group != -1) {
        group = d->group;
        if (group != 32 && group != 64 && group != 128 && group != 256 && group != 512) return EQAT_ERR_GROUP;
        if (d->width % group != 0) return EQAT_ERR_GROUP;
    }
    if (d->tokens == 0 || (S == nullptr && Y == nullptr && codes == nullptr)) return EQAT_OK;
    if (X == nullptr) return EQAT_ERR_NULL;
    LAYER_ALIGNED(X); LAYER_ALIGNED(R); LAYER_ALIGNED(w); LAYER_ALIGNED(S); LAYER_ALIGNED(Y); LAYER_ALIGNED(codes); LAYER_ALIGNED(scales);
    eqat::NormFwd n{d->tokens, d->width, group, d->eps, d->act_dtype == EQAT_BF16, d->w_dtype == EQAT_BF16, X, R, w, S, Y, codes, scales};
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_NORM, st); eqat::launch_norm_fwd(n, st); }
    return launch_status();
}

size_t eqat_norm_workspace_bytes(const eqat_norm_desc *d) { return check_norm(d) == EQAT_OK ? eqat::norm_ws_bytes(d->tokens, d->width) : 0; }

eqat_status eqat_norm_bwd(const eqat_norm_desc *d, const void *S, const void *w, const void *dY, const void *dS, void *dX, float *dw, void *ws, size_t ws_bytes, void *stream)
{
    KV_TRY(check_norm(d));
    if (dX == nullptr && dw == nullptr) return EQAT_OK;
    if (d->tokens > 0 && (S == nullptr || dY == nullptr)) return EQAT_ERR_NULL;
    LAYER_ALIGNED(S); LAYER_ALIGNED(w); LAYER_ALIGNED(dY); LAYER_ALIGNED(dS); LAYER_ALIGNED(dX); LAYER_ALIGNED(dw);
    if (d->tokens == 0 && dw == nullptr) return EQAT_OK;
    if (dw != nullptr && d->tokens > 0) {
        if (ws == nullptr || ws_bytes < eqat::norm_ws_bytes(d->tokens, d->width)) return EQAT_ERR_WORKSPACE;
        if (!aligned(ws, 256)) return EQAT_ERR_ALIGN;
    }
    eqat::NormBwd n{d->tokens, d->width, d->eps, d->act_dtype == EQAT_BF16, d->w_dtype == EQAT_BF16, S, w, dY, dS, dX, dw};
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_NORM, st); eqat::launch_norm_bwd(n, ws, st); }
    return launch_status();
}

eqat_status eqat_rotary(const eqat_rotary_desc *d, int64_t tokens, const int32_t *positions, const void *Q, const int64_t *q_strides, int q_heads, void *q_out,
                        const int64_t *q_out_strides, const void *K, const int64_t *k_strides, int k_heads, void *k_out, const int64_t *k_out_strides, int inverse, void *stream)
{
    eqat::RotaryCall c{};
    KV_TRY(check_rotary(d, &c.turn));
    const bool bf16 = d->act_dtype == EQAT_BF16;
    if (tokens < 0 || tokens >= kMost) return EQAT_ERR_SHAPE;
    if (Q != nullptr && (q_heads < 1 || q_heads > 1 << 20 || tokens * q_heads >= kMost)) return EQAT_ERR_SHAPE;
    if (K != nullptr && (k_heads < 1 || k_heads > 1 << 20 || tokens * k_heads >= kMost)) return EQAT_ERR_SHAPE;
    if ((Q == nullptr) != (q_out == nullptr) || (K == nullptr) != (k_out == nullptr)) return EQAT_ERR_NULL;
    if (tokens == 0 || (Q == nullptr && K == nullptr)) return EQAT_OK;
    if (d->frequencies == nullptr || positions == nullptr) return EQAT_ERR_NULL;
    if (!aligned(positions, 4)) return EQAT_ERR_ALIGN;
    if (Q != nullptr) { KV_TRY(check_strided(Q, q_strides, bf16, &c.q)); KV_TRY(check_strided(q_out, q_out_strides, bf16, &c.q_out)); c.q_heads = q_heads; }
    if (K != nullptr) { KV_TRY(check_strided(K, k_strides, bf16, &c.k)); KV_TRY(check_strided(k_out, k_out_strides, bf16, &c.k_out)); c.k_heads = k_heads; }
    c.pos = positions; c.tokens = tokens; c.head_dim = d->head_dim; c.act_bf16 = bf16; c.inverse = inverse != 0;
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_ROTARY, st); eqat::launch_rotary(c, st); }
    return launch_status();
}

eqat_status eqat_kv_rotary_write(const eqat_kv_desc *d, const eqat_kv_batch *b, const eqat_rotary_desc *r, const void *Q, const int64_t *q_strides, int q_heads, void *q_out,
                                 const int64_t *q_out_strides, const void *K, const int64_t *k_strides, const void *V, const int64_t *v_strides, void *pool, void *stream)
{
    eqat::KvShape s; eqat::KvBatch k; eqat::KvRows qr, qo, kr, vr; eqat::Rotary turn;
    KV_TRY(check_desc(d, &s));
    KV_TRY(check_batch(b, s, &k));
    KV_TRY(check_rotary(r, &turn));
    if (r->head_dim != d->head_dim) return EQAT_ERR_SHAPE;
    if (r->act_dtype != d->act_dtype) return EQAT_ERR_DTYPE;
    if (q_heads < 1 || q_heads > 1 << 20 || b->tokens * q_heads >= kMost) return EQAT_ERR_SHAPE;
    if (k.tokens == 0) return EQAT_OK;
    if (r->frequencies == nullptr) return EQAT_ERR_NULL;
    KV_TRY(check_strided(Q, q_strides, s.act_bf16, &qr));
    KV_TRY(check_strided(q_out, q_out_strides, s.act_bf16, &qo));
    KV_TRY(check_strided(K, k_strides, s.act_bf16, &kr));
    KV_TRY(check_strided(V, v_strides, s.act_bf16, &vr));
    KV_TRY(check_pool(pool));
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_KV_WRITE, st); eqat::launch_kv_rotary_write(s, k, turn, qr, qo, q_heads, kr, vr, pool, st); }
    return launch_status();
}

static eqat_status gate_any(int64_t tokens, int64_t F, int32_t dtype, int kind, const void *Y, const void *dH, void *dY, void *H, bool back, void *stream)
{
    if (!known(dtype)) return EQAT_ERR_DTYPE;
    if (tokens < 0 || F < 8 || F % 8 != 0 || F >= kMost || tokens >= kMost || (tokens > 0 && F / 8 > (kMost - 1) / tokens)) return EQAT_ERR_SHAPE;
    if (kind != EQAT_GATE_SILU && kind != EQAT_GATE_GELU) return EQAT_ERR_HYPER;
    if (tokens == 0 || (back && dY == nullptr && H == nullptr)) return EQAT_OK;
    if (Y == nullptr || (back ? dH == nullptr : H == nullptr)) return EQAT_ERR_NULL;
    LAYER_ALIGNED(Y); LAYER_ALIGNED(dH); LAYER_ALIGNED(dY); LAYER_ALIGNED(H);
    hipStream_t st = (hipStream_t)stream;
    { ProfScope ps(eqat::PK_GATE, st); eqat::launch_gate(eqat::GateCall{tokens, (int)F, kind, dtype == EQAT_BF16, Y, dH, H, dY}, st); }
    return launch_status();
}

eqat_status eqat_gate_fwd(int64_t tokens, int64_t F, int32_t dtype, int kind, const void *Y, void *H, void *stream) { return gate_any(tokens, F, dtype, kind, Y, nullptr, nullptr, H, false, stream); }
eqat_status eqat_gate_bwd(int64_t tokens, int64_t F, int32_t dtype, int kind, const void *Y, const void *dH, void *dY, void *H, void *stream)
{
    return gate_any(tokens, F, dtype, kind, Y, dH, dY, H, true, stream);
}

}  // extern "C"
