// What a decoder layer computes around its quantized linears (norm, rotary positions, the gate of the feed-forward): launchers, and the vectors that their kernels move.
#pragma once
#include "gate.h"
#include "kernels.h"
#include "kv.h"

namespace eqat {

// ---- norm.hip --------------------------------------------------------------------------------
struct NormFwd {
    int64_t rows;
    int width, group;                   // group: elements of a scale, width for a row
    float eps;
    bool act_bf16, w_bf16;
    const void *x, *r, *w;              // r, w may be NULL
    void *s, *y, *codes;                // each may be NULL
    float *scales;
};
struct NormBwd {
    int64_t rows;
    int width;
    float eps;
    bool act_bf16, w_bf16;
    const void *s, *w, *dy, *ds;        // w, ds may be NULL
    void *dx;                           // may be NULL
    float *dw;                          // may be NULL
};
constexpr int kNormMostWidth = 32768;
size_t norm_ws_bytes(int64_t rows, int width);
void launch_norm_fwd(const NormFwd &n, hipStream_t st);
void launch_norm_bwd(const NormBwd &n, void *ws, hipStream_t st);

// ---- rotary.hip ------------------------------------------------------------------------------
struct Rotary {
    const float *freq;                  // [part / 2]
    int part;
    bool interleaved;
    float amplitude;
};
struct RotaryCall {
    Rotary turn;
    const int32_t *pos;
    int64_t tokens;
    int head_dim, q_heads, k_heads;     // 0: none of them
    KvRows q, k, q_out, k_out;
    bool act_bf16, inverse;
};
void launch_rotary(const RotaryCall &c, hipStream_t st);
// the newest tokens' queries turned, and keys, turned, and values into the cache (kv_cache.hip)
void launch_kv_rotary_write(const KvShape &s, const KvBatch &b, const Rotary &turned, const KvRows &q, const KvRows &q_out, int q_heads, const KvRows &k, const KvRows &v, void *pool,
                            hipStream_t st);

// ---- gate.hip --------------------------------------------------------------------------------
struct GateCall {
    int64_t tokens;
    int inter, kind;
    bool act_bf16;
    const void *y, *dh;                 // dh NULL: forward
    void *h, *dy;                       // each may be NULL
};
void launch_gate(const GateCall &c, hipStream_t st);

// ---- 16 bytes of bf16 or 32 of fp32 ----------------------------------------------------------
template <bool ONCE, typename V> __device__ __forceinline__ V load_as(const V *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE, typename V> __device__ __forceinline__ void store_as(V v, V *p)
{
    if constexpr (ONCE) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    uintx4 v;
    template <bool ONCE = false> __device__ __forceinline__ void load(const bf16_t *p) { v = load_as<ONCE>(reinterpret_cast<const uintx4 *>(p)); }
    template <bool ONCE = false> __device__ __forceinline__ void store(bf16_t *p) const { store_as<ONCE>(v, reinterpret_cast<uintx4 *>(p)); }
    __device__ __forceinline__ void zero() { v = uintx4{0, 0, 0, 0}; }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e % 2 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16); }
    __device__ __forceinline__ void set(const float (&x)[8])          // to nearest, ties to even
    {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (bf16_t)x[e];
        v = __builtin_bit_cast(uintx4, o);
    }
};
template <> struct Eight<float> {
    floatx4 v[2];
    template <bool ONCE = false> __device__ __forceinline__ void load(const float *p)
    {
        v[0] = load_as<ONCE>(reinterpret_cast<const floatx4 *>(p)); v[1] = load_as<ONCE>(reinterpret_cast<const floatx4 *>(p) + 1);
    }
    template <bool ONCE = false> __device__ __forceinline__ void store(float *p) const
    {
        store_as<ONCE>(v[0], reinterpret_cast<floatx4 *>(p)); store_as<ONCE>(v[1], reinterpret_cast<floatx4 *>(p) + 1);
    }
    __device__ __forceinline__ void zero() { v[0] = v[1] = floatx4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ float get(int e) const { return v[e / 4][e % 4]; }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = x[e];
    }
};

}  // namespace eqat
