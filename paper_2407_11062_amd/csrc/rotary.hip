// Rotary positions: the pairs of a head's first `part` elements turned by position x frequency.
//
//   (a, b) -> (a cos - b sin, b cos + a sin) times an amplitude, pairs (i, i + part / 2) or (2 i, 2 i + 1); `inverse` turns back, which is the transpose: the backward pass.
//
// Bound by bytes.  A workgroup makes the cosines and sines of its tokens once, in LDS, and turns all (or some) heads of queries and keys with them.  A unit of work is 16 bytes of a
// head, or two times 16 where the partners are part / 2 apart, and both of a pair are read before either is written, so that a tensor can be turned in place.
// 8192 tokens of 72 heads of 128, bf16: 51 us for 302 MB (5.9 TB/s); 1000 tokens of 64 heads of 64, half of it turned, fp32: 7.1 us for 33 MB.
#include "layer.h"
#include "turn.h"

#include <algorithm>

namespace eqat {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTurns = 4096;        // pairs of a workgroup's tokens, 32 KiB

struct RotaryArgs {
    const float *freq;
    const int32_t *pos;
    KvRows q, k, q_out, k_out;
    int64_t tokens;
    float amplitude, amplitude_sin;
    int half, units, turned;            // pairs of a head; units of a head, and how many of them are turned
    int q_heads, heads;                 // of queries; of both
    int block_tokens, block_heads;
};

// V elements of T, up to 16 bytes
template <typename T, int V> struct Piece {
    typedef T vec __attribute__((ext_vector_type(V)));
    vec v;
    template <bool ONCE> __device__ __forceinline__ void load(const T *p) { v = load_as<ONCE>(reinterpret_cast<const vec *>(p)); }
    template <bool ONCE> __device__ __forceinline__ void store(T *p) const { store_as<ONCE>(v, reinterpret_cast<vec *>(p)); }
    __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
    __device__ __forceinline__ void set(int e, float x) { v[e] = (T)x; }
};
template <typename T> struct Piece<T, 1> {
    T v;
    template <bool ONCE> __device__ __forceinline__ void load(const T *p) { v = *p; }
    template <bool ONCE> __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return (float)v; }
    __device__ __forceinline__ void set(int, float x) { v = (T)x; }
};

template <typename T, int V, bool INTER, bool ONCE> __global__ __launch_bounds__(kThreads) void k_rotary(const RotaryArgs a)
{
    extern __shared__ __attribute__((aligned(16))) floatx2 turns[];           // [tokens][half]
    const int64_t token0 = (int64_t)blockIdx.x * a.block_tokens;
    const int tokens = (int)min((int64_t)a.block_tokens, a.tokens - token0), head0 = blockIdx.y * a.block_heads, heads = min(a.block_heads, a.heads - head0);
    for (int e = threadIdx.x; e < tokens * a.half; e += kThreads) {
        const int t = quotient(e, a.half);
        float c, s;
        cos_sin(a.pos[token0 + t], a.freq[e - t * a.half], c, s);
        turns[e] = floatx2{c * a.amplitude, s * a.amplitude_sin};
    }
    __syncthreads();
    struct Unit { const T *from; T *to; int turn; bool any, turned; Piece<T, V> x, y; };
    auto take = [&](int u) {
        Unit w;
        w.any = u < tokens * heads * a.units;
        if (!w.any) return w;
        const int th = quotient(u, a.units), p = u - th * a.units, t = quotient(th, heads), h = head0 + (th - t * heads);
        const bool is_q = h < a.q_heads;
        const KvRows &in = is_q ? a.q : a.k, &out = is_q ? a.q_out : a.k_out;
        const int64_t token = token0 + t, head = is_q ? h : h - a.q_heads;
        w.turned = p < a.turned;
        const int at = (INTER || w.turned ? p : p + a.turned) * V;            // (apart: a turned unit is two pieces)
        w.turn = t * a.half + (INTER ? p * V / 2 : p * V);
        w.from = static_cast<const T *>(in.p) + token * in.token_stride + head * in.head_stride + at;
        w.to = static_cast<T *>(out.p) + token * out.token_stride + head * out.head_stride + at;
        w.x.template load<ONCE>(w.from);
        if (!INTER && w.turned) w.y.template load<ONCE>(w.from + a.half);
        return w;
    };
    auto put = [&](Unit &w) {
        if (!w.any) return;
        if (w.turned) {
            if constexpr (INTER) {
#pragma unroll
                for (int e = 0; e + 1 < V; e += 2) {
                    const floatx2 cs = turns[w.turn + e / 2];
                    const float x = w.x.get(e), y = w.x.get(e + 1);
                    w.x.set(e, __builtin_fmaf(x, cs[0], -(y * cs[1])));
                    w.x.set(e + 1, __builtin_fmaf(y, cs[0], x * cs[1]));
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const floatx2 cs = turns[w.turn + e];
                    const float x = w.x.get(e), y = w.y.get(e);
                    w.x.set(e, __builtin_fmaf(x, cs[0], -(y * cs[1])));
                    w.y.set(e, __builtin_fmaf(y, cs[0], x * cs[1]));
                }
                w.y.template store<ONCE>(w.to + a.half);
            }
        }
        w.x.template store<ONCE>(w.to);
    };
    const int n = tokens * heads * a.units;
    for (int u = threadIdx.x; u < n; u += 2 * kThreads) {     // two on their way at a time
        Unit v = take(u), w = take(u + kThreads);
        put(v);
        put(w);
    }
}

}  // namespace

void launch_rotary(const RotaryCall &c, hipStream_t st)
{
    RotaryArgs a{};
    a.freq = c.turn.freq; a.pos = c.pos; a.q = c.q; a.k = c.k; a.q_out = c.q_out; a.k_out = c.k_out; a.tokens = c.tokens;
    a.amplitude = c.turn.amplitude; a.amplitude_sin = c.inverse ? -c.turn.amplitude : c.turn.amplitude;
    a.q_heads = c.q_heads; a.heads = c.q_heads + c.k_heads; a.half = c.turn.part / 2;
    // the widest pieces that divide what is turned (or half of it) and what is not
    const int whole = c.turn.interleaved ? c.turn.part : a.half;
    int v = c.act_bf16 ? 8 : 4;
    while (v > 1 && (whole % v != 0 || (c.head_dim - c.turn.part) % v != 0)) v /= 2;
    a.turned = whole / v;
    a.units = a.turned + (c.head_dim - c.turn.part) / v;
    // workgroups of about 1024 units, of fewer heads where tokens are few
    const int64_t per_token = (int64_t)a.heads * a.units;
    a.block_heads = a.heads;
    a.block_tokens = (int)std::max<int64_t>(1, std::min<int64_t>(1024 / per_token, kMostTurns / a.half));
    if ((c.tokens + a.block_tokens - 1) / a.block_tokens < 512) {
        a.block_tokens = 1;
        const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((per_token + kThreads - 1) / kThreads, 1024 / std::max<int64_t>(1, c.tokens)));
        a.block_heads = (int)((a.heads + blocks - 1) / blocks);
    }
    // blockIdx.y has 16 bits
    a.block_heads = std::max(a.block_heads, (a.heads + 65534) / 65535);
    const size_t lds = (size_t)a.block_tokens * a.half * sizeof(floatx2);
    // Past the caches from this many bytes on: 8192 tokens of 72 heads of 128, 302 MB, graph replays over three states 58 -> 52 us, 151 MB 31.9 -> 27.6, 75 MB 13.6 -> 15.6
    const bool once = 2 * c.tokens * a.heads * c.head_dim * (c.act_bf16 ? 2 : 4) > (int64_t)96 << 20;
    const int64_t size = c.act_bf16 ? 2 : 4, most = ((int64_t)1 << 31) / kThreads * a.block_tokens;          // a launch has fewer than 2^32 threads
    auto go = [&](auto kern) {
        for (int64_t done = 0; done < c.tokens; done += most) {
            RotaryArgs b = a;
            auto from = [&](KvRows &r) { if (r.p != nullptr) r.p = static_cast<char *>(r.p) + done * r.token_stride * size; };
            from(b.q); from(b.k); from(b.q_out); from(b.k_out);
            b.pos += done;
            b.tokens = std::min(c.tokens - done, most);
            kern<<<dim3((unsigned)((b.tokens + a.block_tokens - 1) / a.block_tokens), (unsigned)((a.heads + a.block_heads - 1) / a.block_heads)), kThreads, lds, st>>>(b);
        }
    };
#define EQAT_ROTARY(T, V) do { if (c.turn.interleaved) { if (once) go(k_rotary<T, V, true, true>); else go(k_rotary<T, V, true, false>); } \
                               else if (once) go(k_rotary<T, V, false, true>); else go(k_rotary<T, V, false, false>); } while (0)
    if (c.act_bf16) {
        if (v == 8) EQAT_ROTARY(bf16_t, 8); else if (v == 4) EQAT_ROTARY(bf16_t, 4); else if (v == 2) EQAT_ROTARY(bf16_t, 2); else go(k_rotary<bf16_t, 1, false, false>);
    } else {
        if (v == 4) EQAT_ROTARY(float, 4); else if (v == 2) EQAT_ROTARY(float, 2); else go(k_rotary<float, 1, false, false>);
    }
#undef EQAT_ROTARY
}

}  // namespace eqat
