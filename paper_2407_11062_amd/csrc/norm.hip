// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   S = round(X + R),  Y = w S rstd,  rstd = 1 / sqrt(mean S^2 + eps),  or Y in 8 bits: codes = e4m3(Y / scale), scale = max |Y| of a group / 448
//   dX = dS + rstd (e - S rstd^2 mean(e S)),  e = w dY;     dw = sum over the rows of dY S rstd
//
// Bound by bytes: every row is read once and kept in registers, eight neighbouring elements to a lane, LANES lanes to a row: part of a wave, a wave, or a workgroup that
// meets in LDS once (a row's maximum, for 8 bits with one scale a row, a second time).  Sums, means and products are binary32; S is what stands in memory, so that the
// backward pass, which makes rstd from S again, is that of what the forward computed.
//
// us over three states that take turns: 8192 rows of 8192 with a residual 93 (537 MB, 5.7 TB/s), their like of 4096 backward 49 (268 MB, 5.5); one row of 4096 2.7 in a graph, 515 rows of 5120 to 8 bits 6.6,
// 333 rows of 4096 backward, fp32, 8.2 and 2.4 for the second launch.
#include "layer.h"

#include <algorithm>
#include <atomic>

namespace eqat {
namespace {

constexpr float kFp8Most = 448.0f, kLeastScale = 0x1p-126f;

template <int LANES, typename F> __device__ __forceinline__ float lanes_all(float v, F f)
{
#pragma unroll
    for (int d = (LANES < 64 ? LANES : 64) / 2; d >= 1; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
    return v;
}
// over the LANES lanes of a row, in every one of them; `part`: an LDS word a wave, of this call's own
template <int LANES, typename F> __device__ __forceinline__ float row_all(float v, float *part, F f)
{
    v = lanes_all<LANES>(v, f);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < LANES / 64; ++w) v = f(v, part[w]);
    }
    return v;
}
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }
__device__ __forceinline__ float most_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }        // NaN wins

struct NormArgs {
    int64_t rows;
    const void *x, *r, *w, *dy;
    void *s, *y, *codes;
    float *scales, *part;
    int width, group, w_bf16;
    float eps, per_width;
};

__device__ __forceinline__ void load_w(const NormArgs &a, int at, float (&w)[8])
{
    if (a.w == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    } else if (a.w_bf16) {
        Eight<bf16_t> v;
        v.load(static_cast<const bf16_t *>(a.w) + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v.get(e);
    } else {
        Eight<float> v;
        v.load(static_cast<const float *>(a.w) + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = v.get(e);
    }
}

template <typename T, int LANES, int NV, bool ONCE>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm_fwd(const NormArgs a)
{
    constexpr int kThreads = LANES > 256 ? LANES : 256;
    __shared__ float part[2][kThreads / 64];
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
    const bool there = row < a.rows;                          // (LANES >= 256: the whole workgroup)
    const T *x = static_cast<const T *>(a.x) + row * a.width, *r = static_cast<const T *>(a.r) + row * a.width;
    Eight<T> s[NV], add[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int at = (k * LANES + lane) * 8;
        s[k].zero();
        add[k].zero();
        if (there && at < a.width) {
            s[k].template load<ONCE>(x + at);
            if (a.r != nullptr) add[k].template load<ONCE>(r + at);
        }
    }
    float w[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) if ((k * LANES + lane) * 8 < a.width) load_w(a, (k * LANES + lane) * 8, w[k]);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int at = (k * LANES + lane) * 8;
        if (a.r != nullptr) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = s[k].get(e) + add[k].get(e);
            s[k].set(v);
        }
        if (a.s != nullptr && there && at < a.width) s[k].template store<ONCE>(static_cast<T *>(a.s) + row * a.width + at);
        float t = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) t = __builtin_fmaf(s[k].get(e), s[k].get(e), t);
        sum += t;
    }
    sum = row_all<LANES>(sum, part[0], sum_of);
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(sum, a.per_width, a.eps));
    float y[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[k][e] = s[k].get(e) * rstd * w[k][e];
    if (a.y != nullptr) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            Eight<T> o;
            o.set(y[k]);
            if (there && at < a.width) o.store(static_cast<T *>(a.y) + row * a.width + at);
        }
    }
    if (a.codes != nullptr) {
        float most[NV], all = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            most[k] = 0.0f;
            if ((k * LANES + lane) * 8 < a.width) {
#pragma unroll
                for (int e = 0; e < 8; ++e) most[k] = most_of(most[k], fabsf(y[k][e]));
            }
            all = most_of(all, most[k]);
        }
        const int lanes = a.group / 8, groups = a.width / a.group;
        if (a.group == a.width) {                             // a row
            all = row_all<LANES>(all, part[1], most_of);
#pragma unroll
            for (int k = 0; k < NV; ++k) most[k] = all;
        } else {                                              // neighbouring lanes, 4 to 64 of them
            for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
                for (int k = 0; k < NV; ++k) most[k] = most_of(most[k], __shfl_xor(most[k], d, 64));
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            if (!there || at >= a.width) continue;
            const float scale = most_of(most[k] / kFp8Most, kLeastScale), by = 1.0f / scale, finite = scale < __builtin_inff() ? scale : 0.0f;
            // the quotient y / scale: the product with the reciprocal and, by what that leaves of y, put right (an infinite scale: 0 or NaN as it is; -0 stays).  The product alone falls to the other
            // side of one tie in some 20000 elements; 515 rows of 5120, bf16, in a graph 4.2 -> 4.4 us, 8192 rows of 8192 44.6 -> 46.7
            auto quotient_of = [&](float v) { const float q = v * by; return __builtin_fmaf(-__builtin_fmaf(q, finite, -v), by, q); };
            uintx2 code;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient_of(y[k][4 * h]), quotient_of(y[k][4 * h + 1]), 0, false);
                v = __builtin_amdgcn_cvt_pk_fp8_f32(quotient_of(y[k][4 * h + 2]), quotient_of(y[k][4 * h + 3]), v, true);
                code[h] = (uint32_t)v;
            }
            *reinterpret_cast<uintx2 *>(static_cast<uint8_t *>(a.codes) + row * a.width + at) = code;
            if (at % a.group == 0) a.scales[row * groups + at / a.group] = scale;
        }
    }
}

// Workgroup b takes the rows b, b + grid, ... (of kThreads / LANES each) and keeps its part of dw in registers: part[b][width], summed over b by k_norm_dw.
template <typename T, int LANES, int NV, bool ONCE>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_norm_bwd(const NormArgs a)
{
    constexpr int kThreads = LANES > 256 ? LANES : 256, kRows = kThreads / LANES;
    constexpr bool kHold = LANES < 1024;                      // 16 waves leave no registers for w and dw (in LDS instead), and dS is fetched where it is wanted
    __shared__ float part[2][2][kThreads / 64];
    extern __shared__ __attribute__((aligned(16))) float sums[];              // [kRows][width], where several rows are in the workgroup, or rows are wide, and dw is wanted
    const int lane = threadIdx.x % LANES;
    float w[kHold ? NV : 1][8], dw[kHold ? NV : 1][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int at = (k * LANES + lane) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dw[kHold ? k : 0][e] = w[kHold ? k : 0][e] = 0.0f;
            if (!kHold && a.part != nullptr && at < a.width) sums[at + e] = 0.0f;
        }
        if (kHold && at < a.width) load_w(a, at, w[kHold ? k : 0]);
    }
    const int64_t n = (a.rows + kRows - 1) / kRows;
    int turn = 0;
    for (int64_t b = blockIdx.x; b < n; b += gridDim.x, turn ^= 1) {
        const int64_t row = b * kRows + threadIdx.x / LANES;
        const bool there = row < a.rows;
        Eight<T> s[NV], dy[NV], ds[kHold ? NV : 1];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            s[k].zero(); dy[k].zero(); ds[kHold ? k : 0].zero();
            if (there && at < a.width) {
                s[k].template load<ONCE>(static_cast<const T *>(a.x) + row * a.width + at);
                dy[k].template load<ONCE>(static_cast<const T *>(a.dy) + row * a.width + at);
                if (kHold && a.r != nullptr) ds[kHold ? k : 0].template load<ONCE>(static_cast<const T *>(a.r) + row * a.width + at);
            }
        }
        float ss = 0.0f, es = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            if (!kHold && at < a.width) load_w(a, at, w[0]);
            const float (&wk)[8] = w[kHold ? k : 0];
            float t = 0.0f, u = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = s[k].get(e);
                t = __builtin_fmaf(x, x, t);
                u = __builtin_fmaf(dy[k].get(e) * wk[e], x, u);
            }
            ss += t; es += u;
            if (!kHold) __builtin_amdgcn_sched_barrier(0);    // one vector's weights at a time
        }
        ss = lanes_all<LANES>(ss, sum_of);
        es = lanes_all<LANES>(es, sum_of);
        if constexpr (LANES > 64) {                           // (the words of the turn before may still be read)
            if ((threadIdx.x & 63) == 0) { part[turn][0][threadIdx.x >> 6] = ss; part[turn][1][threadIdx.x >> 6] = es; }
            __syncthreads();
            ss = part[turn][0][0]; es = part[turn][1][0];
#pragma unroll
            for (int v = 1; v < LANES / 64; ++v) { ss += part[turn][0][v]; es += part[turn][1][v]; }
        }
        // a row that is not there shares a workgroup with others and adds to their dw: its terms are 0 only while rstd is finite, which with eps = 0 the square root of no sum is not
        const float rstd = kRows > 1 && !there ? 0.0f : 1.0f / sqrtf(__builtin_fmaf(ss, a.per_width, a.eps)), c = es * a.per_width * rstd * rstd;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            if (!kHold && there && at < a.width) {
                load_w(a, at, w[0]);
                if (a.r != nullptr) ds[0].load(static_cast<const T *>(a.r) + row * a.width + at);
            }
            const float (&wk)[8] = w[kHold ? k : 0];
            const Eight<T> &dsk = ds[kHold ? k : 0];
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = s[k].get(e), g = dy[k].get(e);
                d[e] = __builtin_fmaf(rstd, __builtin_fmaf(-x, c, g * wk[e]), dsk.get(e));
                if (kHold) dw[kHold ? k : 0][e] = __builtin_fmaf(g * rstd, x, dw[kHold ? k : 0][e]);
            }
            if (!kHold && a.part != nullptr && at < a.width) {          // the lane's own
                floatx4 *const mine = reinterpret_cast<floatx4 *>(sums + at);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    floatx4 v = mine[h];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(dy[k].get(4 * h + e) * rstd, s[k].get(4 * h + e), v[e]);
                    mine[h] = v;
                }
            }
            if (a.y != nullptr && there && at < a.width) {
                Eight<T> o;
                o.set(d);
                o.store(static_cast<T *>(a.y) + row * a.width + at);
            }
            if (!kHold) __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (a.part == nullptr) return;
    float *to = a.part + (int64_t)blockIdx.x * a.width;
    if constexpr (kRows > 1) {                                // the rows' parts meet in a fixed order
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            if (at < a.width) {
                Eight<float> o;
                o.set(dw[kHold ? k : 0]);
                o.store(sums + (int)threadIdx.x / LANES * a.width + at);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.width; i += kThreads) {
            float v = sums[i];
#pragma unroll
            for (int k = 1; k < kRows; ++k) v += sums[k * a.width + i];
            to[i] = v;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int at = (k * LANES + lane) * 8;
            if (at < a.width) {
                Eight<float> o;
                if constexpr (kHold) o.set(dw[k]); else o.load(sums + at);
                o.store(to + at);
            }
        }
    }
}

// dw[i] = the sum over b of part[b][i]: 32 neighbouring columns, four to a thread, to a workgroup, 32 threads a column, each every 32nd part, then theirs in order
constexpr int kDwRows = 32, kDwColumns = 8;
__global__ __launch_bounds__(256) void k_norm_dw(const float *__restrict__ part, float *__restrict__ dw, int parts, int width)
{
    __shared__ floatx4 sums[kDwRows * kDwColumns];
    const int c = threadIdx.x % kDwColumns, k = threadIdx.x / kDwColumns, at = ((int)blockIdx.x * kDwColumns + c) * 4;
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
    if (at < width) {
#pragma unroll 8
        for (int b = k; b < parts; b += kDwRows) s += *reinterpret_cast<const floatx4 *>(part + (int64_t)b * width + at);
    }
    sums[threadIdx.x] = s;
    __syncthreads();
    if (k == 0 && at < width) {
#pragma unroll
        for (int v = 1; v < kDwRows; ++v) s += sums[v * kDwColumns + c];
        *reinterpret_cast<floatx4 *>(dw + at) = s;
    }
}

// From this many bytes of rows on what is read goes past the caches, and S with it, which is next wanted a layer on; Y and dX, which the next call reads, do not.  Graph replays over three
// states, us, through the caches / past them: norm 67 MB 13.4 / 13.8, 134 MB 29.5 / 25.6, 269 MB 58 / 51, 537 MB 103 / 96; its gradients 67 MB 18.7 / 20.7, 134 MB 34.0 / 30.0, 269 MB 57 / 50.
constexpr int64_t kOnceBytes = (int64_t)96 << 20;

// Workgroups of a backward pass at most: two a compute unit.  One each where few of them would have two rows and the others one, and where waves of a row fill a compute unit; the second launch has
// half the parts then.  us, three states in turn, 512 / 256, bf16: 300 rows of 4096 9.0 / 8.5, 512 12.0 / 10.0, 768 12.8 / 11.1, 600 of 16384 25.6 / 21.1, 1500 of 20000 76 / 64, 1024 of 8192 18.3 / 18.3,
// 2048 of 8192 28.6 / 31.1; fp32: 512 of 4096 13.6 / 11.4, 768 13.6 / 13.0, 600 of 16384 42 / 37, 1500 of 20000 112 / 104, 1024 of 8192 29.0 / 27.2, 2048 of 8192 47.5 / 48.5 (300 of 4096 10.7 / 10.9).
constexpr int kNormParts = 512;

// Lanes and vectors a lane of a row.  Few vectors a lane where the chip has waves to spare: a row is a chain of a fetch, a sum, the results, and the shorter its links the better; with more rows than
// compute units whole workgroups hide each other's.  bf16.  Forward with a residual, us, 256 lanes / 512 / 1024: one row of 4096 3.3 / 2.9, 515 rows 5.5 / 5.3, one of 8192 4.5 / 3.5 / 3.1, 256 rows 6.4 / 5.2 / 4.9, 515 rows
// 9.5 / 8.9 / 9.6, 4096 rows 50.9 / 46.3 / 45.5.  Backward: 1024 rows of 4096 14.1 / 13.2; 64 of 8192 8.6 / 7.9 / 7.9, 333 14.8 / 15.1 / 14.7, 4096 52 / 60 / 68.
template <bool BACK, typename F> void by_width(int64_t rows, int width, F f)
{
    const int n = width / 8;            // vectors of a row
    const bool few = rows <= 256;
    if (n <= 8) f(IC<8>{}, IC<1>{});
    else if (n <= 16) f(IC<16>{}, IC<1>{});
    else if (n <= 32) f(IC<32>{}, IC<1>{});
    else if (n <= 64) f(IC<64>{}, IC<1>{});
    else if (n <= 128) f(IC<64>{}, IC<2>{});
    else if (n <= 256) f(IC<256>{}, IC<1>{});
    else if (n <= 512) f(IC<512>{}, IC<1>{});
    else if (n > 2048) f(IC<1024>{}, IC<4>{});
    else if constexpr (BACK) {
        if (n > 1024) f(IC<512>{}, IC<4>{});
        else if (few) f(IC<512>{}, IC<2>{});
        else if (n <= 768) f(IC<256>{}, IC<3>{});
        else f(IC<256>{}, IC<4>{});
    } else {
        if (n <= 1024) { if (few) f(IC<1024>{}, IC<1>{}); else f(IC<512>{}, IC<2>{}); }
        else if (few) f(IC<1024>{}, IC<2>{});
        else f(IC<512>{}, IC<4>{});
    }
}

int bwd_blocks(int64_t rows, int width)
{
    int per = 1;
    by_width<true>(rows, width, [&](auto lanes, auto) { per = decltype(lanes)::value < 256 ? 256 / decltype(lanes)::value : 1; });
    const int64_t n = (rows + per - 1) / per;
    return (int)std::min<int64_t>(n, n <= 768 || width > 16384 ? kNormParts / 2 : kNormParts);
}

}  // namespace

size_t norm_ws_bytes(int64_t rows, int width) { return rows > 0 ? (size_t)bwd_blocks(rows, width) * width * sizeof(float) : 0; }

void launch_norm_fwd(const NormFwd &n, hipStream_t st)
{
    NormArgs a{};
    a.w = n.w;
    a.width = n.width; a.group = n.group; a.w_bf16 = n.w_bf16; a.eps = n.eps; a.per_width = 1.0f / (float)n.width;
    const int64_t per = n.rows * n.width * (n.act_bf16 ? 2 : 4);
    const bool once = per * (1 + (n.r != nullptr) + (n.s != nullptr) + (n.y != nullptr)) > kOnceBytes;
    by_width<false>(n.rows, n.width, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, N = decltype(nv)::value, kThreads = L > 256 ? L : 256;
        // a launch has fewer than 2^32 threads
        constexpr int64_t kRows = kThreads / L, kMostRows = ((int64_t)1 << 31) / kThreads * kRows;
        const int64_t ax = n.act_bf16 ? 2 : 4;
        for (int64_t done = 0; done < n.rows; done += kMostRows) {
            auto from = [&](const void *p, int64_t bytes) { return p == nullptr ? nullptr : static_cast<char *>(const_cast<void *>(p)) + done * bytes; };
            a.rows = std::min(n.rows - done, kMostRows);
            a.x = from(n.x, n.width * ax); a.r = from(n.r, n.width * ax); a.s = from(n.s, n.width * ax); a.y = from(n.y, n.width * ax); a.codes = from(n.codes, n.width);
            a.scales = reinterpret_cast<float *>(from(n.scales, n.width / n.group * 4));
            const unsigned blocks = (unsigned)((a.rows + kRows - 1) / kRows);
            auto go = [&](auto kern) { kern<<<blocks, kThreads, 0, st>>>(a); };
            if (n.act_bf16) {
                if (once) go(k_norm_fwd<bf16_t, L, N, true>); else go(k_norm_fwd<bf16_t, L, N, false>);
            } else {
                if (once) go(k_norm_fwd<float, L, N, true>); else go(k_norm_fwd<float, L, N, false>);
            }
        }
    });
}

void launch_norm_bwd(const NormBwd &n, void *ws, hipStream_t st)
{
    NormArgs a{};
    const int blocks = bwd_blocks(n.rows, n.width);
    a.rows = n.rows; a.x = n.s; a.r = n.ds; a.w = n.w; a.dy = n.dy; a.y = n.dx;
    a.part = n.dw == nullptr ? nullptr : blocks == 1 ? n.dw : static_cast<float *>(ws);
    a.width = n.width; a.w_bf16 = n.w_bf16; a.eps = n.eps; a.per_width = 1.0f / (float)n.width;
    if (blocks > 0) by_width<true>(n.rows, n.width, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, N = decltype(nv)::value, kThreads = L > 256 ? L : 256;
        const size_t lds = (L < 256 || L == 1024) && n.dw != nullptr ? (size_t)(kThreads / L) * n.width * sizeof(float) : 0;          // up to 16 KiB; 128 KiB
        if constexpr (L == 1024) {      // more than the default limit: once per device
            static std::atomic<uint64_t> allowed{0};
            int dev = 0;
            if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev > 63) dev = 0;
            if (!((allowed.load(std::memory_order_relaxed) >> dev) & 1u)) {
                (void)hipFuncSetAttribute((const void *)k_norm_bwd<bf16_t, L, N, false>, hipFuncAttributeMaxDynamicSharedMemorySize, kNormMostWidth * (int)sizeof(float));
                (void)hipFuncSetAttribute((const void *)k_norm_bwd<float, L, N, false>, hipFuncAttributeMaxDynamicSharedMemorySize, kNormMostWidth * (int)sizeof(float));
                allowed.fetch_or((uint64_t)1 << dev, std::memory_order_relaxed);
            }
        }
        const bool once = L < 1024 && n.rows * n.width * (n.act_bf16 ? 2 : 4) * (2 + (n.ds != nullptr) + (n.dx != nullptr)) > kOnceBytes;
        if (n.act_bf16) {
            if (once) k_norm_bwd<bf16_t, L, N, L < 1024><<<blocks, kThreads, lds, st>>>(a); else k_norm_bwd<bf16_t, L, N, false><<<blocks, kThreads, lds, st>>>(a);
        } else {
            if (once) k_norm_bwd<float, L, N, L < 1024><<<blocks, kThreads, lds, st>>>(a); else k_norm_bwd<float, L, N, false><<<blocks, kThreads, lds, st>>>(a);
        }
    });
    if (n.dw != nullptr && blocks != 1) k_norm_dw<<<(n.width / 4 + kDwColumns - 1) / kDwColumns, 256, 0, st>>>(a.part, n.dw, blocks, n.width);
}

}  // namespace eqat
