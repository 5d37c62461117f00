// The GEMM for few output tiles (gemm_mid.h) of the plain forward, and where it is taken.
#include "gemm_mid.h"

namespace eqat {

// From 3-bit codes as packed, which have no byte alignment, a K step takes 0.45 us longer than from the working layout.  With two
// rounds of workgroups and three token tiles or more that is more than the re-layout costs, and even the 128 x 128 tiles
// behind a re-layout are faster then (g = 128, us, as packed / tiles / re-laid: 1300 tokens, 4096 x 11008 198 / 181 / 167;
// 384 tokens, 11008 x 8192 148 / 136 / 122; 640 tokens, 8192 x 5120 95 / 90 / 83).  With two token tiles every weight is
// rebuilt twice only: 160 tokens, 28672 x 4096 76 as packed, 81 re-laid.
FwdRoute mid_route(const Problem &p, bool from_packed)
{
    const int tokens = token_tile(p);
    return FwdRoute{from_packed && p.bits == 3 && p.T > 2 * tokens && rounds_of(p, tokens) > 1 ? FWD_RELAY_MID : FWD_MID, tokens, kMidBN};
}

double mid_us(const Problem &p) { return launch_us(p, token_tile(p)); }

// The small launch that pairs step sizes and zero points takes 2 us beside the forward.  Without it the forward fetches twice the cache lines of them a K step, with groups of 64 and
// more: 200 random sizes of 256 to 16000 inputs, 65 to 2000 tokens, us, with that launch / without:
// - one group to a row: 288 -> 544 8.6 / 6.6, 7360 -> 1144 38.1 / 36.1, 14624 -> 1880 91.5 / 89.7; with the backward, 14880 -> 1408 193.9 / 191.9;
// - groups of 32: 8160 -> 1856 54.8 / 46.7, 13856 -> 3640 97.8 / 95.2.  A forward that leaves many pairs for few workgroups to write loses, though: with the backward 4928 -> 7368
//   107.5 / 104.3, 14016 -> 1272, 82 tokens 117.9 / 126.4;
// - others gain up to 24 steps of 256 inputs, counted over the rounds of workgroups: 3200 -> 2360 19.4 / 17.7, 4992 -> 4096 37.5 / 36.1, 6592 -> 208 32.0 / 32.4, 9216 -> 1096 40.5 / 41.2, 14464 -> 544
//   70.2 / 77.9; two rounds, 7424 -> 3672 with the backward 218.6 / 222.3.
bool mid_pairs_itself(const Problem &p, bool keep)
{
    if (mid_us(p) > 120.0) return false;
    return p.G == 1 || (p.g == 32 && !keep) || rounds_of(p, token_tile(p)) * ((p.I + kMidBK - 1) / kMidBK) <= 24;
}

// Against k_gemm_ksplit while there are at most 256 tiles of 128 x 128 (with one workgroup per tile 4.8 us and 0.8 to 1.1, with
// the fill, a pair of 64-wide K tiles; 1024 inputs, 2000 tokens, 2048 rows: 12 us there, 14 here).  With more than 640 inputs one
// round of 64- or 96-token tiles runs here whatever these estimates say.  Where the contraction is short they leave out what a
// launch there costs beside its K tiles: us, here / there, from the packed arrays 443 tokens, 832 x 552 10.1 / 15.2, from a prepared
// layer 109 tokens, 896 x 1680 12.0 / 14.3, and in all of 64 sizes between 672 and 1280 inputs by 1 to 80 %.  Where it is long
// and the tiles are few, several workgroups share a tile there, which this rule does not weigh: from the packed arrays / prepared,
// 128 tokens, 28672 x 8192 121 here and 127 there / 113 and 106; 256 tokens, 11008 x 4096 49 and 51 / 48 and 46; 256 tokens, 8192 x 1024
// 36 and 31 / 35 and 27.
// Against the 128 x 128-tile kernel with two tiles per compute unit beyond 256 tiles (0.9 us per K tile; 11008 x 4096: 288 tokens,
// 258 tiles 61 us there and 42 here; 400 tokens 63 and 51).  More than two rounds here, or more than two tiles per compute unit there: the 256 x 256 tiles are the better kernel.  The GEMMs
// alone are compared: a forward from the packed arrays saves the re-layout as well and would gain a little earlier, but every
// forward entry point shares the rule, so that their results stay bitwise equal.
bool mid_applies(const Problem &p)
{
    if (!p.act_bf16 || !group_by_magic(p) || p.T <= 32) return false;
    if (p.T <= 64) return !gemv_work_applies(p);
    const int64_t tiles = ((p.T + 127) / 128) * ((p.O + 127) / 128);
    const int bm = token_tile(p);
    if (tiles <= 256 && p.I > 640 && bm < 128 && rounds_of(p, bm) == 1) return true;
    const double other = tiles <= 256 ? 4.8 + (double)((p.I + 127) / 128) * (0.8 + 0.3 * (double)tiles / 256.0)
                                      : 4.0 + (double)((p.I + 63) / 64) * 0.9;
    return tiles <= 512 && mid_us(p) < other;
}

void launch_mid(const Problem &p, const void *X, const void *Wpacked, const float *s, const void *zpacked, const float *zfloat,
                void *Y, hipStream_t st)
{
    const MidArgs a = packed_args(p, X, Wpacked, s, zpacked, zfloat, Y);
    if (zfloat != nullptr) launch_src<kFloatZ>(p, a, st); else launch_src<kPackedZ>(p, a, st);
}

void launch_mid_work(const Problem &p, const void *X, const void *codes, const void *sz, void *Y, hipStream_t st)
{
    MidArgs a = mid_args(p, X, codes, sz, Y);
    a.code_row_bytes = (uint32_t)(work_code_bytes(p) / p.O);
    a.codes_bytes = (uint32_t)work_code_bytes(p);
    a.s_bytes = (uint32_t)(p.O * p.G * 8);
    launch_src<kWorking>(p, a, st);
}

void launch_mid_prepared(const Problem &p, const void *X, const void *codes, const float *s, const float *z, void *pairs, void *Y, hipStream_t st)
{
    MidArgs a = prepared_args(p, X, codes, s, z, Y);
    a.pairs = (float *)pairs;
    launch_src<kPrepared>(p, a, st);
}

}  // namespace eqat
