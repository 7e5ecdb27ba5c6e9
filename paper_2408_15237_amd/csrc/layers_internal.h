// Parameter blocks, launchers and common device code of the layer operators (block_norm.hip, gated_recurrence.hip, gated_backward.hip,
// logit_rules.hip).
#pragma once

#include "ssmv_internal.h"
#include "ssmv_layers.h"

namespace ssmv {

struct BlockNormParams {
    const void *x, *z, *res;
    const float *post, *scale, *pre;
    void *r_out, *n_out;
    size_t x_stride, z_stride, res_stride, r_stride, n_stride;
    int rows, C, io, res_io;
    float eps, alpha;
};

struct BlockNormGradParams {
    const void *x, *z, *res;
    const float *post, *scale, *pre;
    const void *dr, *dn;
    void *dx, *dz, *dres;
    float *dpost, *dscale, *dpre;
    float *partial;          // [parts][3][C]: dpre, dscale, dpost of a workgroup's rows; NULL: none is wanted
    size_t x_stride, z_stride, res_stride, dr_stride, dn_stride, dx_stride, dz_stride, dres_stride;
    int rows, C, io, res_io, parts;
    float eps, alpha;
};

struct GatedParams {
    const void *x, *f, *i, *z;
    const float *A, *f_bias, *i_bias, *h_in;
    const int32_t *src_row, *seq_len;
    void *y;
    float *h_out, *states;
    size_t x_stride, f_stride, i_stride, z_stride, y_stride;
    int batch, rows_in, C, L, io, lru;
    int wide, seg_len, seg_count;        // see GatedPlan
    int past;                // a large output is stored past the caches
    float *seg_p;            // [batch][seg_count][C] products of the segments' decays
    float *seg_h;            // [batch][seg_count][C] end states of the segments from zero (the first one's from its start); last place: the start state
};

struct GatedGradParams {
    const void *x, *f, *i, *z, *dy;
    const float *A, *f_bias, *i_bias, *states, *dh_out;
    const int32_t *seq_len;
    void *dx, *df, *di, *dz;
    float *dA, *df_bias, *di_bias, *dh_in;
    size_t x_stride, f_stride, i_stride, z_stride, dy_stride, dx_stride, df_stride, di_stride, dz_stride;
    int batch, C, L, io, lru;
    int wide, seg_len, seg_count;
    float *seg_p;            // [batch][seg_count][C] products of the segments' decays
    float *seg_r;            // [batch][seg_count][C] what flows out of a segment's front when nothing flows into its end
    float *partial;          // [batch][seg_count][3][C] sums for A, f_bias, i_bias of a segment's tokens; NULL: none is wanted
};

struct RulesParams {
    const void *logits;
    const int32_t *hist, *hist_len, *src_row, *token, *prompt_len;
    const float *repetition, *frequency, *presence;
    const int32_t *bias_token;
    const float *bias;
    const uint32_t *mask;
    const int32_t *mask_row;
    void *out;
    int32_t *hist_out, *hist_len_out;
    size_t row_stride, out_stride, mask_stride;
    int rows, rows_in, V, io, room, bias_n, mask_rows;
};

int launch_block_norm(const BlockNormParams &p, hipStream_t stream);
int launch_block_norm_backward(const BlockNormGradParams &p, hipStream_t stream);
int launch_gated_recurrence(const GatedParams &p, hipStream_t stream);
int launch_gated_backward(const GatedGradParams &p, hipStream_t stream);
int launch_logit_rules(const RulesParams &p, hipStream_t stream);

// Sums over the rows of partial [parts][n_out][C]: out[k][c], divided by over[c] where that is given (0 where over[c] is 0).
struct ColumnSums {
    float *out[3];
    const float *over[3];
};
int launch_column_sums(const float *partial, int parts, int C, const ColumnSums &to, hipStream_t stream);

// The gradients of vectors are summed over the rows by at most so many workgroups: two on every compute unit.
constexpr int kNormParts = 512;
inline int norm_parts(int rows) { return rows < kNormParts ? rows : kNormParts; }

// How the recurrence is laid on the chip.  A lane takes 4 bytes of a token's row (two bf16 channels, one fp32) for four tokens.  Wide workgroups are 8 waves whose lanes lie 32 over the
// channels, 64 tokens a tile; narrow ones lie 16 over the channels, with 16 waves (forward, 256 tokens a tile) or 8 (backward, 128).
struct GatedPlan {
    int wide;
    int seg_len, seg_count;  // tokens of a segment (whole tiles), segments of the longest sequence
};
// Width and segments: the least time by a model whose constants were measured for LRU with both gates in bf16.  The other forms and fp32 take the same plan, which was not looked for among theirs: with fewer
// tensors or transcendental functions a tile they run ahead of the model's time (1 x 32768 x 1024 MIX without i, us by the model / measured: forward 123 / 95, backward 247 / 163; 4 x 2048 x 5120 fp32 LRU
// 184 / 192 and 376 / 366).  A workgroup that shares a compute unit with few others takes `lone` us a tile,
// a chip with g of them g / 256 times `busy` where that is more.  A cut sequence costs a pass over all segments but one for their pairs (0.65 of a full one, whatever it reads) and 5 us.
// (us, forward, wide whole / narrow whole / best cut: 1 x 2048 x 8192 62 / 50 / 61, 1 x 2048 x 4096 62 / 44 / 38, 1 x 2048 x 1024 59 / 33 / 17, 8 x 2048 x 5120 196 / 233 / 258,
//  2 x 8192 x 2048 233 / 158 / 118; backward: 1 x 2048 x 8192 139 / 96 / 105, 1 x 2048 x 1024 127 / 84 / 28, 8 x 2048 x 5120 386 / 443 / 434.)
inline GatedPlan gated_plan(int batch, int C, int L, int io, bool backward)
{
    const int ch = io == SSMV_BF16 ? 2 : 1;
    GatedPlan best{1, L, 1};
    if (L <= 64) return best;                                       // one tile
    double least = 1e30;
    for (int wide = 1; wide >= 0; --wide) {
        const int lanes = wide ? 32 : 16, tile = wide ? 64 : backward ? 128 : 256, tiles = (L + tile - 1) / tile;
        const double groups = (double)batch * ((C + lanes * ch - 1) / (lanes * ch));
        const double lone = backward ? (wide ? 4.2 : 5.3) : (wide ? 1.95 : 5.0), busy = backward ? (wide ? 4.7 : 6.0) : (wide ? 2.3 : 6.2);
        for (int want = 1; want <= 32 && want <= tiles; want *= 2) {
            const int per = (tiles + want - 1) / want, count = (tiles + per - 1) / per;
            auto pass = [&](double g) { return per * (g / 256 * busy > lone ? g / 256 * busy : lone); };
            const double us = pass(groups * count) + (count > 1 ? 0.65 * pass(groups * (count - 1)) + 5.0 : 0.0);
            if (us < least) {
                least = us;
                best = GatedPlan{wide, count > 1 ? per * tile : L, count};
            }
        }
    }
    return best;
}

// ---- device code --------------------------------------------------------------------------------------------------------

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// 8 adjacent elements at any alignment, `live` of them: the others are not touched and count as 0
template <int T>
__device__ __forceinline__ void load8(const void *base, size_t idx, int live, float (&v)[8])
{
    if (live == 8) {
        if constexpr (T == SSMV_BF16) {
            uint4 r;
            __builtin_memcpy(&r, static_cast<const char *>(base) + idx * 2, sizeof(r));
            IoVec<SSMV_BF16>::decode(r, v);
        } else {
            __builtin_memcpy(v, static_cast<const char *>(base) + idx * 4, sizeof(v));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < live ? load_io(base, idx + j, T) : 0.f;
    }
}

template <int T>
__device__ __forceinline__ void store8(void *base, size_t idx, int live, const float (&v)[8])
{
    if (live == 8) {
        if constexpr (T == SSMV_BF16) {
            const uint4 r = IoVec<SSMV_BF16>::encode(v);
            __builtin_memcpy(static_cast<char *>(base) + idx * 2, &r, sizeof(r));
        } else {
            __builtin_memcpy(static_cast<char *>(base) + idx * 4, v, sizeof(v));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < live) store_io(base, idx + j, v[j], T);
    }
}

// sigmoid(-v ln 2) and 1 minus it, both to within a few roundings for every v
__device__ __forceinline__ void sigmoids_log2(float v, float &s, float &other)
{
    const float t = __builtin_amdgcn_exp2f(-fabsf(v)), w = __builtin_amdgcn_rcpf(1.f + t), tw = t * w;
    s = v > 0.f ? tw : w;
    other = v > 0.f ? w : tw;
}
// sigmoid(v) for e = e^-v, and 1 - sigmoid(v) as e / (1 + e).  Where sigmoid(v) leaves the range of fp32 (v < -87) it is 0 and the other one may be 0, too: for products of both, or with the first.
__device__ __forceinline__ void sigmoid_pair(float e, float &s, float &other)
{
    s = __builtin_amdgcn_rcpf(1.f + e);
    other = fminf(e, 3e38f) * s;
}
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

// A log2 e, finite (a decay of 0 must stay 0 times anything)
__device__ __forceinline__ float decay_exponent(float A)
{
    const float a = A * kLog2e;
    return a < -3.402823466e+38f ? -3.402823466e+38f : a;
}

// 1 - a^2 for a = 2^q, q <= 0.  Near a = 1, where the difference loses it, -expm1(u) at u = 2 q ln 2, |u| < 0.35, by a polynomial of degree 4 for (1 - e^u) / -u (it
// interpolates at the Chebyshev points; with the coefficients as they are stored off by 3.2e-8 of the value, in fp32 by 1.4e-7); elsewhere a^2 is at most 0.71 and its roundings count 2.4 times.
__device__ __forceinline__ float one_minus_square(float q, float a)
{
    float s = fmaf(q, 0.03692220151424408f, 0.1526535451412201f);
    s = fmaf(s, q, 0.44392266869544983f);
    s = fmaf(s, q, 0.9609025716781616f);
    s = fmaf(s, q, 1.3862943649291992f);
    return q > -0.25246699f ? -q * s : fmaf(-a, a, 1.f);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float add_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// the sum over a wave, in every lane
__device__ __forceinline__ float sum_of_wave(float v)
{
    v = add_dpp<0x111, 0xf>(v);     // row_shr:1, 2, 4, 8: lane 15 of a row holds the row's sum
    v = add_dpp<0x112, 0xf>(v);
    v = add_dpp<0x114, 0xf>(v);
    v = add_dpp<0x118, 0xf>(v);
    v = add_dpp<0x142, 0xa>(v);     // row_bcast:15 into rows 1 and 3
    v = add_dpp<0x143, 0xc>(v);     // row_bcast:31 into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// The z-th longest of up to 64 sequences: workgroups start in the order of their indexes, and a long sequence that starts last has the chip to itself.
__device__ __forceinline__ int zth_longest(const int32_t *seq_len, int batch, int z, unsigned lane)
{
    const int mine = (int)lane < batch ? seq_len[lane] : 0;
    int rank = 0;
    for (int i = 0; i < batch; ++i) {
        const int other = __builtin_amdgcn_readlane(mine, i);
        rank += other > mine || (other == mine && i < (int)lane);
    }
    return __builtin_ctzll(__ballot((int)lane < batch && rank == z));
}

}  // namespace ssmv
