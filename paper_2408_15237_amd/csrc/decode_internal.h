// Parameter blocks and launchers of plain and beam decoding: the calls that move a sequence from state to state without a cache
// (causal_conv.hip, selective_scan.hip, selective_step.hip, beam_select.hip).
#pragma once

#include "ssmv_internal.h"

namespace ssmv {

// log(1 + e^v) for all v: max(v, 0) + log(1 + t), t = e^-|v|; what the rounding of w = 1 + t loses of a small t is given back, as
// log(w + r) = log(w) + r to within 2^-25 for w in [1, 2].  Within 2e-7 of the exact value for every t, where the plain log(1 + t) is
// off by 4e-6 at t = 2^-6; no select and no series.
__device__ __forceinline__ float softplus_exact(float v)
{
    const float t = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(v)), w = 1.f + t;
    return fmaf(__builtin_amdgcn_logf(w), 0.69314718055994531f, t - (w - 1.f)) + fmaxf(v, 0.f);
}

// A log2 e, finite: times the step 0 of a token that is none it must give 0, also where A is -inf.  (Steps below 2^-121 then leave
// something of the state: exp2 of the lowest finite value times so little is not 0.)
__device__ __forceinline__ float decay_rate(float A)
{
    const float a = A * 1.4426950408889634f;
    return a < -3.402823466e+38f ? -3.402823466e+38f : a;
}

struct CausalConvParams {
    const void *x, *wgt, *bias, *conv_in;
    const int32_t *src_row, *seq_len;
    void *out, *conv_out;
    size_t x_stride, out_stride;
    int batch, rows_in, C, L, io, act;
};

struct ScanParams {
    const void *x, *dt, *Bm, *Cm, *z;
    const float *dt_bias, *A, *D, *h_in;
    const int32_t *src_row, *seq_len;
    void *y;
    float *h_out;
    size_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
    int batch, rows_in, C, N, L, io, softplus;
    int channels_wg;         // channels of a workgroup: 64, 32, 16
    int seg_len, seg_count;  // a cut prompt: tokens of a segment, segments of the longest prompt; seg_count 1: not cut
    float *seg_h;            // [batch][seg_count][C][N] end states of the segments, the first slice of each sequence; see selective_scan.hip
    float *seg_dt;           // [batch][seg_count][C]    their sums of step sizes
};

struct TokenParams {
    const void *x, *dt, *Bm, *Cm, *z;
    const float *dt_bias, *A, *D, *h_in;
    const int32_t *src_row;
    void *y;
    float *h_out;
    size_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
    int rows, rows_in, H, P, N, G, io, diag, softplus;
};

struct BeamParams {
    const void *logits;
    const float *scores;
    const int32_t *done;
    int32_t *parent, *token;
    float *scores_out;
    int32_t *done_out;
    size_t row_stride;
    int batch, beams_in, beams_out, V, io, eos;
    int small, pieces, piece_len, chunks;   // see BeamPlan
    int keep;                // candidates kept of a row: min(beams_out, V)
    unsigned long long *keys;    // [row][piece][keep] the best of a part, best first; 0 = none
    float2 *sums;                // [row][piece] largest logit, sum of exp(logit - largest)
};

struct ConvHistoryParams {
    int batch, R, Cx, io;
    const void *ring;
    const int32_t *conv_head;
    void *out;
};

// ---- how a prompt is cut and a row of logits divided: the workspaces follow from it --------------------------------------

constexpr int kScanTile = 64;        // tokens of a segment: a multiple of this

struct ScanPlan {
    int channels;            // of a workgroup: 64, 32 or 16
    int seg_len, seg_count;  // tokens of a segment, segments of the longest prompt
};

// Which width of workgroup, and how many segments: the least time by a model of the kernel, whose constants were measured.  Of a
// token a workgroup that has a compute unit to itself takes lone = 15 + N ns (16 channels), 18 + 1.6 N (32), 35 + 2.6 N (64); a compute
// unit with k of them takes k times 14 + 0.75 N (N = 64: its LDS has room for one, k times lone), 15 + 1.3 N, 22 + 2.5 N where that is more.  A cut prompt costs a pass over all
// segments but the last that forms their end states (0.65 of a full pass), and 5 us.
// (us, N = 16, 2048 tokens, 64 / 32 / 16 channels: 1 x 8192 140 / 79 / 91, in 8 segments 106 / 112 / 139; 1 x 1536 137 / 78 / 55, in 16 segments
//  36 / 30 / 37; 8 x 5120 342 / 334 / 427; 16 x 8192 909 / 1045 / 1336, in 8 segments 1481 / 1732 / 2131; N = 64, 32 / 16
//  channels: 1 x 4096 x 64 64 / 45, 4 x 600 x 1024 69 / 59, 1 x 183 x 343 23 / 18.  Over 29 shapes, of 1 to 32 sequences, 64 to
//  8192 channels and all N, its choice is the best of up to 24 in 23, and 1 to 6 % slower than the best in the others.)
inline ScanPlan scan_plan(int batch, int C, int N, int L)
{
    const int tiles = (L + kScanTile - 1) / kScanTile;
    ScanPlan best{64, L, 1};
    double least = 1e30;
    for (int w = 64; w >= 16; w /= 2) {
        const double lone = w == 64 ? 35 + 2.6 * N : w == 32 ? 18 + 1.6 * N : 15 + 1.0 * N;
        const double busy = w == 64 ? 22 + 2.5 * N : w == 32 ? 15 + 1.3 * N : N == 64 ? lone : 14 + 0.75 * N;
        const double groups = (double)batch * ((C + w - 1) / w);
        for (int want = 1; want <= 16 && want <= tiles; ++want) {
            const int len = (tiles + want - 1) / want * kScanTile, count = (L + len - 1) / len;
            if (count != want) continue;
            auto pass = [&](double g) {
                const double k = (double)(long)((g + 255) / 256) * busy;
                return 1e-3 * (count > 1 ? len : L) * (k > lone ? k : lone);
            };
            const double us = pass(groups * count) + (count > 1 ? 0.65 * pass(groups * (count - 1)) + 5.0 : 0.0);
            if (us < least) {
                least = us;
                best = ScanPlan{w, count > 1 ? len : L, count};
            }
        }
    }
    return best;
}

constexpr int kSmallKeep = 16;       // candidates of a small piece at most
constexpr int kMergeKeys = 8192;     // keys that the merge of a sequence has room for: of three rows at least
__host__ __device__ constexpr int merge_room(int n) { return (n + 2) / 2 * 2; }    // of a row's n: pairs, and a place behind the last

struct BeamPlan {
    int small;               // 1: chunks of 2048 logits, 0: of 8192
    int pieces, len, chunks; // pieces of a row; logits of a piece (the last one's may be fewer); chunks of a piece
};

// Small chunks where large ones would be too few to fill the chip, and few candidates are kept of each.  Of large ones a piece takes
// several where that leaves 1024 workgroups: as many as run at once with bf16 logits (four on a compute unit; of fp32 ones, with 131 registers, three).
inline BeamPlan beam_plan(int rows, int V, int keep)
{
    BeamPlan r;
    r.small = (long)rows * ((V + 8191) / 8192) < 512 && keep <= kSmallKeep && V <= 64 * 2048;
    const int chunk = r.small ? 2048 : 8192, all = (V + chunk - 1) / chunk, align = r.small ? 8 : 64;
    const int enough = (1024 + rows - 1) / rows, most = r.small ? 64 : enough < 32 ? enough : 32;
    const int pieces = all < most ? all : most;
    r.len = ((V + pieces - 1) / pieces + align - 1) / align * align;   // pieces alike: one that is nearly empty has no bound to offer
    r.pieces = (V + r.len - 1) / r.len;
    r.chunks = (r.len + chunk - 1) / chunk;
    return r;
}

int launch_causal_conv(const CausalConvParams &p, hipStream_t stream);
int launch_selective_scan(const ScanParams &p, hipStream_t stream);
int launch_selective_step(const TokenParams &p, hipStream_t stream);
int launch_beam_select(const BeamParams &p, hipStream_t stream);
int launch_conv_history(const ConvHistoryParams &p, hipStream_t stream);

}  // namespace ssmv
