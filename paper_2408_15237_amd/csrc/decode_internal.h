// Parameter blocks and launchers of plain and beam decoding: the calls that move a sequence from state to state without a cache
// (causal_conv.hip, selective_scan.hip, selective_step.hip, beam_select.hip).
#pragma once

#include "ssmv_internal.h"

namespace ssmv {

struct CausalConvParams {
    const void *x, *wgt, *bias, *conv_in;
    const int32_t *src_row, *seq_len;
    void *out, *conv_out;
    size_t x_stride, out_stride;
    int batch, rows_in, C, L, io, act;
    int vec;                 // 1: 16-byte accesses everywhere
};

struct ScanParams {
    const void *x, *dt, *Bm, *Cm, *z;
    const float *dt_bias, *A, *D, *h_in;
    const int32_t *src_row, *seq_len;
    void *y;
    float *h_out;
    size_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
    int batch, rows_in, C, N, L, io, softplus;
    int vec;                 // 1: 16-byte accesses of x, dt, z and y
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
    int vec;                 // 1: 16-byte accesses of the logits
    int pieces;              // parts of a row
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

constexpr int kScanTile = 32;        // tokens that a workgroup of the scan takes at a time

// Tokens of a segment and segments of the longest prompt.
inline void scan_cut(int batch, int C, int N, int L, int *seg_len, int *seg_count)
{
    *seg_len = L;
    *seg_count = 1;
}

constexpr int kBeamPiece = 8192;     // logits that a workgroup of the selection takes

inline int beam_pieces(int rows, int V) { return (V + kBeamPiece - 1) / kBeamPiece; }

// Weak: a build of the argument checks alone (api.hip without the kernels) loads without them; its calls end on the host.
__attribute__((weak)) int launch_causal_conv(const CausalConvParams &p, hipStream_t stream);
__attribute__((weak)) int launch_selective_scan(const ScanParams &p, hipStream_t stream);
__attribute__((weak)) int launch_selective_step(const TokenParams &p, hipStream_t stream);
__attribute__((weak)) int launch_beam_select(const BeamParams &p, hipStream_t stream);
__attribute__((weak)) int launch_conv_history(const ConvHistoryParams &p, hipStream_t stream);

}  // namespace ssmv
