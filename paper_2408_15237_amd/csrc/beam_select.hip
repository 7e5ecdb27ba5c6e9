// Beam search's choice over all beams and the vocabulary.
#include "decode_internal.h"

namespace ssmv {
namespace {

typedef unsigned long long Key;

// A candidate of a row as a whole number: larger is better - the logit in an order-preserving form above, the token's
// complement below, so that keys are unique and equal logits go by the lower token.  0 stands for none.
__device__ __forceinline__ Key key_of(float v, unsigned token)
{
    unsigned u = __float_as_uint(v + 0.f);                                        // -0 + 0 = 0
    u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (Key)u << 32 | (0xffffffffu - token);
}
__device__ __forceinline__ float key_logit(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ unsigned key_token(Key k) { return 0xffffffffu - (unsigned)k; }

// NaN is a token that is not allowed, +inf the largest finite logit
__device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : fminf(v, 3.402823466e+38f); }

constexpr int THREADS = 256, E = kBeamPiece / THREADS;

// The best `keep` candidates of a piece of a row, best first, and its part of the row's sum.
// The keep-th largest of the threads' best keys is a bound that at least `keep` candidates reach, and only the keep threads at or above
// it can hold any: what reaches it is collected (at most keep * E keys, usually little more than keep) and ranked.
template <int IO, bool VEC>
__global__ __launch_bounds__(THREADS) void beam_piece_kernel(const BeamParams p)
{
    __shared__ Key sBest[THREADS];
    __shared__ Key sList[SSMV_BEAMS_MAX * E];
    __shared__ float sMax[THREADS / 64], sSum[THREADS / 64];
    __shared__ Key sBound;
    __shared__ int sCount;
    const unsigned tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const unsigned piece = blockIdx.x;
    const size_t row = blockIdx.y;
    if (p.done && p.done[row] != 0) return;                                       // a finished row's logits are not read
    const unsigned first = piece * kBeamPiece, n = min((unsigned)p.V - first, (unsigned)kBeamPiece);
    constexpr int EV = VEC ? IoVec<IO>::EV : 1;
    float v[E];
    const size_t at = row * p.row_stride + first;
    auto token = [&](int i) { return (unsigned)(i / EV) * (THREADS * EV) + tid * EV + i % EV; };       // of the piece
#pragma unroll
    for (int i = 0; i < E; i += EV) {
        const unsigned t = token(i);
        if constexpr (VEC) {
            float d[EV];
            if (t + EV <= n) {
                IoVec<IO>::load(p.logits, at + t, d);
#pragma unroll
                for (int j = 0; j < EV; ++j) v[i + j] = clean(d[j]);
            } else {
#pragma unroll
                for (int j = 0; j < EV; ++j) v[i + j] = t + j < n ? clean(load_io(p.logits, at + t + j, IO)) : -INFINITY;
            }
        } else {
            v[i] = t < n ? clean(load_io(p.logits, at + t, IO)) : -INFINITY;
        }
    }
    // ---- the piece's largest logit and sum
    float m = -3.402823466e+38f;
#pragma unroll
    for (int i = 0; i < E; ++i) m = fmaxf(m, v[i]);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) sMax[wave] = m;
    Key best = 0;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (token(i) < n) {
            const Key k = key_of(v[i], first + token(i));
            best = k > best ? k : best;
        }
    sBest[tid] = best;
    if (tid == 0) { sCount = 0; sBound = 1; }                                     // 1: every candidate there is
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) m = fmaxf(m, sMax[w]);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += __builtin_amdgcn_exp2f((v[i] - m) * 1.4426950408889634f);
#pragma unroll
    for (int o = 32; o > 0; o /= 2) sum += __shfl_xor(sum, o);
    if (lane == 0) sSum[wave] = sum;
    int rank = 0;
    for (int i = 0; i < THREADS; ++i) rank += sBest[i] > best;
    if (best != 0 && rank == p.keep - 1) sBound = best;                           // keys are unique: one thread at most
    __syncthreads();
    if (tid == 0) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) s += sSum[w];
        p.sums[row * p.pieces + piece] = make_float2(m, s);
    }
    const Key bound = sBound;
    if (best >= bound) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if (token(i) >= n) continue;
            const Key k = key_of(v[i], first + token(i));
            if (k >= bound) sList[atomicAdd(&sCount, 1)] = k;
        }
    }
    __syncthreads();
    const int count = sCount;
    Key *out = p.keys + (row * p.pieces + piece) * p.keep;
    for (int i = tid; i < count; i += THREADS) {
        const Key k = sList[i];
        int r = 0;
        for (int j = 0; j < count; ++j) r += sList[j] > k;
        if (r < p.keep) out[r] = k;
    }
    for (int i = count + tid; i < p.keep; i += THREADS) out[i] = 0;
}

// how many of a list's n keys, best first, are larger
__device__ __forceinline__ int larger(const Key *list, int n, Key k)
{
    int lo = 0;
    while (n > 0) {
        const int half = n / 2;
        if (list[lo + half] > k) { lo += half + 1; n -= half + 1; }
        else n = half;
    }
    return lo;
}

// A workgroup per sequence: the pieces of each row merged, then the rows.  A candidate's place is its place in its own list plus the
// number of better ones in each other list (they are sorted).
__global__ __launch_bounds__(THREADS) void beam_merge_kernel(const BeamParams p)
{
    __shared__ Key sKeys[SSMV_BEAMS_MAX * SSMV_BEAMS_MAX];
    __shared__ double sScore[SSMV_BEAMS_MAX * SSMV_BEAMS_MAX];
    const unsigned tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const int W = p.beams_in, keep = p.keep;
    const size_t row0 = (size_t)blockIdx.x * W;
    for (int r = wave; r < W; r += THREADS / 64) {
        const size_t row = row0 + r;
        float given = p.scores[row];
        given = given != given ? -INFINITY : fminf(given, 3.402823466e+38f);
        if (p.done && p.done[row] != 0) {
            for (int i = lane; i < keep; i += 64) {
                sKeys[r * keep + i] = key_of(0.f, (unsigned)p.eos);
                sScore[r * keep + i] = i == 0 ? (double)given : -INFINITY;
            }
            continue;
        }
        const float2 *sums = p.sums + row * p.pieces;
        float m = -3.402823466e+38f;
        for (int i = lane; i < p.pieces; i += 64) m = fmaxf(m, sums[i].x);
        for (int o = 32; o > 0; o /= 2) m = fmaxf(m, __shfl_xor(m, o));
        double s = 0.0;
        for (int i = lane; i < p.pieces; i += 64) s += (double)sums[i].y * (double)__builtin_amdgcn_exp2f((sums[i].x - m) * 1.4426950408889634f);
        for (int o = 32; o > 0; o /= 2) s += __shfl_xor(s, o);
        const double lse = log(s);
        const Key *lists = p.keys + row * p.pieces * keep;
        for (int i = lane; i < p.pieces * keep; i += 64) {
            const Key k = lists[i];
            if (k == 0) continue;
            const int own = i / keep;
            int rank = i - own * keep;
            for (int q = 0; q < p.pieces; ++q)
                if (q != own) rank += larger(lists + q * keep, keep, k);
            if (rank < keep) {
                const float l = key_logit(k);
                sKeys[r * keep + rank] = k;
                sScore[r * keep + rank] = l == -INFINITY ? -INFINITY : (double)given + ((double)l - (double)m - lse);
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < W * keep; i += THREADS) {
        const int r = i / keep;
        const double s = sScore[i];
        int rank = i - r * keep;
        for (int q = 0; q < W; ++q) {
            if (q == r) continue;
            int lo = 0, n = keep;                                                 // better: a larger score, or the same in a lower row
            while (n > 0) {
                const int half = n / 2;
                const double o = sScore[q * keep + lo + half];
                if (o > s || (o == s && q < r)) { lo += half + 1; n -= half + 1; }
                else n = half;
            }
            rank += lo;
        }
        if (rank < p.beams_out) {
            const size_t at = (size_t)blockIdx.x * p.beams_out + rank, row = row0 + r;
            const int token = (int)key_token(sKeys[i]);
            p.parent[at] = (int32_t)row;
            p.token[at] = token;
            p.scores_out[at] = (float)s;
            if (p.done_out) p.done_out[at] = (p.done && p.done[row] != 0) || token == p.eos;
        }
    }
}

}  // namespace

int launch_beam_select(const BeamParams &p, hipStream_t stream)
{
    const unsigned rows = (unsigned)p.batch * p.beams_in;
    if (rows > 65535) return (int)hipErrorInvalidValue;                                    // refused by the host's checks
    const dim3 grid((unsigned)p.pieces, rows);
    if (p.io == SSMV_BF16) {
        if (p.vec) hipLaunchKernelGGL((beam_piece_kernel<SSMV_BF16, true>), grid, dim3(THREADS), 0, stream, p);
        else hipLaunchKernelGGL((beam_piece_kernel<SSMV_BF16, false>), grid, dim3(THREADS), 0, stream, p);
    } else {
        if (p.vec) hipLaunchKernelGGL((beam_piece_kernel<SSMV_F32, true>), grid, dim3(THREADS), 0, stream, p);
        else hipLaunchKernelGGL((beam_piece_kernel<SSMV_F32, false>), grid, dim3(THREADS), 0, stream, p);
    }
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    hipLaunchKernelGGL(beam_merge_kernel, dim3((unsigned)p.batch), dim3(THREADS), 0, stream, p);
    return (int)hipGetLastError();
}

}  // namespace ssmv
