// The gated linear recurrence over a sequence, from state to state, and over one token of every row.
#include "gated_common.h"

namespace ssmv {
namespace {

// decay and m of a token: see the header
template <bool LRU>
__device__ __forceinline__ void coefficients(float f, float rate, float &a, float &m)
{
    if constexpr (LRU) {
        const float q = rate * sigmoid(f);
        a = __builtin_amdgcn_exp2f(q);
        m = __builtin_amdgcn_sqrtf(one_minus_square(q, a));
    } else {
        sigmoids(f, a, m);
    }
}

// h <- a h + v: a run of tokens is the pair (product of a, state that it leaves from zero), and pairs combine in order.  A lane forms the pair of its run, the lanes of a
// wave and then the waves of the workgroup combine theirs (LDS, one barrier a tile), and every lane goes through its run again from the state that it starts from.  So a
// token is read once; the gates stay in registers between the two walks.
// OUT false: only the pairs of whole segments, of all but the last.
template <int IO, int CL, bool LRU, bool OUT>
__global__ __launch_bounds__(64 * kGatedWaves) void gated_recurrence_kernel(const GatedParams p)
{
    using Ln = GatedLane<IO, CL>;
    constexpr int CH = Ln::CH, G = Ln::G, T = Ln::T, K = kGatedRun, W = kGatedWaves;
    __shared__ __attribute__((aligned(16))) float pairs[2][W][CL][2 * CH];
    const unsigned lane = threadIdx.x & 63u, cl = lane % CL, grp = lane / CL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = (int)xcd_contiguous(blockIdx.x, gridDim.x) * Ln::CW + (int)cl * CH, live = min(max(p.C - c0, 0), CH), seg = blockIdx.y;
    int b = blockIdx.z;
    if (p.seq_len && p.batch > 1 && p.batch <= 64) b = zth_longest(p.seq_len, p.batch, b, lane);
    const int all = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    const int from = seg * p.seg_len, len = min(all, from + p.seg_len);
    const bool last = len == all;
    if (seg > 0 && (OUT ? from >= all : last)) return;
    const size_t seg0 = (size_t)b * p.seg_count * p.C + c0;

    float h[CH], prod[CH], rate[CH], fb[CH], ib[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        h[c] = 0.f;
        prod[c] = 1.f;
        rate[c] = LRU && c < live ? decay_exponent(p.A[c0 + c]) : 0.f;
        fb[c] = p.f_bias && c < live ? p.f_bias[c0 + c] : 0.f;
        ib[c] = p.i_bias && c < live ? p.i_bias[c0 + c] : 0.f;
    }
    if (seg == 0) {
        const int src = p.src_row ? p.src_row[b] : b;
        if (OUT && p.seg_count > 1) load_channels<CH>(p.seg_h + seg0 + (size_t)(p.seg_count - 1) * p.C, live, h);    // h_out may be h_in, and its writer another workgroup
        else if (p.h_in && (unsigned)src < (unsigned)p.rows_in) load_channels<CH>(p.h_in + (size_t)src * p.C + c0, live, h);
        if (!OUT && wave == 0 && grp == 0) store_channels<CH>(p.seg_h + seg0 + (size_t)(p.seg_count - 1) * p.C, live, h);
        if (!OUT && last) return;
    } else if (OUT) {
        load_channels<CH>(p.seg_h + seg0, live, h);
        for (int j = 1; j < seg; ++j) {
            float sp[CH], sh[CH];
            load_channels<CH>(p.seg_p + seg0 + (size_t)j * p.C, live, sp);
            load_channels<CH>(p.seg_h + seg0 + (size_t)j * p.C, live, sh);
#pragma unroll
            for (int c = 0; c < CH; ++c) h[c] = fmaf(sp[c], h[c], sh[c]);
        }
    }

    const size_t tok0 = (size_t)b * p.L;
    const int run0 = (wave * G + (int)grp) * K;                     // the lane's tokens in a tile
    auto offset = [&](size_t stride) { return (unsigned)((grp * K * (unsigned)stride + (unsigned)c0) * Ln::ES); };
    const unsigned ox = offset(p.x_stride), of = offset(p.f_stride), oi = offset(p.i_stride), oz = offset(p.z_stride), oy = offset(p.y_stride);
    uint32_t rx[K], rf[K], ri[K], rz[K];
    auto fetch = [&](int t0) {
        const size_t at = tok0 + t0 + wave * G * K;
        Ln::load_run(rx, p.x, p.x_stride, at, ox, live, t0 + run0, len);
        Ln::load_run(rf, p.f, p.f_stride, at, of, live, t0 + run0, len);
        if (p.i) Ln::load_run(ri, p.i, p.i_stride, at, oi, live, t0 + run0, len);
        if (OUT && p.z) Ln::load_run(rz, p.z, p.z_stride, at, oz, live, t0 + run0, len);
    };
    if (from < len) fetch(from);
    for (int t0 = from, buf = 0; t0 < len; t0 += T, buf ^= 1) {
        const int t = t0 + run0;
        float a[K][CH], v[K][CH], gate[OUT ? K : 1][CH];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float f[CH], x[CH];
            Ln::decode(rf[k], f);
            Ln::decode(rx[k], x);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float m;
                coefficients<LRU>(f[c] + fb[c], rate[c], a[k][c], m);
                v[k][c] = m * x[c];
            }
        }
        if (p.i) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float g[CH];
                Ln::decode(ri[k], g);
#pragma unroll
                for (int c = 0; c < CH; ++c) v[k][c] *= sigmoid(g[c] + ib[c]);
            }
        }
        if (OUT && p.z) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float z[CH];
                Ln::decode(rz[k], z);
#pragma unroll
                for (int c = 0; c < CH; ++c) gate[OUT ? k : 0][c] = z[c] * sigmoid(z[c]);
            }
        }
        if (t + K > len) {                                          // tokens that are none leave the state as it is
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    a[k][c] = t + k < len ? a[k][c] : 1.f;
                    v[k][c] = t + k < len ? v[k][c] : 0.f;
                }
        }
        if (t0 + T < len) fetch(t0 + T);
        float P[CH], H[CH], Pe[CH], He[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            P[c] = a[0][c];
            H[c] = v[0][c];
#pragma unroll
            for (int k = 1; k < K; ++k) {
                P[c] *= a[k][c];
                H[c] = fmaf(a[k][c], H[c], v[k][c]);
            }
            Pe[c] = 1.f;
            He[c] = 0.f;
            if constexpr (G > 1) {
#pragma unroll
                for (int d = CL; d < 64; d *= 2) {
                    const float p1 = __shfl_up(P[c], d), h1 = __shfl_up(H[c], d);
                    if ((int)lane >= d) {
                        H[c] = fmaf(P[c], h1, H[c]);
                        P[c] *= p1;
                    }
                }
                const float p1 = __shfl_up(P[c], CL), h1 = __shfl_up(H[c], CL);
                Pe[c] = grp > 0 ? p1 : 1.f;
                He[c] = grp > 0 ? h1 : 0.f;
            }
        }
        if (grp == G - 1) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs[buf][wave][cl][c] = P[c];
                pairs[buf][wave][cl][CH + c] = H[c];
            }
        }
        __syncthreads();
        float start[CH];
#pragma unroll
        for (int w = 0; w < W; ++w) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (w == wave) start[c] = h[c];
                const float pw = pairs[buf][w][cl][c];
                h[c] = fmaf(pw, h[c], pairs[buf][w][cl][CH + c]);
                if (!OUT) prod[c] *= pw;
            }
        }
        if constexpr (OUT) {
#pragma unroll
            for (int c = 0; c < CH; ++c) start[c] = fmaf(Pe[c], start[c], He[c]);
            if (p.states && t % SSMV_GATED_TILE == 0 && t < len)
                store_channels<CH>(p.states + ((size_t)b * ((p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE) + t / SSMV_GATED_TILE) * p.C + c0, live, start);
            char *row = static_cast<char *>(p.y) + (tok0 + t0 + wave * G * K) * p.y_stride * Ln::ES;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float y[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    start[c] = fmaf(a[k][c], start[c], v[k][c]);
                    y[c] = p.z ? start[c] * gate[k][c] : start[c];
                }
                if (t + k < len) Ln::store(row + k * p.y_stride * Ln::ES, oy, live, y);
            }
        }
    }
    if (wave != 0 || grp != 0) return;
    if constexpr (OUT) {
        if (last && p.h_out) store_channels<CH>(p.h_out + (size_t)b * p.C + c0, live, h);
        if (all == 0 && p.states) store_channels<CH>(p.states + (size_t)b * ((p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE) * p.C + c0, live, h);
    } else {
        store_channels<CH>(p.seg_h + seg0 + (size_t)seg * p.C, live, h);
        store_channels<CH>(p.seg_p + seg0 + (size_t)seg * p.C, live, prod);
    }
}

// One token of every row: a lane per 4 bytes of it.
template <int IO, bool LRU>
__global__ __launch_bounds__(256) void gated_token_kernel(const GatedParams p)
{
    using Ln = GatedLane<IO, 64>;
    constexpr int CH = Ln::CH;
    const int c0 = ((int)blockIdx.x * 256 + (int)threadIdx.x) * CH, live = min(max(p.C - c0, 0), CH), b = blockIdx.y;
    if (live == 0) return;
    const bool none = p.seq_len && p.seq_len[b] <= 0;
    const int src = p.src_row ? p.src_row[b] : b;
    auto at = [&](const void *t, size_t stride) { return static_cast<const char *>(t) + (size_t)b * stride * Ln::ES; };
    const unsigned off = (unsigned)c0 * Ln::ES;
    float h[CH], x[CH], f[CH], i[CH], z[CH];
    uint32_t rx = 0, rf = 0, ri = 0, rz = 0;
    if (!none) {
        rx = Ln::load(at(p.x, p.x_stride), off, live);
        rf = Ln::load(at(p.f, p.f_stride), off, live);
        if (p.i) ri = Ln::load(at(p.i, p.i_stride), off, live);
        if (p.z) rz = Ln::load(at(p.z, p.z_stride), off, live);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) h[c] = 0.f;
    if (p.h_in && (unsigned)src < (unsigned)p.rows_in) load_channels<CH>(p.h_in + (size_t)src * p.C + c0, live, h);
    if (p.states) store_channels<CH>(p.states + (size_t)b * p.C + c0, live, h);
    Ln::decode(rx, x);
    Ln::decode(rf, f);
    Ln::decode(ri, i);
    Ln::decode(rz, z);
    float y[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int ch = min(c0 + c, p.C - 1);
        float a, m;
        coefficients<LRU>(f[c] + (p.f_bias ? p.f_bias[ch] : 0.f), LRU ? decay_exponent(p.A[ch]) : 0.f, a, m);
        float v = m * x[c];
        if (p.i) v *= sigmoid(i[c] + (p.i_bias ? p.i_bias[ch] : 0.f));
        if (!none) h[c] = fmaf(a, h[c], v);
        y[c] = p.z ? h[c] * (z[c] * sigmoid(z[c])) : h[c];
    }
    if (!none) Ln::store(const_cast<char *>(at(p.y, p.y_stride)), off, live, y);
    if (p.h_out) store_channels<CH>(p.h_out + (size_t)b * p.C + c0, live, h);
}

template <int IO, int CL, bool LRU>
int launch(const GatedParams &p, hipStream_t stream)
{
    constexpr int CW = GatedLane<IO, CL>::CW;
    const unsigned groups = (unsigned)((p.C + CW - 1) / CW);
    const dim3 block(64 * kGatedWaves);
    if (p.seg_count > 1) {
        hipLaunchKernelGGL((gated_recurrence_kernel<IO, CL, LRU, false>), dim3(groups, p.seg_count - 1, p.batch), block, 0, stream, p);
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL((gated_recurrence_kernel<IO, CL, LRU, true>), dim3(groups, p.seg_count, p.batch), block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, bool LRU>
int launch_lanes(const GatedParams &p, hipStream_t stream)
{
    if (p.L == 1) {
        constexpr int per = 256 * GatedLane<IO, 64>::CH;
        hipLaunchKernelGGL((gated_token_kernel<IO, LRU>), dim3((p.C + per - 1) / per, p.batch), dim3(256), 0, stream, p);
        return (int)hipGetLastError();
    }
    switch (p.lanes) {
        case 64: return launch<IO, 64, LRU>(p, stream);
        case 32: return launch<IO, 32, LRU>(p, stream);
        case 16: return launch<IO, 16, LRU>(p, stream);
        case 8: return launch<IO, 8, LRU>(p, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_gated_recurrence(const GatedParams &p, hipStream_t stream)
{
    if (p.io == SSMV_BF16) return p.lru ? launch_lanes<SSMV_BF16, true>(p, stream) : launch_lanes<SSMV_BF16, false>(p, stream);
    return p.lru ? launch_lanes<SSMV_F32, true>(p, stream) : launch_lanes<SSMV_F32, false>(p, stream);
}

}  // namespace ssmv
