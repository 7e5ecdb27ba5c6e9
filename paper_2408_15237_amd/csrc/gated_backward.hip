// The gradients of the gated linear recurrence.
#include "gated_common.h"

namespace ssmv {
namespace {

// h_t = a_t h_{t-1} + v_t,  y_t = h_t silu(z_t).  With g_t = dy_t silu(z_t) and c the gradient that flows into the state from the tokens behind (dh_out at the end):
//   G_t = g_t + c,   c <- a_t G_t          (dh_in at the front)
//   MIX, a = r, m = 1 - r, r = sigmoid(f), u = i x:    df = G r (1 - r) (h_{t-1} - u)
//   LRU, a = e^-s, s = -A r, m = sqrt(1 - a^2), v = m u:
//     E = s dL/ds = G s a (v a / m^2 - h_{t-1}),   df = E (1 - r),   dA = sum E / A        (E falls with sqrt(s) as s goes to 0)
//   dx = G m i,   di = G v (1 - i),   dz = dy h silu'(z)
// The tiles from the last to the first.  A lane's run is the pair (P, H) of the forward pass and, from its last token to its first, the pair (P, R): c <- P c + R, with the
// same product.  Lanes and waves combine both in one exchange: forwards inside 64 tokens, from the state that the forward pass left ahead of them, backwards through the whole tile.
// OUT false: only the pairs (P, R) of whole segments, of all but the first.
template <int IO, int CL, bool LRU, bool OUT>
__global__ __launch_bounds__(64 * kGatedWaves) void gated_backward_kernel(const GatedGradParams p)
{
    using Ln = GatedLane<IO, CL>;
    constexpr int CH = Ln::CH, G = Ln::G, T = Ln::T, K = kGatedRun, W = kGatedWaves;
    constexpr int BW = SSMV_GATED_TILE / (G * K);                   // waves that share a state of the forward pass
    static_assert(BW >= 1 && BW * G * K == SSMV_GATED_TILE && T % SSMV_GATED_TILE == 0, "tile");
    __shared__ __attribute__((aligned(16))) float pairs[2][W][CL][3 * CH];
    const unsigned lane = threadIdx.x & 63u, cl = lane % CL, grp = lane / CL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c0 = (int)xcd_contiguous(blockIdx.x, gridDim.x) * Ln::CW + (int)cl * CH, live = min(max(p.C - c0, 0), CH);
    const int seg = OUT ? blockIdx.y : blockIdx.y + 1;
    int b = blockIdx.z;
    if (p.seq_len && p.batch > 1 && p.batch <= 64) b = zth_longest(p.seq_len, p.batch, b, lane);
    const int all = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    const int from = seg * p.seg_len, len = min(all, from + p.seg_len);
    const bool have = seg == 0 || from < all;                       // segments behind the sequence's end: nothing but zeros in the sums
    const size_t seg0 = (size_t)b * p.seg_count * p.C + c0;
    if (!OUT && !have) return;

    float carry[CH], prod[CH], rate[CH], fb[CH], ib[CH], sumA[CH], sumF[CH], sumI[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        carry[c] = sumA[c] = sumF[c] = sumI[c] = 0.f;
        prod[c] = 1.f;
        rate[c] = LRU && c < live ? decay_exponent(p.A[c0 + c]) : 0.f;
        fb[c] = p.f_bias && c < live ? p.f_bias[c0 + c] : 0.f;
        ib[c] = p.i_bias && c < live ? p.i_bias[c0 + c] : 0.f;
    }
    if (have && (OUT || len == all)) {
        if (p.dh_out) load_channels<CH>(p.dh_out + (size_t)b * p.C + c0, live, carry);
        if (OUT)
            for (int j = (all + p.seg_len - 1) / p.seg_len - 1; j > seg; --j) {      // the last segment's R has dh_out in it
                float sp[CH], sr[CH];
                load_channels<CH>(p.seg_p + seg0 + (size_t)j * p.C, live, sp);
                load_channels<CH>(p.seg_r + seg0 + (size_t)j * p.C, live, sr);
                const bool end = (j + 1) * (size_t)p.seg_len >= (size_t)all;
#pragma unroll
                for (int c = 0; c < CH; ++c) carry[c] = end ? sr[c] : fmaf(sp[c], carry[c], sr[c]);
            }
    }

    const size_t tok0 = (size_t)b * p.L, blocks = (p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE;
    const int run0 = (wave * G + (int)grp) * K;
    auto offset = [&](size_t stride) { return (unsigned)((grp * K * (unsigned)stride + (unsigned)c0) * Ln::ES); };
    const unsigned ox = offset(p.x_stride), of = offset(p.f_stride), oi = offset(p.i_stride), oz = offset(p.z_stride), oy = offset(p.dy_stride);
    const unsigned odx = offset(p.dx_stride), odf = offset(p.df_stride), odi = offset(p.di_stride), odz = offset(p.dz_stride);
    const int tiles = have ? (len - from + T - 1) / T : 0;
    for (int n = tiles - 1, buf = 0; n >= 0; --n, buf ^= 1) {
        const int t0 = from + n * T, t = t0 + run0;
        const size_t at = tok0 + t0 + wave * G * K;
        uint32_t rx[K], rf[K], ri[K], rz[K], ry[K];
        Ln::load_run(rf, p.f, p.f_stride, at, of, live, t, len);
        Ln::load_run(ry, p.dy, p.dy_stride, at, oy, live, t, len);
        if (p.z) Ln::load_run(rz, p.z, p.z_stride, at, oz, live, t, len);
        float begin[CH];
        if constexpr (OUT) {
            Ln::load_run(rx, p.x, p.x_stride, at, ox, live, t, len);
            if (p.i) Ln::load_run(ri, p.i, p.i_stride, at, oi, live, t, len);
            // of the block of 64 tokens; one that has none is not looked at
            const int first = t / SSMV_GATED_TILE * SSMV_GATED_TILE;
#pragma unroll
            for (int c = 0; c < CH; ++c) begin[c] = 0.f;
            if (first < len) load_channels<CH>(p.states + ((size_t)b * blocks + t / SSMV_GATED_TILE) * p.C + c0, live, begin);
        }
        float a[K][CH], v[OUT ? K : 1][CH], g[K][CH];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float f[CH], x[CH], i[CH], z[CH], dy[CH];
            Ln::decode(rf[k], f);
            Ln::decode(ry[k], dy);
            if (OUT) Ln::decode(rx[k], x);
            if (OUT && p.i) Ln::decode(ri[k], i);
            if (p.z) Ln::decode(rz[k], z);
            const bool is = t + k < len;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float m;
                if constexpr (LRU) {
                    const float q = rate[c] * sigmoid(f[c] + fb[c]);
                    a[k][c] = __builtin_amdgcn_exp2f(q);
                    if (OUT) m = __builtin_amdgcn_sqrtf(one_minus_square(q, a[k][c]));
                } else {
                    sigmoids(f[c] + fb[c], a[k][c], m);
                }
                if (OUT) {
                    float w = m * x[c];
                    if (p.i) w *= sigmoid(i[c] + ib[c]);
                    v[OUT ? k : 0][c] = is ? w : 0.f;
                }
                a[k][c] = is ? a[k][c] : 1.f;
                const float d = p.z ? dy[c] * (z[c] * sigmoid(z[c])) : dy[c];
                g[k][c] = is ? d : 0.f;
            }
        }
        float P[CH], H[CH], R[CH], Pf[CH], Hf[CH], Pr[CH], Rr[CH];   // of the run; exclusive over the wave's runs before and behind
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            P[c] = a[0][c];
            H[c] = OUT ? v[0][c] : 0.f;
#pragma unroll
            for (int k = 1; k < K; ++k) {
                P[c] *= a[k][c];
                if (OUT) H[c] = fmaf(a[k][c], H[c], v[OUT ? k : 0][c]);
            }
            R[c] = a[K - 1][c] * g[K - 1][c];
#pragma unroll
            for (int k = K - 2; k >= 0; --k) R[c] = a[k][c] * (g[k][c] + R[c]);
            Pf[c] = Pr[c] = 1.f;
            Hf[c] = Rr[c] = 0.f;
            if constexpr (G > 1) {
                float P2 = P[c];
#pragma unroll
                for (int d = CL; d < 64; d *= 2) {
                    const float p1 = __shfl_up(P[c], d), h1 = __shfl_up(H[c], d), p2 = __shfl_down(P2, d), r2 = __shfl_down(R[c], d);
                    if ((int)lane >= d) {
                        H[c] = fmaf(P[c], h1, H[c]);
                        P[c] *= p1;
                    }
                    if ((int)lane + d < 64) {
                        R[c] = fmaf(P2, r2, R[c]);
                        P2 *= p2;
                    }
                }
                const float p1 = __shfl_up(P[c], CL), h1 = __shfl_up(H[c], CL), p2 = __shfl_down(P2, CL), r2 = __shfl_down(R[c], CL);
                Pf[c] = grp > 0 ? p1 : 1.f;
                Hf[c] = grp > 0 ? h1 : 0.f;
                Pr[c] = grp < G - 1 ? p2 : 1.f;
                Rr[c] = grp < G - 1 ? r2 : 0.f;
            }
        }
        if (grp == G - 1) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs[buf][wave][cl][c] = P[c];
                pairs[buf][wave][cl][CH + c] = H[c];
            }
        }
        if (grp == 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) pairs[buf][wave][cl][2 * CH + c] = R[c];
        }
        __syncthreads();
        float flow[CH];                                             // into the lane's last token
#pragma unroll
        for (int w = W - 1; w >= 0; --w) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (w == wave) flow[c] = carry[c];
                const float pw = pairs[buf][w][cl][c];
                carry[c] = fmaf(pw, carry[c], pairs[buf][w][cl][2 * CH + c]);
                if (!OUT) prod[c] *= pw;
            }
        }
        if constexpr (OUT) {
#pragma unroll
            for (int c = 0; c < CH; ++c) flow[c] = fmaf(Pr[c], flow[c], Rr[c]);
            if constexpr (BW > 1) {
                for (int w = wave / BW * BW; w < wave; ++w)
#pragma unroll
                    for (int c = 0; c < CH; ++c) begin[c] = fmaf(pairs[buf][w][cl][c], begin[c], pairs[buf][w][cl][CH + c]);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) begin[c] = fmaf(Pf[c], begin[c], Hf[c]);
            float before[K][CH];                                    // the state ahead of every token
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    before[k][c] = begin[c];
                    begin[c] = fmaf(a[k][c], begin[c], v[k][c]);
                }
            char *to_x = static_cast<char *>(p.dx) + at * p.dx_stride * Ln::ES, *to_f = static_cast<char *>(p.df) + at * p.df_stride * Ln::ES;
            char *to_i = static_cast<char *>(p.di) + at * p.di_stride * Ln::ES, *to_z = static_cast<char *>(p.dz) + at * p.dz_stride * Ln::ES;
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                if (t + k >= len) continue;
                float f[CH], x[CH], i[CH], z[CH], dy[CH], dx[CH], df[CH], di[CH], dz[CH];
                Ln::decode(rf[k], f);
                Ln::decode(rx[k], x);
                if (p.i) Ln::decode(ri[k], i);
                if (p.z) {
                    Ln::decode(rz[k], z);
                    Ln::decode(ry[k], dy);
                }
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const float Gt = g[k][c] + flow[c], at_k = a[k][c], w = v[k][c];
                    flow[c] = at_k * Gt;
                    if (p.z) {
                        const float s = sigmoid(z[c]), h = fmaf(at_k, before[k][c], w);
                        dz[c] = dy[c] * h * s * fmaf(z[c], 1.f - s, 1.f);
                    }
                    float si = 1.f, ni = 0.f;
                    if (p.i) sigmoids(i[c] + ib[c], si, ni);
                    float r, nr, m;
                    sigmoids(f[c] + fb[c], r, nr);
                    if constexpr (LRU) {
                        const float q = rate[c] * r, m2 = one_minus_square(q, at_k);
                        m = __builtin_amdgcn_sqrtf(m2);
                        const float s = -kLn2 * q;
                        const float E = (s * at_k) * Gt * fmaf(w * at_k, __builtin_amdgcn_rcpf(fmaxf(m2, 1e-37f)), -before[k][c]);
                        sumA[c] += E;
                        df[c] = E * nr;
                    } else {
                        m = nr;
                        df[c] = Gt * (r * nr) * (before[k][c] - si * x[c]);
                    }
                    sumF[c] += df[c];
                    dx[c] = Gt * m * si;
                    if (p.i) {
                        di[c] = Gt * w * ni;
                        sumI[c] += di[c];
                    }
                }
                if (p.dx) Ln::store(to_x + k * p.dx_stride * Ln::ES, odx, live, dx);
                if (p.df) Ln::store(to_f + k * p.df_stride * Ln::ES, odf, live, df);
                if (p.di) Ln::store(to_i + k * p.di_stride * Ln::ES, odi, live, di);
                if (p.dz) Ln::store(to_z + k * p.dz_stride * Ln::ES, odz, live, dz);
            }
        }
    }
    if constexpr (!OUT) {
        if (wave != 0 || grp != 0) return;
        store_channels<CH>(p.seg_r + seg0 + (size_t)seg * p.C, live, carry);
        store_channels<CH>(p.seg_p + seg0 + (size_t)seg * p.C, live, prod);
    } else {
        if (seg == 0 && p.dh_in && wave == 0 && grp == 0) store_channels<CH>(p.dh_in + (size_t)b * p.C + c0, live, carry);
        if (!p.partial) return;
        __syncthreads();                                            // the last tile's pairs have been read
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int d = CL; d < 64; d *= 2) {
                sumA[c] += __shfl_xor(sumA[c], d);
                sumF[c] += __shfl_xor(sumF[c], d);
                sumI[c] += __shfl_xor(sumI[c], d);
            }
        }
        if (grp == 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs[0][wave][cl][c] = sumA[c];
                pairs[0][wave][cl][CH + c] = sumF[c];
                pairs[0][wave][cl][2 * CH + c] = sumI[c];
            }
        }
        __syncthreads();
        if (wave >= 3 || grp != 0) return;                          // wave k adds the k-th vector's
        float s[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            s[c] = 0.f;
            for (int w = 0; w < W; ++w) s[c] += pairs[0][w][cl][wave * CH + c];
        }
        store_channels<CH>(p.partial + (((size_t)b * p.seg_count + seg) * 3 + wave) * p.C + c0, live, s);
    }
}

template <int IO, int CL, bool LRU>
int launch(const GatedGradParams &p, hipStream_t stream)
{
    constexpr int CW = GatedLane<IO, CL>::CW;
    const unsigned groups = (unsigned)((p.C + CW - 1) / CW);
    const dim3 block(64 * kGatedWaves);
    if (p.seg_count > 1) {
        hipLaunchKernelGGL((gated_backward_kernel<IO, CL, LRU, false>), dim3(groups, p.seg_count - 1, p.batch), block, 0, stream, p);
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL((gated_backward_kernel<IO, CL, LRU, true>), dim3(groups, p.seg_count, p.batch), block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, bool LRU>
int launch_lanes(const GatedGradParams &p, hipStream_t stream)
{
    switch (p.lanes) {
        case 64: return launch<IO, 64, LRU>(p, stream);
        case 32: return launch<IO, 32, LRU>(p, stream);
        case 16: return launch<IO, 16, LRU>(p, stream);
        case 8: return launch<IO, 8, LRU>(p, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_gated_backward(const GatedGradParams &p, hipStream_t stream)
{
    int e;
    if (p.io == SSMV_BF16) e = p.lru ? launch_lanes<SSMV_BF16, true>(p, stream) : launch_lanes<SSMV_BF16, false>(p, stream);
    else e = p.lru ? launch_lanes<SSMV_F32, true>(p, stream) : launch_lanes<SSMV_F32, false>(p, stream);
    if (e != 0 || !p.partial) return e;
    const ColumnSums to{{p.dA, p.df_bias, p.di_bias}, {p.A, nullptr, nullptr}};
    return launch_column_sums(p.partial, p.batch * p.seg_count, p.C, to, stream);
}

}  // namespace ssmv
