// The gradients of the gated linear recurrence.
#include <type_traits>

#include "gated_common.h"

namespace ssmv {
namespace {

// h_t = a_t h_{t-1} + v_t,  y_t = h_t silu(z_t).  With g_t = dy_t silu(z_t) and c the gradient that flows into the state from the tokens behind (dh_out at the end):
//   G_t = g_t + c,   c <- a_t G_t          (dh_in at the front)
//   MIX, a = r, m = 1 - r, r = sigmoid(f), u = sigmoid(i) x:      df = G r (1 - r) (h_{t-1} - u)
//   LRU, a = e^-s, s = -A r, m = sqrt(1 - a^2), v = m u:
//     E = s dL/ds = G s a (v a / m^2 - h_{t-1}),   df = E (1 - r),   dA = sum E / A        (E falls with sqrt(s) as s goes to 0)
//   dx = G m sigmoid(i),   di = G v (1 - sigmoid(i)),   dz = dy h silu'(z)
// The tiles from the last to the first.  A lane's run is the pair (P, H) of the forward pass and, from its last token to its first, the pair (P, R): c <- P c + R, with the
// same product.  Runs and waves combine both in one exchange: forwards inside 64 tokens, from the state that the forward pass left ahead of them, backwards through the whole
// tile.  What the gradients take of the gates is formed on the first walk, so that nothing of a token is worked out twice.
// Registers decide: nine values of each of a lane's 8 elements live between the two walks.  The next tile's inputs wait in LDS instead, and `settle` keeps the compiler from holding a value's operands
// until it is used: 241 -> 128 registers, two workgroups a compute unit.  8 x 2048 x 5120 bf16 with both gates, 1.51 GB, 382 us, 4.0 TB/s, of which the same walk without arithmetic takes
// 345 (see gated_recurrence.hip); it was 1070 with runs of 8 tokens in registers and 431 with 64-byte pieces.  One workgroup alone takes 4.3 us a tile, 60 % of it vector instructions; of the 382 us they
// are 189 by the counters.
// OUT false: only the pairs (P, R) of whole segments, of all but the first.
template <int IO, int CL, int W, bool LRU, bool HASI, bool HASZ, bool OUT>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(CL == 32 ? 4 : 2))) void gated_backward_kernel(const GatedGradParams p)
{
    using Ln = GatedLane<IO, CL>;
    constexpr int CH = Ln::CH, T = W * Ln::WT, K = kRun;
    constexpr int BW = SSMV_GATED_TILE / Ln::WT;                    // waves that share a state of the forward pass
    static_assert(W % BW == 0, "tiles are whole blocks of 64 tokens");
    __shared__ __attribute__((aligned(16))) float pairs[2][W][CL][3 * CH];
    // the next tile's values, on their way, and the states ahead of its blocks of 64 tokens: each wave's own
    constexpr int TENSORS = OUT ? 3 + HASI + HASZ : 2 + HASZ, WORDS = TENSORS * K + (OUT ? CH : 0);
    __shared__ __attribute__((aligned(16))) uint32_t ahead[WORDS][W][64];
    const unsigned lane = threadIdx.x & 63u, cl = lane % CL;
    unsigned run = lane / CL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (int)xcd_contiguous(blockIdx.x, gridDim.x) * Ln::CW, seg = OUT ? blockIdx.y : blockIdx.y + 1;
    Ln ln(first + (int)cl * CH, p.C);
    int b = blockIdx.z;
    if (p.seq_len && p.batch > 1 && p.batch <= 64) b = __builtin_amdgcn_readfirstlane(zth_longest(p.seq_len, p.batch, b, lane));
    const int all = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    const int from = seg * p.seg_len, len = min(all, from + p.seg_len);
    const bool have = seg == 0 || from < all;                       // segments behind the sequence's end: nothing but zeros in the sums
    const size_t seg0 = (size_t)b * p.seg_count * p.C;
    if (!OUT && !have) return;

    float carry[CH], prod[CH], rate[CH], fb[CH], ib[CH], sumA[CH], sumF[CH], sumI[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        carry[c] = sumA[c] = sumF[c] = sumI[c] = rate[c] = fb[c] = ib[c] = 0.f;
        prod[c] = 1.f;
    }
    if (LRU) ln.floats(p.A, rate);
    if (p.f_bias) ln.floats(p.f_bias, fb);
    if (HASI && p.i_bias) ln.floats(p.i_bias, ib);
    if (have && (OUT || len == all)) {
        if (p.dh_out) ln.floats(p.dh_out + (size_t)b * p.C, carry);
        if (OUT)
            for (int j = (all + p.seg_len - 1) / p.seg_len - 1; j > seg; --j) {      // the last segment's R has dh_out in it
                float sp[CH], sr[CH];
                ln.floats(p.seg_p + seg0 + (size_t)j * p.C, sp);
                ln.floats(p.seg_r + seg0 + (size_t)j * p.C, sr);
                const bool end = (j + 1) * (size_t)p.seg_len >= (size_t)all;
#pragma unroll
                for (int c = 0; c < CH; ++c) carry[c] = end ? sr[c] : fmaf(sp[c], carry[c], sr[c]);
            }
    }

    const size_t blocks = (p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE;
    const int wave0 = wave * Ln::WT, run0 = wave0 + (int)run * K;
    // the last tile, where it is not whole (all of them of a row of one bf16 channel), then whole ones
    const int n = have ? len - from : 0, whole = p.C >= CH ? n - n % T : 0;
    int t0 = from + (n + T - 1) / T * T - T;
    const size_t tok0 = (size_t)b * p.L + wave0 + t0;               // of a tile that is there, but where there is none
    Walk<IO, CL> wx(p.x, p.x_stride, tok0, run, ln), wf(p.f, p.f_stride, tok0, run, ln), wi(p.i, p.i_stride, tok0, run, ln), wz(p.z, p.z_stride, tok0, run, ln),
        wy(p.dy, p.dy_stride, tok0, run, ln);
    Walk<IO, CL> wdx(p.dx, p.dx_stride, tok0, run, ln), wdf(p.df, p.df_stride, tok0, run, ln), wdi(p.di, p.di_stride, tok0, run, ln), wdz(p.dz, p.dz_stride, tok0, run, ln);
    uint32_t rx[K], rf[K], ri[K], rz[K], ry[K];
    float block[CH];                                                // the state ahead of the lane's block of 64 tokens
    auto each = [&](auto &&fn) {                                    // the tensors of a tile
        fn(wf, rf, 0);
        fn(wy, ry, 1);
        if (HASZ) fn(wz, rz, 2);
        if (OUT) fn(wx, rx, 2 + HASZ);
        if (OUT && HASI) fn(wi, ri, 3 + HASZ);
    };
    auto block_of = [&](int t0) { return p.states + ((size_t)b * blocks + (t0 + wave0) / SSMV_GATED_TILE) * p.C; };
    auto fetch_tail = [&](int t0) {
        if (OUT) ln.floats(block_of(min(t0, len - 1 - wave0)), block);       // of a block that has no token the last block's, which nothing comes of
        each([&](auto &w, uint32_t (&r)[K], int) {
            w.load_tail(r, t0 + wave0, run, len, ln);
            w.move(-T);
#pragma unroll
            for (int k = 0; k < K; ++k) asm volatile("" : "+v"(r[k]));
        });
    };
    const unsigned state_off = (unsigned)ln.c0 * 4;
    auto prefetch = [&](int t0) {
        each([&](auto &w, uint32_t (&)[K], int i) {
            w.prefetch(&ahead[i * K][wave][0], W * 64);
            w.move(-T);
        });
        if (OUT) {
            const char *row = reinterpret_cast<const char *>(block_of(t0));
#pragma unroll
            for (int c = 0; c < CH; ++c) load_to_lds(row + 4 * c, state_off, &ahead[TENSORS * K + c][wave][0]);
        }
    };
    auto tile = [&](auto tail, int t0, int buf) {
        constexpr bool TAIL = decltype(tail)::value;
        const int t = t0 + run0;
        float a[K][CH], g[K][CH], v[OUT ? K : 1][CH], zz[OUT ? K : 1][CH];
        float e0[OUT ? K : 1][CH], e1[OUT ? K : 1][CH], e2[OUT ? K : 1][CH], ex[OUT ? K : 1][CH], ei[OUT ? K : 1][CH], begin[CH];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float f[CH], x[CH], i[CH], z[CH], dy[CH];
            Ln::decode(rf[k], f);
            Ln::decode(ry[k], dy);
            if (OUT) Ln::decode(rx[k], x);
            if (OUT && HASI) Ln::decode(ri[k], i);
            if (HASZ) Ln::decode(rz[k], z);
            constexpr int O = OUT ? 1 : 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float r, nr, q = 0.f, m = 0.f, m2 = 0.f;
                const float fe = fmaf(f[c], -kLog2e, fb[c]);
                if (LRU) sigmoid_pair(__builtin_amdgcn_exp2f(fe), r, nr);
                else sigmoids_log2(fe, r, nr);
                a[k][c] = r;
                if (LRU) {
                    q = rate[c] * r;
                    a[k][c] = __builtin_amdgcn_exp2f(q);
                }
                g[k][c] = dy[c];
                if (HASZ) {
                    const float sg = sigmoid(z[c]), s = z[c] * sg;
                    g[k][c] = dy[c] * s;
                    if (OUT) zz[O * k][c] = dy[c] * fmaf(s, 1.f - sg, sg);
                }
                if (OUT) {
                    float si = 1.f, ni = 0.f;
                    if (HASI) sigmoid_pair(__builtin_amdgcn_exp2f(fmaf(i[c], -kLog2e, ib[c])), si, ni);
                    const float u = HASI ? x[c] * si : x[c];
                    if (LRU) {
                        m2 = one_minus_square(q, a[k][c]);
                        m = __builtin_amdgcn_sqrtf(m2);
                    } else {
                        m = nr;
                    }
                    const float w = m * u;
                    v[O * k][c] = w;
                    ex[O * k][c] = HASI ? m * si : m;
                    if (HASI) ei[O * k][c] = w * ni;
                    if (LRU) {                                      // E = G e0 (e1 - h)
                        e0[O * k][c] = (-kLn2 * q) * a[k][c];
                        e1[O * k][c] = w * a[k][c] * __builtin_amdgcn_rcpf(fmaxf(m2, 1e-37f));
                        e2[O * k][c] = nr;
                    } else {                                        // df = G e0 (h - e1)
                        e0[O * k][c] = r * nr;
                        e1[O * k][c] = u;
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                constexpr int O = OUT ? 1 : 0;
                settle(a[k][c]);
                settle(g[k][c]);
                if (OUT) {
                    settle(v[O * k][c]);
                    settle(e0[O * k][c]);
                    settle(e1[O * k][c]);
                    if (LRU) settle(e2[O * k][c]);
                    settle(ex[O * k][c]);
                    if (HASI) settle(ei[O * k][c]);
                    if (HASZ) settle(zz[O * k][c]);
                }
            }
#pragma unroll
        for (int c = 0; c < CH; ++c) begin[c] = block[c];
        if (TAIL) {                                                 // tokens that are none: nothing flows into them, and through them as it is
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const bool is = t + k < len;
                    a[k][c] = is ? a[k][c] : 1.f;
                    g[k][c] = is ? g[k][c] : 0.f;
                    if (OUT) v[OUT ? k : 0][c] = is ? v[OUT ? k : 0][c] : 0.f;
                }
        }
        float Pf[CH], Hf[CH], Pr[CH], Rr[CH], Pt[CH], Ht[CH], Rt[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float P = a[0][c], H = OUT ? v[0][c] : 0.f, R = a[K - 1][c] * g[K - 1][c];
#pragma unroll
            for (int k = 1; k < K; ++k) {
                P *= a[k][c];
                if (OUT) H = fmaf(a[k][c], H, v[OUT ? k : 0][c]);
                R = a[K - 1 - k][c] * (g[K - 1 - k][c] + R);
            }
            combine_forward<CL>(P, H, run, Pf[c], Hf[c], Pt[c], Ht[c]);
            combine_backward<CL>(P, R, run, Pr[c], Rr[c], Rt[c]);
        }
        if (run == 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs[buf][wave][cl][c] = Pt[c];
                pairs[buf][wave][cl][CH + c] = Rt[c];
                pairs[buf][wave][cl][2 * CH + c] = Ht[c];
            }
        }
        __syncthreads();
        float flow[CH];                                             // into the lane's last token
#pragma unroll
        for (int w = W - 1; w >= 0; --w) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                flow[c] = w == wave ? carry[c] : w == W - 1 ? 0.f : flow[c];
                const float pw = pairs[buf][w][cl][c];
                carry[c] = fmaf(pw, carry[c], pairs[buf][w][cl][CH + c]);
                if (!OUT) prod[c] *= pw;
                settle(carry[c]);
                settle(flow[c]);
            }
        }
        if constexpr (OUT) {
            for (int w = wave / BW * BW; w < wave; ++w)
#pragma unroll
                for (int c = 0; c < CH; ++c) begin[c] = fmaf(pairs[buf][w][cl][c], begin[c], pairs[buf][w][cl][2 * CH + c]);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                flow[c] = fmaf(Pr[c], flow[c], Rr[c]);
                begin[c] = fmaf(Pf[c], begin[c], Hf[c]);
            }
            // e1 becomes what E or df takes of the state ahead of the token, zz the gradient of z
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    e1[k][c] = LRU ? e1[k][c] - begin[c] : begin[c] - e1[k][c];
                    begin[c] = fmaf(a[k][c], begin[c], v[k][c]);
                    if (HASZ) zz[k][c] *= begin[c];
                }
            if (HASZ && p.dz) wdz.template store<TAIL>(zz, t0 + wave0, run, len, ln, false);
#pragma unroll
            for (int k = K - 1; k >= 0; --k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const float G = g[k][c] + flow[c];
                    const bool is = !TAIL || t + k < len;           // 0 times what is no number would be none
                    flow[c] = a[k][c] * G;
                    ex[k][c] *= G;
                    if (HASI) {
                        ei[k][c] *= G;
                        sumI[c] += is ? ei[k][c] : 0.f;
                    }
                    e0[k][c] *= G * e1[k][c];
                    if (LRU) {
                        sumA[c] += is ? e0[k][c] : 0.f;
                        e0[k][c] *= e2[k][c];
                    }
                    sumF[c] += is ? e0[k][c] : 0.f;
                }
            if (p.dx) wdx.template store<TAIL>(ex, t0 + wave0, run, len, ln, false);
            if (p.df) wdf.template store<TAIL>(e0, t0 + wave0, run, len, ln, false);
            if (HASI && p.di) wdi.template store<TAIL>(ei, t0 + wave0, run, len, ln, false);
            wdx.move(-T);
            wdf.move(-T);
            wdi.move(-T);
            wdz.move(-T);
        }
    };
#pragma unroll
    for (int c = 0; c < CH; ++c) {                                  // as exponents of 2
        if (LRU) rate[c] = decay_exponent(rate[c]);
        fb[c] *= -kLog2e;
        ib[c] *= -kLog2e;
    }
    const std::true_type tail{};
    const std::false_type full{};
    int buf = 0;
    for (; t0 >= from + whole; t0 -= T, buf ^= 1) {
        asm volatile("" : "+v"(ln.c0), "+v"(ln.skip), "+v"(run));   // what only this loop needs of them is worked out in it
        fetch_tail(t0);
        tile(tail, t0, buf);
    }
    if (whole > 0) {
        // Behind a tile's loads a wave has issued the stores of the tile before: how many is known where every lane of the workgroup stores and all gradients are wanted.
        const bool known = OUT && first + Ln::CW <= p.C && p.dx && p.df && (!HASI || p.di) && (!HASZ || p.dz);
        prefetch(t0);
        bool stored = false;
        for (; t0 >= from; t0 -= T, buf ^= 1) {
            if (known && stored) wait_but<K * (2 + HASI + HASZ)>();
            else wait_but<0>();
            stored = true;
            each([&](auto &, uint32_t (&r)[K], int i) {
#pragma unroll
                for (int k = 0; k < K; ++k) r[k] = ahead[i * K + k][wave][lane];
            });
            if (OUT)
#pragma unroll
                for (int c = 0; c < CH; ++c) block[c] = __uint_as_float(ahead[OUT ? TENSORS * K + c : 0][wave][lane]);
            if (t0 > from) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // what is there has been read
                prefetch(t0 - T);
            }
            tile(full, t0, buf);
        }
    }
    if constexpr (!OUT) {
        if (wave != 0 || run != 0) return;
        ln.put_floats(p.seg_r + seg0 + (size_t)seg * p.C, carry);
        ln.put_floats(p.seg_p + seg0 + (size_t)seg * p.C, prod);
    } else {
        if (seg == 0 && p.dh_in && wave == 0 && run == 0) ln.put_floats(p.dh_in + (size_t)b * p.C, carry);
        if (!p.partial) return;
        __syncthreads();                                            // the last tile's pairs have been read
        float sums[3][CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            sums[0][c] = sumA[c];
            sums[1][c] = sumF[c];
            sums[2][c] = sumI[c];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
#pragma unroll
                for (int d = CL; d < 64; d *= 2) sums[k][c] += __shfl_xor(sums[k][c], d);
                if (run == 0) pairs[0][wave][cl][k * CH + c] = sums[k][c];
            }
        }
        __syncthreads();
        if (wave >= 3 || run != 0) return;                          // wave k adds the k-th vector's
        float s[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            s[c] = 0.f;
            for (int w = 0; w < W; ++w) s[c] += pairs[0][w][cl][wave * CH + c];
        }
        ln.put_floats(p.partial + (((size_t)b * p.seg_count + seg) * 3 + wave) * p.C, s);
    }
}

template <int IO, int CL, int W, bool LRU, bool HASI, bool HASZ>
int launch(const GatedGradParams &p, hipStream_t stream)
{
    constexpr int CW = GatedLane<IO, CL>::CW;
    const unsigned groups = (unsigned)((p.C + CW - 1) / CW);
    const dim3 block(64 * W);
    if (p.seg_count > 1) {
        hipLaunchKernelGGL((gated_backward_kernel<IO, CL, W, LRU, false, HASZ, false>), dim3(groups, p.seg_count - 1, p.batch), block, 0, stream, p);
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL((gated_backward_kernel<IO, CL, W, LRU, HASI, HASZ, true>), dim3(groups, p.seg_count, p.batch), block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, int CL, int W, bool LRU>
int launch_gates(const GatedGradParams &p, hipStream_t stream)
{
    if (p.i) return p.z ? launch<IO, CL, W, LRU, true, true>(p, stream) : launch<IO, CL, W, LRU, true, false>(p, stream);
    return p.z ? launch<IO, CL, W, LRU, false, true>(p, stream) : launch<IO, CL, W, LRU, false, false>(p, stream);
}

template <int IO, bool LRU>
int launch_width(const GatedGradParams &p, hipStream_t stream)
{
    return p.wide ? launch_gates<IO, 32, 8, LRU>(p, stream) : launch_gates<IO, 16, 8, LRU>(p, stream);
}

}  // namespace

int launch_gated_backward(const GatedGradParams &p, hipStream_t stream)
{
    int e;
    if (p.io == SSMV_BF16) e = p.lru ? launch_width<SSMV_BF16, true>(p, stream) : launch_width<SSMV_BF16, false>(p, stream);
    else e = p.lru ? launch_width<SSMV_F32, true>(p, stream) : launch_width<SSMV_F32, false>(p, stream);
    if (e != 0 || !p.partial) return e;
    const ColumnSums to{{p.dA, p.df_bias, p.di_bias}, {p.A, nullptr, nullptr}};
    return launch_column_sums(p.partial, p.batch * p.seg_count, p.C, to, stream);
}

}  // namespace ssmv
