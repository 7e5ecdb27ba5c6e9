// The gated linear recurrence over a sequence, from state to state, and over one token of every row.
#include <type_traits>

#include "gated_common.h"

namespace ssmv {
namespace {

// Decay and m of a token: see the header.  nfb = -f_bias log2 e.
template <bool LRU>
__device__ __forceinline__ void coefficients(float f, float nfb, float rate, float &a, float &m)
{
    if constexpr (LRU) {
        const float q = rate * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(fmaf(f, -kLog2e, nfb)));
        a = __builtin_amdgcn_exp2f(q);
        m = __builtin_amdgcn_sqrtf(one_minus_square(q, a));
    } else {
        sigmoids_log2(fmaf(f, -kLog2e, nfb), a, m);
    }
}

// h <- a h + v: a run of tokens is the pair (product of a, state that it leaves from zero), and pairs combine in order.  A lane forms the pair of its run of four, the runs of a
// wave (permutes) and then the waves of the workgroup combine theirs (LDS, one barrier a tile), and every lane goes through its run again from the state that it starts from.  So a
// token is read once; the gates stay in registers between the two walks, and the next tile's values are on their way.
// Many channels: bound by memory.  On a walk down the rows of 5 to 9 tensors, a few channels a workgroup, lines of 128 bytes reach 4.4 TB/s and pieces of 64 bytes 3.5, whatever a lane loads at
// once; 8 x 2048 x 5120 bf16 with both gates, 839 MB, 191 us, 4.4 TB/s (64-byte pieces 217).  Few: by vector instructions, 40 and 8 transcendental ones a value, of 4 and 16 cycles each:
// 1 x 2048 x 8192 50 us, where the bytes take 28.
// Loads into LDS (as the backward pass has them) were slower here, 197 -> 217 and 50 -> 62, and so was a branch in place of the choice of `start` for every w, 62 -> 64.
// OUT false: only the pairs of whole segments, of all but the last.
template <int IO, int CL, int W, bool LRU, bool HASI, bool HASZ, bool OUT>
__global__ __launch_bounds__(64 * W) void gated_recurrence_kernel(const GatedParams p)
{
    using Ln = GatedLane<IO, CL>;
    constexpr int CH = Ln::CH, T = W * Ln::WT, K = kRun;
    __shared__ __attribute__((aligned(16))) float pairs[2][W][CL][2 * CH];
    const unsigned lane = threadIdx.x & 63u, cl = lane % CL;
    unsigned run = lane / CL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = (int)xcd_contiguous(blockIdx.x, gridDim.x) * Ln::CW, seg = blockIdx.y;
    Ln ln(first + (int)cl * CH, p.C);
    int b = blockIdx.z;
    if (p.seq_len && p.batch > 1 && p.batch <= 64) b = __builtin_amdgcn_readfirstlane(zth_longest(p.seq_len, p.batch, b, lane));
    const int all = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    const int from = seg * p.seg_len, len = min(all, from + p.seg_len);
    const bool last = len == all;
    if (seg > 0 && (OUT ? from >= all : last)) return;
    const size_t seg0 = (size_t)b * p.seg_count * p.C;

    float h[CH], prod[CH], rate[CH], fb[CH], ib[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        h[c] = rate[c] = fb[c] = ib[c] = 0.f;
        prod[c] = 1.f;
    }
    if (LRU) ln.floats(p.A, rate);
    if (p.f_bias) ln.floats(p.f_bias, fb);
    if (HASI && p.i_bias) ln.floats(p.i_bias, ib);
    if (seg == 0) {
        const int src = p.src_row ? p.src_row[b] : b;
        if (OUT && p.seg_count > 1) ln.floats(p.seg_h + seg0 + (size_t)(p.seg_count - 1) * p.C, h);    // h_out may be h_in, and its writer another workgroup
        else if (p.h_in && (unsigned)src < (unsigned)p.rows_in) ln.floats(p.h_in + (size_t)src * p.C, h);
        if (!OUT && wave == 0 && run == 0) ln.put_floats(p.seg_h + seg0 + (size_t)(p.seg_count - 1) * p.C, h);
        if (!OUT && last) return;
    } else if (OUT) {
        ln.floats(p.seg_h + seg0, h);
        for (int j = 1; j < seg; ++j) {
            float sp[CH], sh[CH];
            ln.floats(p.seg_p + seg0 + (size_t)j * p.C, sp);
            ln.floats(p.seg_h + seg0 + (size_t)j * p.C, sh);
#pragma unroll
            for (int c = 0; c < CH; ++c) h[c] = fmaf(sp[c], h[c], sh[c]);
        }
    }

    const int wave0 = wave * Ln::WT, run0 = wave0 + (int)run * kRun;       // the wave's and the lane's tokens in a tile
    const size_t tok0 = (size_t)b * p.L + from + wave0;
    Walk<IO, CL> wx(p.x, p.x_stride, tok0, run, ln), wf(p.f, p.f_stride, tok0, run, ln), wi(p.i, p.i_stride, tok0, run, ln), wz(p.z, p.z_stride, tok0, run, ln),
        wy(p.y, p.y_stride, tok0, run, ln);
    const int whole = p.C >= CH ? len - from - (len - from) % T : 0;             // tokens in whole tiles; a row of one bf16 channel takes the other path, too
    uint32_t rx[kRun], rf[kRun], ri[kRun], rz[kRun];
    auto each = [&](auto &&fn) {                                    // the tensors of a tile
        fn(wf, rf, 0);
        fn(wx, rx, 1);
        if (HASI) fn(wi, ri, 2);
        if (OUT && HASZ) fn(wz, rz, 2 + HASI);
    };
    auto fetch = [&] {
        each([&](auto &w, uint32_t (&r)[K], int) {
            w.load(r);
            w.move(T);
        });
    };
    auto tile = [&](auto tail, int t0, int buf, auto &&next) {
        constexpr bool TAIL = decltype(tail)::value;
        const int t = t0 + run0;
        float a[K][CH], v[K][CH], y[OUT ? K : 1][CH], f[K][CH], i[HASI ? K : 1][CH];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Ln::decode(rf[k], f[k]);
            Ln::decode(rx[k], v[k]);
            if (HASI) Ln::decode(ri[k], i[HASI ? k : 0]);
            if (OUT && HASZ) Ln::decode(rz[k], y[OUT ? k : 0]);
        }
        next();
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float m;
                coefficients<LRU>(f[k][c], fb[c], rate[c], a[k][c], m);
                v[k][c] *= m;
                if (HASI) v[k][c] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(fmaf(i[HASI ? k : 0][c], -kLog2e, ib[c])));
                if (OUT && HASZ) y[OUT ? k : 0][c] *= sigmoid(y[OUT ? k : 0][c]);
                if (TAIL) {                                         // tokens that are none leave the state as it is
                    a[k][c] = t + k < len ? a[k][c] : 1.f;
                    v[k][c] = t + k < len ? v[k][c] : 0.f;
                }
            }
        float Pe[CH], He[CH], Pt[CH], Ht[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float P = a[0][c], H = v[0][c];
#pragma unroll
            for (int k = 1; k < kRun; ++k) {
                P *= a[k][c];
                H = fmaf(a[k][c], H, v[k][c]);
            }
            combine_forward<CL>(P, H, run, Pe[c], He[c], Pt[c], Ht[c]);
        }
        if (run == 0) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs[buf][wave][cl][c] = Pt[c];
                pairs[buf][wave][cl][CH + c] = Ht[c];
            }
        }
        __syncthreads();
        float start[CH];
#pragma unroll
        for (int w = 0; w < W; ++w) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                start[c] = w == wave ? h[c] : w == 0 ? 0.f : start[c];
                const float pw = pairs[buf][w][cl][c];
                h[c] = fmaf(pw, h[c], pairs[buf][w][cl][CH + c]);
                if (!OUT) prod[c] *= pw;
            }
        }
        if constexpr (OUT) {
#pragma unroll
            for (int c = 0; c < CH; ++c) start[c] = fmaf(Pe[c], start[c], He[c]);
            if (p.states && t % SSMV_GATED_TILE == 0 && t < len)
                ln.put_floats(p.states + ((size_t)b * ((p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE) + t / SSMV_GATED_TILE) * p.C, start);
#pragma unroll
            for (int k = 0; k < kRun; ++k)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    start[c] = fmaf(a[k][c], start[c], v[k][c]);
                    y[k][c] = HASZ ? start[c] * y[k][c] : start[c];
                }
            wy.template store<TAIL>(y, t0 + wave0, run, len, ln, p.past);
            wy.move(T);
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
    int t0 = from, buf = 0;
    const int full_end = from + whole;
    if (whole > 0) {
        fetch();
        for (; t0 < full_end; t0 += T, buf ^= 1)
            tile(full, t0, buf, [&] { if (t0 + T < full_end) fetch(); });
    }
    for (; t0 < len; t0 += T, buf ^= 1) {                           // once, but for a row of one bf16 channel
        asm volatile("" : "+v"(ln.c0), "+v"(ln.skip), "+v"(run));   // what only this loop needs of them is worked out in it
        each([&](auto &w, uint32_t (&r)[K], int) {
            w.load_tail(r, t0 + wave0, run, len, ln);
            w.move(T);
        });
        tile(tail, t0, buf, [] {});
    }
    if (wave != 0 || run != 0) return;
    if constexpr (OUT) {
        if (last && p.h_out) ln.put_floats(p.h_out + (size_t)b * p.C, h);
        if (all == 0 && p.states) ln.put_floats(p.states + (size_t)b * ((p.L + SSMV_GATED_TILE - 1) / SSMV_GATED_TILE) * p.C, h);
    } else {
        ln.put_floats(p.seg_h + seg0 + (size_t)seg * p.C, h);
        ln.put_floats(p.seg_p + seg0 + (size_t)seg * p.C, prod);
    }
}

// One token of every row: a lane per 4 bytes of it.
template <int IO, bool LRU>
__global__ __launch_bounds__(256) void gated_token_kernel(const GatedParams p)
{
    using Ln = GatedLane<IO, 16>;
    constexpr int CH = Ln::CH;
    const int b = blockIdx.y;
    const Ln ln(((int)blockIdx.x * 256 + (int)threadIdx.x) * CH, p.C);
    if (ln.skip >= CH || !ln.mine(CH - 1) && !ln.mine(0)) return;
    const bool none = p.seq_len && p.seq_len[b] <= 0;
    const int src = p.src_row ? p.src_row[b] : b;
    auto row = [&](const void *t, size_t stride) { return static_cast<const char *>(t) + (size_t)b * stride * Ln::ES; };
    float h[CH], x[CH], f[CH], i[CH], z[CH], rate[CH], fb[CH], ib[CH];
    uint32_t rx = 0, rf = 0, ri = 0, rz = 0;
    if (!none) {
        rx = ln.load_any(row(p.x, p.x_stride));
        rf = ln.load_any(row(p.f, p.f_stride));
        if (p.i) ri = ln.load_any(row(p.i, p.i_stride));
        if (p.z) rz = ln.load_any(row(p.z, p.z_stride));
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) h[c] = rate[c] = fb[c] = ib[c] = 0.f;
    if (p.h_in && (unsigned)src < (unsigned)p.rows_in) ln.floats(p.h_in + (size_t)src * p.C, h);
    if (LRU) ln.floats(p.A, rate);
    if (p.f_bias) ln.floats(p.f_bias, fb);
    if (p.i_bias) ln.floats(p.i_bias, ib);
    if (p.states) ln.put_floats(p.states + (size_t)b * p.C, h);
    Ln::decode(rx, x);
    Ln::decode(rf, f);
    Ln::decode(ri, i);
    Ln::decode(rz, z);
    float y[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float a, m;
        coefficients<LRU>(f[c], -kLog2e * fb[c], LRU ? decay_exponent(rate[c]) : 0.f, a, m);
        float v = m * x[c];
        if (p.i) v *= sigmoid(i[c] + ib[c]);
        if (!none) h[c] = fmaf(a, h[c], v);
        y[c] = p.z ? h[c] * (z[c] * sigmoid(z[c])) : h[c];
    }
    if (!none) ln.store_any(const_cast<char *>(row(p.y, p.y_stride)), y);
    if (p.h_out) ln.put_floats(p.h_out + (size_t)b * p.C, h);
}

template <int IO, int CL, int W, bool LRU, bool HASI, bool HASZ>
int launch(const GatedParams &p, hipStream_t stream)
{
    constexpr int CW = GatedLane<IO, CL>::CW;
    const unsigned groups = (unsigned)((p.C + CW - 1) / CW);
    const dim3 block(64 * W);
    if (p.seg_count > 1) {
        hipLaunchKernelGGL((gated_recurrence_kernel<IO, CL, W, LRU, HASI, false, false>), dim3(groups, p.seg_count - 1, p.batch), block, 0, stream, p);
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL((gated_recurrence_kernel<IO, CL, W, LRU, HASI, HASZ, true>), dim3(groups, p.seg_count, p.batch), block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, int CL, int W, bool LRU>
int launch_gates(const GatedParams &p, hipStream_t stream)
{
    if (p.i) return p.z ? launch<IO, CL, W, LRU, true, true>(p, stream) : launch<IO, CL, W, LRU, true, false>(p, stream);
    return p.z ? launch<IO, CL, W, LRU, false, true>(p, stream) : launch<IO, CL, W, LRU, false, false>(p, stream);
}

template <int IO, bool LRU>
int launch_width(const GatedParams &p, hipStream_t stream)
{
    if (p.L == 1) {
        constexpr int per = 256 * GatedLane<IO, 16>::CH;
        hipLaunchKernelGGL((gated_token_kernel<IO, LRU>), dim3((p.C + per - 1) / per, p.batch), dim3(256), 0, stream, p);
        return (int)hipGetLastError();
    }
    return p.wide ? launch_gates<IO, 32, 8, LRU>(p, stream) : launch_gates<IO, 16, 16, LRU>(p, stream);
}

}  // namespace

int launch_gated_recurrence(const GatedParams &q, hipStream_t stream)
{
    // Whatever comes next finds an output in the caches as long as they can hold it (8 x 2048 x 5120 bf16, 168 MB: 198 us through them, 192 past; 34 MB next to what reads it
    // is better left in them).
    GatedParams p = q;
    p.past = (size_t)p.batch * p.L * p.C * (p.io == SSMV_BF16 ? 2 : 4) > (128u << 20);
    if (p.io == SSMV_BF16) return p.lru ? launch_width<SSMV_BF16, true>(p, stream) : launch_width<SSMV_BF16, false>(p, stream);
    return p.lru ? launch_width<SSMV_F32, true>(p, stream) : launch_width<SSMV_F32, false>(p, stream);
}

}  // namespace ssmv
