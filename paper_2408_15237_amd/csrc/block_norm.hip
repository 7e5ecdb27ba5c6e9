// What stands between two blocks of a residual network: gate, norm, residual scale and sum, and the norm ahead of the next block; forward and backward.
#include "layers_internal.h"

namespace ssmv {
namespace {

constexpr int kMaxWaves = 16;

// Sums of N values over the threads of a row: `waves` waves from wave `first` on.  All threads of the workgroup come here.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*part)[kMaxWaves], int first, int waves, int wave, unsigned lane)
{
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = sum_of_wave(v[j]);
    if (waves == 1) return;
    if (lane == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) part[j][wave] = v[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float s = 0.f;
        for (int w = 0; w < waves; ++w) s += part[j][first + w];
        v[j] = s;
    }
}

// Bound by memory: x, z and res in, r and n out.  `waves` waves to a row, as many rows as the workgroup has room for; a thread owns NV times 8 adjacent
// channels of its row, which stay in registers between the passes.
template <int IO, int RES, int NV>
__global__ __launch_bounds__(1024) void block_norm_kernel(const BlockNormParams p, int waves)
{
    __shared__ float part[2][1][kMaxWaves];
    const unsigned lane = threadIdx.x & 63u;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave / waves, first = sub * waves;
    const int per_wg = (int)(blockDim.x >> 6) / waves;
    const size_t row_raw = (size_t)blockIdx.x * per_wg + sub;
    const bool have = row_raw < (size_t)p.rows;
    const size_t row = have ? row_raw : p.rows - 1;                 // waves past the last row read it again and store nothing
    const int t = (wave - first) * 64 + (int)lane, threads = waves * 64;

    float a[NV][8], r[NV][8];
    int c0[NV], live[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        c0[k] = (t + k * threads) * 8;
        live[k] = min(max(p.C - c0[k], 0), 8);
        if (p.x) load8<IO>(p.x, row * p.x_stride + c0[k], live[k], a[k]);
        if (p.res) load8<RES>(p.res, row * p.res_stride + c0[k], live[k], r[k]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) r[k][j] = 0.f;
        }
    }
    if (p.x) {
        if (p.z) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float z[8];
                load8<IO>(p.z, row * p.z_stride + c0[k], live[k], z);
#pragma unroll
                for (int j = 0; j < 8; ++j) a[k][j] *= z[j] * sigmoid(z[j]);
            }
        }
        float scale = 1.f;
        if (p.post) {
            float ss[1] = {0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[0] = fmaf(a[k][j], a[k][j], ss[0]);
            row_sums<1>(ss, part[0], first, waves, wave, lane);
            scale = rsqrtf(ss[0] / (float)p.C + p.eps);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[8], c[8];
            if (p.post) load8<SSMV_F32>(p.post, c0[k], live[k], w);
            if (p.scale) load8<SSMV_F32>(p.scale, c0[k], live[k], c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = a[k][j];
                if (p.post) v = v * scale * w[j];
                v *= p.alpha;
                if (p.scale) v *= c[j];
                r[k][j] += v;
            }
            if (p.r_out && have) store8<RES>(p.r_out, row * p.r_stride + c0[k], live[k], r[k]);
        }
    }
    if (!p.n_out) return;
    float ss[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) ss[0] = fmaf(r[k][j], r[k][j], ss[0]);
    row_sums<1>(ss, part[1], first, waves, wave, lane);
    const float scale = rsqrtf(ss[0] / (float)p.C + p.eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float w[8];
        if (p.pre) load8<SSMV_F32>(p.pre, c0[k], live[k], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[k][j] = p.pre ? r[k][j] * scale * w[j] : r[k][j] * scale;
        if (have) store8<IO>(p.n_out, row * p.n_stride + c0[k], live[k], r[k]);
    }
}

// With g = dn * pre_wgt and the row's scales rho (of r) and sigma (of a):
//   D = dr + rho (g - r rho^2 mean(g r))            = dres
//   dp = D alpha ch_scale,  g2 = dp post_wgt,  da = sigma (g2 - a sigma^2 mean(g2 a))
//   dx = da silu(z),  dz = da x silu'(z);   dpre = sum dn r rho,  dscale = sum D alpha p,  dpost = sum dp a sigma over the rows.
// a, p and r are formed again from the inputs, which have to be read anyway.  A workgroup walks over rows; the sums of the vectors stay in registers, one set a
// thread, and go to `partial` at the end, where a second launch adds them in a fixed order.
template <int IO, int RES, int NV>
__global__ __launch_bounds__(1024) void block_norm_backward_kernel(const BlockNormGradParams p, int waves)
{
    __shared__ float part[2][3][2][kMaxWaves];                      // of even and odd rows: one barrier lies between any two uses of the same
    const unsigned lane = threadIdx.x & 63u;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave / waves, first = sub * waves;
    const int per_wg = (int)(blockDim.x >> 6) / waves;
    const int t = (wave - first) * 64 + (int)lane, threads = waves * 64;
    const float inv = 1.f / (float)p.C;
    int c0[NV], live[NV];
    float sum_pre[NV][8], sum_scale[NV][8], sum_post[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        c0[k] = (t + k * threads) * 8;
        live[k] = min(max(p.C - c0[k], 0), 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum_pre[k][j] = sum_scale[k][j] = sum_post[k][j] = 0.f;
    }
    const int step = (int)gridDim.x * per_wg;
    for (int base = (int)blockIdx.x * per_wg, odd = 0; base < p.rows; base += step, odd ^= 1) {    // the same count for all waves of the workgroup
        const bool have = base + sub < p.rows;
        const size_t row = have ? base + sub : p.rows - 1;
        float a[NV][8], r[NV][8], pv[NV][8];
        float ss[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (p.x) load8<IO>(p.x, row * p.x_stride + c0[k], live[k], a[k]);
            if (p.z) {
                float z[8];
                load8<IO>(p.z, row * p.z_stride + c0[k], live[k], z);
#pragma unroll
                for (int j = 0; j < 8; ++j) a[k][j] *= z[j] * sigmoid(z[j]);
            }
            if (p.post)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[0] = fmaf(a[k][j], a[k][j], ss[0]);
        }
        float sigma = 1.f;
        if (p.post) {
            row_sums<1>(ss, part[odd][0], first, waves, wave, lane);
            sigma = rsqrtf(ss[0] * inv + p.eps);
        }
        float rs[2] = {0.f, 0.f};                                  // sum r^2, sum g r
        float dn[NV][8], d[NV][8];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float w[8];
            if (p.res) load8<RES>(p.res, row * p.res_stride + c0[k], live[k], r[k]);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) r[k][j] = 0.f;
            }
            if (p.x) {
                float c[8];
                if (p.post) load8<SSMV_F32>(p.post, c0[k], live[k], w);
                if (p.scale) load8<SSMV_F32>(p.scale, c0[k], live[k], c);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    pv[k][j] = p.post ? a[k][j] * sigma * w[j] : a[k][j];
                    float v = pv[k][j] * p.alpha;
                    if (p.scale) v *= c[j];
                    r[k][j] += v;
                }
            }
            if (p.dn) {
                if (p.pre) load8<SSMV_F32>(p.pre, c0[k], live[k], w);
                load8<IO>(p.dn, row * p.dn_stride + c0[k], live[k], dn[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = p.pre ? dn[k][j] * w[j] : dn[k][j];
                    rs[0] = fmaf(r[k][j], r[k][j], rs[0]);
                    rs[1] = fmaf(g, r[k][j], rs[1]);
                }
            }
            if (p.dr) load8<RES>(p.dr, row * p.dr_stride + c0[k], live[k], d[k]);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[k][j] = 0.f;
            }
        }
        if (p.dn) {
            row_sums<2>(rs, part[odd][1], first, waves, wave, lane);
            const float rho = rsqrtf(rs[0] * inv + p.eps), back = rho * rho * (rs[1] * inv);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float w[8];
                if (p.pre) load8<SSMV_F32>(p.pre, c0[k], live[k], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = p.pre ? dn[k][j] * w[j] : dn[k][j];
                    d[k][j] = fmaf(rho, fmaf(-r[k][j], back, g), d[k][j]);
                    sum_pre[k][j] = fmaf(have ? dn[k][j] * rho : 0.f, r[k][j], sum_pre[k][j]);
                }
            }
        }
        if (p.dres && have)
#pragma unroll
            for (int k = 0; k < NV; ++k) store8<RES>(p.dres, row * p.dres_stride + c0[k], live[k], d[k]);
        if (p.x) {
            float gs[1] = {0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float c[8], w[8];
                if (p.scale) load8<SSMV_F32>(p.scale, c0[k], live[k], c);
                if (p.post) load8<SSMV_F32>(p.post, c0[k], live[k], w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float v = d[k][j] * p.alpha;
                    if (p.scale) {
                        sum_scale[k][j] = fmaf(have ? v : 0.f, pv[k][j], sum_scale[k][j]);
                        v *= c[j];
                    }
                    if (p.post) {
                        sum_post[k][j] = fmaf(have ? v * sigma : 0.f, a[k][j], sum_post[k][j]);
                        v *= w[j];
                        gs[0] = fmaf(v, a[k][j], gs[0]);
                    }
                    d[k][j] = v;
                }
            }
            if (p.post) {
                row_sums<1>(gs, part[odd][2], first, waves, wave, lane);
                const float back = sigma * sigma * (gs[0] * inv);
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[k][j] = sigma * fmaf(-a[k][j], back, d[k][j]);
            }
            if (p.z) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float x[8], z[8], dz[8];
                    load8<IO>(p.x, row * p.x_stride + c0[k], live[k], x);
                    load8<IO>(p.z, row * p.z_stride + c0[k], live[k], z);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float sg = sigmoid(z[j]);
                        dz[j] = d[k][j] * x[j] * sg * fmaf(z[j], 1.f - sg, 1.f);
                        d[k][j] *= z[j] * sg;
                    }
                    if (p.dz && have) store8<IO>(p.dz, row * p.dz_stride + c0[k], live[k], dz);
                }
            }
            if (p.dx && have)
#pragma unroll
                for (int k = 0; k < NV; ++k) store8<IO>(p.dx, row * p.dx_stride + c0[k], live[k], d[k]);
        }
    }
    if (!p.partial) return;
    float *to = p.partial + ((size_t)blockIdx.x * per_wg + sub) * 3 * p.C;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        store8<SSMV_F32>(to, c0[k], live[k], sum_pre[k]);
        store8<SSMV_F32>(to, (size_t)p.C + c0[k], live[k], sum_scale[k]);
        store8<SSMV_F32>(to, (size_t)2 * p.C + c0[k], live[k], sum_post[k]);
    }
}

// 64 columns side by side, 16 parts of the rows; the parts are added in order
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *partial, int parts, int C, ColumnSums to)
{
    __shared__ float acc[16][64];
    const int c = (int)blockIdx.x * 64 + (int)(threadIdx.x & 63), k = blockIdx.y, w = threadIdx.x >> 6;
    if (!to.out[k]) return;
    float s = 0.f;
    if (c < C)
        for (int r = w; r < parts; r += 16) s += partial[((size_t)r * gridDim.y + k) * C + c];
    acc[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (w != 0 || c >= C) return;
    for (int j = 1; j < 16; ++j) s += acc[j][threadIdx.x];
    if (to.over[k]) s = to.over[k][c] == 0.f ? 0.f : s / to.over[k][c];
    to.out[k][c] = s;
}

// waves of a row, and vectors of 8 channels a thread: one, or two where a workgroup has not the threads for that
struct RowShape {
    int nv, waves, per_wg;
};
RowShape row_shape(int C)
{
    const int vectors = (C + 7) / 8;
    RowShape s;
    s.nv = vectors > 64 * kMaxWaves ? 2 : 1;
    s.waves = (vectors + 64 * s.nv - 1) / (64 * s.nv);
    s.per_wg = s.waves >= 4 ? 1 : 4 / s.waves;
    return s;
}

template <int IO, int RES>
int launch_forward(const BlockNormParams &p, hipStream_t stream)
{
    const RowShape s = row_shape(p.C);
    const dim3 grid((unsigned)((p.rows + s.per_wg - 1) / s.per_wg)), block(64 * s.waves * s.per_wg);
    if (s.nv == 1) hipLaunchKernelGGL((block_norm_kernel<IO, RES, 1>), grid, block, 0, stream, p, s.waves);
    else hipLaunchKernelGGL((block_norm_kernel<IO, RES, 2>), grid, block, 0, stream, p, s.waves);
    return (int)hipGetLastError();
}

template <int IO, int RES>
int launch_backward(const BlockNormGradParams &q, hipStream_t stream)
{
    BlockNormGradParams p = q;
    const RowShape s = row_shape(p.C);
    // no more partial sums than the workspace has room for
    int wgs = (p.rows + s.per_wg - 1) / s.per_wg;
    const int most = norm_parts(p.rows) / s.per_wg > 0 ? norm_parts(p.rows) / s.per_wg : 1;
    if (wgs > most) wgs = most;
    const dim3 grid((unsigned)wgs), block(64 * s.waves * s.per_wg);
    if (s.nv == 1) hipLaunchKernelGGL((block_norm_backward_kernel<IO, RES, 1>), grid, block, 0, stream, p, s.waves);
    else hipLaunchKernelGGL((block_norm_backward_kernel<IO, RES, 2>), grid, block, 0, stream, p, s.waves);
    const int e = (int)hipGetLastError();
    if (e != 0 || !p.partial) return e;
    const ColumnSums to{{p.dpre, p.dscale, p.dpost}, {nullptr, nullptr, nullptr}};
    return launch_column_sums(p.partial, wgs * s.per_wg, p.C, to, stream);
}

}  // namespace

int launch_column_sums(const float *partial, int parts, int C, const ColumnSums &to, hipStream_t stream)
{
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((C + 63) / 64), 3), dim3(1024), 0, stream, partial, parts, C, to);
    return (int)hipGetLastError();
}

int launch_block_norm(const BlockNormParams &p, hipStream_t stream)
{
    if (p.io == SSMV_F32) return launch_forward<SSMV_F32, SSMV_F32>(p, stream);
    return p.res_io == SSMV_F32 ? launch_forward<SSMV_BF16, SSMV_F32>(p, stream) : launch_forward<SSMV_BF16, SSMV_BF16>(p, stream);
}

int launch_block_norm_backward(const BlockNormGradParams &p, hipStream_t stream)
{
    if (p.io == SSMV_F32) return launch_backward<SSMV_F32, SSMV_F32>(p, stream);
    return p.res_io == SSMV_F32 ? launch_backward<SSMV_BF16, SSMV_F32>(p, stream) : launch_backward<SSMV_BF16, SSMV_BF16>(p, stream);
}

}  // namespace ssmv
