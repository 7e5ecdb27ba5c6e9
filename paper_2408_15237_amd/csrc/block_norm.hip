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

// 8 adjacent channels of a row as stored.  The last ones of a row are a vector moved back, whose first `skip` channels are another thread's: they count as zeros here and
// are not stored.  Threads behind the row have skip 8.  A row of fewer than 8 channels is loaded by elements (SMALL).
template <int T>
struct Eight {
    uint4 w[T == SSMV_BF16 ? 1 : 2];
    template <bool SMALL>
    __device__ __forceinline__ void load(const void *base, size_t idx, int C)
    {
        constexpr int ES = T == SSMV_BF16 ? 2 : 4;
        if constexpr (!SMALL) {
            __builtin_memcpy(w, static_cast<const char *>(base) + idx * ES, sizeof(w));
        } else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < C ? load_io(base, idx + j, T) : 0.f;
            if constexpr (T == SSMV_BF16) w[0] = IoVec<T>::encode(v);
            else __builtin_memcpy(w, v, sizeof(w));
        }
    }
    __device__ __forceinline__ void get(float (&v)[8], int skip) const
    {
        if constexpr (T == SSMV_BF16) IoVec<T>::decode(w[0], v);
        else __builtin_memcpy(v, w, sizeof(w));
        if (skip != 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < skip ? 0.f : v[j];
        }
    }
};

template <int T, bool SMALL>
__device__ __forceinline__ void put(void *base, size_t idx, int skip, int C, const float (&v)[8])
{
    if (!SMALL && skip == 0) {
        store8<T>(base, idx, 8, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= skip && (!SMALL || j < C)) store_io(base, idx + j, v[j], T);
    }
}

template <bool SMALL>
__device__ __forceinline__ void weights(const float *from, int c0, int C, float (&w)[8])
{
    if constexpr (!SMALL) {
        __builtin_memcpy(w, from + c0, sizeof(w));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = j < C ? from[c0 + j] : 0.f;
    }
}

// where a thread's channels are
template <int NV, bool SMALL>
struct Place {
    int c0[NV], skip[NV];
    __device__ __forceinline__ Place(int t, int threads, int C)
    {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int own = (t + k * threads) * 8;
            c0[k] = SMALL ? 0 : min(own, C - 8);
            skip[k] = SMALL ? (own == 0 ? 0 : 8) : min(own - c0[k], 8);
        }
    }
};

// Bound by memory: x, z and res in, r and n out.  `waves` waves to a row, as many rows as the workgroup has room for; a thread owns NV times 8 adjacent
// channels of its row, which stay in registers between the passes.  Everything is requested before the first wait.  16384 x 4096 bf16, sum and norm alone, 537 MB, other tensors in
// every call: 92 to 95 us, 5.7 TB/s (a copy of 1 GiB 6.1); with gate, norm behind the block and scale 135.  Stores past the caches gave 2 %, and would leave the next product
// without them.
template <int IO, int RES, int NV, bool SMALL>
__global__ __launch_bounds__(1024) void block_norm_kernel(const BlockNormParams p, int waves)
{
    __shared__ float part[2][1][kMaxWaves];
    const unsigned lane = threadIdx.x & 63u;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave / waves, first = sub * waves;
    const int per_wg = (int)(blockDim.x >> 6) / waves;
    const size_t row_raw = (size_t)blockIdx.x * per_wg + sub;
    const bool have = row_raw < (size_t)p.rows;
    const size_t row = have ? row_raw : p.rows - 1;                 // waves past the last row read it again and store nothing
    const Place<NV, SMALL> at((wave - first) * 64 + (int)lane, waves * 64, p.C);

    Eight<IO> xr[NV], zr[NV];
    Eight<RES> rr[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (p.x) xr[k].template load<SMALL>(p.x, row * p.x_stride + at.c0[k], p.C);
        if (p.z) zr[k].template load<SMALL>(p.z, row * p.z_stride + at.c0[k], p.C);
        if (p.res) rr[k].template load<SMALL>(p.res, row * p.res_stride + at.c0[k], p.C);
    }
    float w2[NV][8], cs[NV][8], w1[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (p.post) weights<SMALL>(p.post, at.c0[k], p.C, w2[k]);
        if (p.scale) weights<SMALL>(p.scale, at.c0[k], p.C, cs[k]);
        if (p.pre && p.n_out) weights<SMALL>(p.pre, at.c0[k], p.C, w1[k]);
    }
    float r[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (p.res) rr[k].get(r[k], at.skip[k]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) r[k][j] = 0.f;
        }
    }
    if (p.x) {
        float a[NV][8];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            xr[k].get(a[k], at.skip[k]);
            if (p.z) {
                float z[8];
                zr[k].get(z, at.skip[k]);
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
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = a[k][j];
                if (p.post) v = v * scale * w2[k][j];
                v *= p.alpha;
                if (p.scale) v *= cs[k][j];
                r[k][j] += v;
            }
            if (p.r_out && have) put<RES, SMALL>(p.r_out, row * p.r_stride + at.c0[k], at.skip[k], p.C, r[k]);
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
#pragma unroll
        for (int j = 0; j < 8; ++j) r[k][j] = p.pre ? r[k][j] * scale * w1[k][j] : r[k][j] * scale;
        if (have) put<IO, SMALL>(p.n_out, row * p.n_stride + at.c0[k], at.skip[k], p.C, r[k]);
    }
}

// With g = dn * pre_wgt, k = alpha ch_scale post_wgt and the row's scales rho (of r) and sigma (of a):
//   r = res + sigma k a,   D = dr + rho (g - r rho^2 mean(g r))                 = dres
//   da = sigma (D k - a sigma^2 mean(D k a)),   dx = da silu(z),  dz = da x silu'(z)
//   dpre = sum dn rho r;  with S = sum D sigma a:  dscale = alpha post_wgt S,  dpost = alpha ch_scale S                 (sums over the rows)
// a and r are formed again from the inputs, which have to be read anyway.  A workgroup walks over rows, the next one's values on their way while it works on this one's;
// k, pre_wgt and the two sums of a thread's channels stay in registers.  The sums go to `partial` at the end, where a second launch adds them in a fixed order.
// Bound by memory and the three sums of a row one after the other: 8192 x 5120 bf16 with an fp32 stream, 923 MB, 181 us with the second launch's 5 (a copy's rate: 151), 90 of them vector instructions by the counters.  Steps that it took: loads that
// wait for no branch 525 -> 261; one sum for dscale and dpost, k and pre_wgt in registers 261 -> 210; one workgroup of more than 8 waves a compute unit, not two in turn, 193; no question which row a wave has where a row takes the workgroup, 181.
// Above 6144 channels a thread has two vectors of every tensor.  Up to 8192 that fits (4096 x 8192: bf16 120 us, with an fp32 stream 157, fp32 270 with 60 bytes of scratch a lane); above, more than 8 waves leave a
// thread 128 registers and 396 to 588 bytes of scratch: 4096 x 16384 971, 1201 and 1888 us, 1.1 to 1.2 TB/s.
template <int IO, int RES, int NV, int MAXW, bool SMALL>
__global__ __launch_bounds__(64 * MAXW) void block_norm_backward_kernel(const BlockNormGradParams p, int waves)
{
    __shared__ float part[2][3][2][kMaxWaves];                      // of even and odd rows: one barrier lies between any two uses of the same
    const unsigned lane = threadIdx.x & 63u;
    constexpr bool ONE = NV == 2 || MAXW > 8;                       // rows of so many waves have a workgroup to themselves
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = ONE ? 0 : wave / waves, first = sub * waves;
    const int per_wg = ONE ? 1 : (int)(blockDim.x >> 6) / waves;
    const Place<NV, SMALL> at((wave - first) * 64 + (int)lane, waves * 64, p.C);
    const float inv = 1.f / (float)p.C;
    float sum_pre[NV][8], S[NV][8], kk[NV][8], w1[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum_pre[k][j] = S[k][j] = 0.f;
            kk[k][j] = p.alpha;
            w1[k][j] = 1.f;
        }
        if (p.pre) weights<SMALL>(p.pre, at.c0[k], p.C, w1[k]);
        float w[8];
        if (p.scale) {
            weights<SMALL>(p.scale, at.c0[k], p.C, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) kk[k][j] *= w[j];
        }
        if (p.post) {
            weights<SMALL>(p.post, at.c0[k], p.C, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) kk[k][j] *= w[j];
        }
    }
    struct Row {
        Eight<IO> x[NV], z[NV], dn[NV];
        Eight<RES> res[NV], dr[NV];
    } next{};
    auto fetch = [&](Row &f, size_t row) {                          // of a row that is there: past the last one nothing is read (where dx is dn or dres dr, that may be stored by now) ...
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (p.x) f.x[k].template load<SMALL>(p.x, row * p.x_stride + at.c0[k], p.C);
            if (p.z) f.z[k].template load<SMALL>(p.z, row * p.z_stride + at.c0[k], p.C);
            if (p.res) f.res[k].template load<SMALL>(p.res, row * p.res_stride + at.c0[k], p.C);
            if (p.dn) f.dn[k].template load<SMALL>(p.dn, row * p.dn_stride + at.c0[k], p.C);
            if (p.dr) f.dr[k].template load<SMALL>(p.dr, row * p.dr_stride + at.c0[k], p.C);
        }
    };
    const int step = (int)gridDim.x * per_wg;
    if ((int)blockIdx.x * per_wg + sub < p.rows) fetch(next, (int)blockIdx.x * per_wg + sub);
    for (int base = (int)blockIdx.x * per_wg, odd = 0; base < p.rows; base += step, odd ^= 1) {    // the same count for all waves of the workgroup
        const bool have = ONE || base + sub < p.rows;               // ... and nothing of it is added: 0 times what is no number would be none
        const size_t row = base + sub;
        const Row cur = next;
        if (base + step + sub < p.rows) fetch(next, base + step + sub);
        float a[NV][8], r[NV][8], d[NV][8];
        float sigma = 1.f;
        if (p.x) {
            float ss[1] = {0.f};
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                cur.x[k].get(a[k], at.skip[k]);
                if (p.z) {
                    float z[8];
                    cur.z[k].get(z, at.skip[k]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) a[k][j] *= z[j] * sigmoid(z[j]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[0] = fmaf(a[k][j], a[k][j], ss[0]);
            }
            if (p.post) {
                row_sums<1>(ss, part[odd][0], first, waves, wave, lane);
                sigma = rsqrtf(ss[0] * inv + p.eps);
            }
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (p.res) cur.res[k].get(r[k], at.skip[k]);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) r[k][j] = 0.f;
            }
            if (p.x)
#pragma unroll
                for (int j = 0; j < 8; ++j) r[k][j] = fmaf(a[k][j], sigma * kk[k][j], r[k][j]);
            if (p.dr) cur.dr[k].get(d[k], at.skip[k]);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[k][j] = 0.f;
            }
        }
        if (p.dn) {
            float rs[2] = {0.f, 0.f};                              // sum r^2, sum g r
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float dn[8];
                cur.dn[k].get(dn, at.skip[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    rs[0] = fmaf(r[k][j], r[k][j], rs[0]);
                    rs[1] = fmaf(dn[j] * w1[k][j], r[k][j], rs[1]);
                }
            }
            row_sums<2>(rs, part[odd][1], first, waves, wave, lane);
            const float rho = rsqrtf(rs[0] * inv + p.eps), back = rho * rho * (rs[1] * inv);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float dn[8];
                cur.dn[k].get(dn, at.skip[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[k][j] = fmaf(rho, fmaf(-r[k][j], back, dn[j] * w1[k][j]), d[k][j]);
                    if (have) sum_pre[k][j] = fmaf(dn[j], rho * r[k][j], sum_pre[k][j]);      // rho r is near 1, where dn rho may overflow
                }
            }
        }
        if (p.dres && have)
#pragma unroll
            for (int k = 0; k < NV; ++k) put<RES, SMALL>(p.dres, row * p.dres_stride + at.c0[k], at.skip[k], p.C, d[k]);
        if (!p.x) continue;
        float gs[1] = {0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (have) S[k][j] = fmaf(d[k][j], sigma * a[k][j], S[k][j]);
                d[k][j] *= kk[k][j];
                gs[0] = fmaf(d[k][j], a[k][j], gs[0]);
            }
        if (p.post) {
            row_sums<1>(gs, part[odd][2], first, waves, wave, lane);
            const float back = sigma * sigma * (gs[0] * inv);
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) d[k][j] = sigma * fmaf(-a[k][j], back, d[k][j]);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (p.z) {
                float x[8], z[8], dz[8];
                cur.x[k].get(x, at.skip[k]);
                cur.z[k].get(z, at.skip[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float sg = sigmoid(z[j]), s = z[j] * sg;
                    dz[j] = d[k][j] * x[j] * fmaf(s, 1.f - sg, sg);
                    d[k][j] *= s;
                }
                if (p.dz && have) put<IO, SMALL>(p.dz, row * p.dz_stride + at.c0[k], at.skip[k], p.C, dz);
            }
            if (p.dx && have) put<IO, SMALL>(p.dx, row * p.dx_stride + at.c0[k], at.skip[k], p.C, d[k]);
        }
    }
    if (!p.partial) return;
    if (per_wg > 1) {                                               // the rows of the workgroup, in order
        extern __shared__ __attribute__((aligned(16))) float sums[];     // [2][threads of a row][8 NV]
        const int t = (wave - first) * 64 + (int)lane, each = waves * 64 * 8 * NV;
        for (int s = 1; s < per_wg; ++s) {
            __syncthreads();
            if (sub == s) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        sums[(k * 8 + j) * waves * 64 + t] = sum_pre[k][j];
                        sums[each + (k * 8 + j) * waves * 64 + t] = S[k][j];
                    }
            }
            __syncthreads();
            if (sub == 0) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        sum_pre[k][j] += sums[(k * 8 + j) * waves * 64 + t];
                        S[k][j] += sums[each + (k * 8 + j) * waves * 64 + t];
                    }
            }
        }
        if (sub != 0) return;
    }
    float *to = p.partial + (size_t)blockIdx.x * 3 * p.C;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        put<SSMV_F32, SMALL>(to, at.c0[k], at.skip[k], p.C, sum_pre[k]);
        float w[8], v[8];
        if (p.scale) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 1.f;
            if (p.post) weights<SMALL>(p.post, at.c0[k], p.C, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p.alpha * w[j] * S[k][j];
            put<SSMV_F32, SMALL>(to, (size_t)p.C + at.c0[k], at.skip[k], p.C, v);
        }
        if (p.post) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 1.f;
            if (p.scale) weights<SMALL>(p.scale, at.c0[k], p.C, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p.alpha * w[j] * S[k][j];
            put<SSMV_F32, SMALL>(to, (size_t)2 * p.C + at.c0[k], at.skip[k], p.C, v);
        }
    }
}

// 32 columns side by side, 32 strands of the parts; the strands are added in order
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *partial, int parts, int C, ColumnSums to)
{
    __shared__ float acc[32][32];
    const int col = threadIdx.x & 31, w = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + col, k = blockIdx.y;
    if (!to.out[k]) return;
    float s = 0.f;
    if (c < C) {
        const float *from = partial + (size_t)k * C + c;
        const size_t row = (size_t)gridDim.y * C;
#pragma unroll 4
        for (int r = w; r < parts; r += 32) s += from[r * row];
    }
    acc[w][col] = s;
    __syncthreads();
    if (w != 0 || c >= C) return;
    for (int j = 1; j < 32; ++j) s += acc[j][col];
    if (to.over[k]) s = to.over[k][c] == 0.f ? 0.f : s / to.over[k][c];
    to.out[k][c] = s;
}

// Waves of a row, vectors of 8 channels a thread - one, or two where `most_waves` are too few for that -, and rows of a workgroup of about `waves_wg` waves.
struct RowShape {
    int nv, waves, per_wg;
};
RowShape row_shape(int C, int most_waves, int waves_wg)
{
    const int vectors = (C + 7) / 8;
    RowShape s;
    s.nv = vectors > 64 * most_waves ? 2 : 1;
    s.waves = (vectors + 64 * s.nv - 1) / (64 * s.nv);
    s.per_wg = s.waves >= waves_wg ? 1 : waves_wg / s.waves;
    return s;
}

template <int IO, int RES>
int launch_forward(const BlockNormParams &p, hipStream_t stream)
{
    const RowShape s = row_shape(p.C, kMaxWaves, 4);
    const dim3 grid((unsigned)((p.rows + s.per_wg - 1) / s.per_wg)), block(64 * s.waves * s.per_wg);
    if (p.C < 8) hipLaunchKernelGGL((block_norm_kernel<IO, RES, 1, true>), grid, block, 0, stream, p, s.waves);
    else if (s.nv == 1) hipLaunchKernelGGL((block_norm_kernel<IO, RES, 1, false>), grid, block, 0, stream, p, s.waves);
    else hipLaunchKernelGGL((block_norm_kernel<IO, RES, 2, false>), grid, block, 0, stream, p, s.waves);
    return (int)hipGetLastError();
}

template <int IO, int RES>
int launch_backward(const BlockNormGradParams &q, hipStream_t stream)
{
    BlockNormGradParams p = q;
    const RowShape s = row_shape(p.C, 12, 8);                       // one vector a thread in up to 12 waves: more leave a thread 128 registers, too few for the loop
    int wgs = (p.rows + s.per_wg - 1) / s.per_wg;
    const int most = s.nv == 1 && s.waves <= 8 ? kNormParts : kNormParts / 2;     // two workgroups of 8 waves run on a compute unit, one of more
    if (wgs > most) wgs = most;
    const dim3 grid((unsigned)wgs), block(64 * s.waves * s.per_wg);
    const size_t lds = s.per_wg > 1 && p.partial ? (size_t)2 * s.waves * 64 * 8 * sizeof(float) : 0;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, lds, stream, p, s.waves); };
    if (p.C < 8) go(block_norm_backward_kernel<IO, RES, 1, 8, true>);
    else if (s.nv == 1 && s.waves <= 8) go(block_norm_backward_kernel<IO, RES, 1, 8, false>);
    else if (s.nv == 1) go(block_norm_backward_kernel<IO, RES, 1, 12, false>);
    else if (s.waves <= 8) go(block_norm_backward_kernel<IO, RES, 2, 8, false>);
    else go(block_norm_backward_kernel<IO, RES, 2, 16, false>);
    const int e = (int)hipGetLastError();
    if (e != 0 || !p.partial) return e;
    const ColumnSums to{{p.dpre, p.dscale, p.dpost}, {nullptr, nullptr, nullptr}};
    return launch_column_sums(p.partial, wgs, p.C, to, stream);
}

}  // namespace

int launch_column_sums(const float *partial, int parts, int C, const ColumnSums &to, hipStream_t stream)
{
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)((C + 31) / 32), 3), dim3(1024), 0, stream, partial, parts, C, to);
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
