// One token of every row through the recurrence, from state to state.
#include "decode_internal.h"

namespace ssmv {
namespace {

typedef float v4 __attribute__((ext_vector_type(4)));

// N/4 lanes share a state row, 16 bytes each, so that a wave's accesses are contiguous.  A workgroup takes 1024/N rows (channels) of
// U rows of the batch; all loads of a thread come before its first use of any.
template <int IO, int N, bool DIAG, int U>
__global__ __launch_bounds__(256) void selective_step_kernel(const TokenParams p)
{
    constexpr int LP = N / 4, ROWS = 256 / LP;
    constexpr float LOG2E = 1.4426950408889634f;
    const unsigned sub = threadIdx.x % LP;
    const unsigned r_raw = blockIdx.x * ROWS + threadIdx.x / LP, total = (unsigned)p.H * p.P;
    const bool have = r_raw < total;
    const unsigned r = have ? r_raw : total - 1;             // lanes past the end read the last row again and store nothing
    const unsigned hd = DIAG ? r : r / (unsigned)p.P;
    const unsigned grp = DIAG ? 0 : hd / (unsigned)(p.H / p.G);
    const unsigned b0 = blockIdx.y * U;

    v4 h[U];
    float x[U], dt[U], z[U], B[U][4], C[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned b = min(b0 + u, (unsigned)p.rows - 1);
        const int src = p.src_row ? p.src_row[b] : (int)b;
        h[u] = v4{0.f, 0.f, 0.f, 0.f};
        if (p.h_in && (unsigned)src < (unsigned)p.rows_in)
            h[u] = *reinterpret_cast<const v4 *>(p.h_in + ((size_t)src * total + r) * N + 4 * sub);
        x[u] = load_io(p.x, b * p.x_stride + r, IO);
        dt[u] = load_io(p.dt, b * p.dt_stride + hd, IO);
        z[u] = p.z ? load_io(p.z, b * p.z_stride + r, IO) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            B[u][i] = load_io(p.Bm, b * p.b_stride + (size_t)grp * N + 4 * sub + i, IO);
            C[u][i] = load_io(p.Cm, b * p.c_stride + (size_t)grp * N + 4 * sub + i, IO);
        }
    }
    const v4 a = DIAG ? *reinterpret_cast<const v4 *>(p.A + (size_t)r * N + 4 * sub) * LOG2E : v4{1.f, 1.f, 1.f, 1.f} * (p.A[hd] * LOG2E);
    const float D = p.D[hd], bias = p.dt_bias ? p.dt_bias[hd] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float d = p.softplus ? softplus_exact(dt[u] + bias) : dt[u];
        const float dx = d * x[u];
        float y = 0.f;
        if constexpr (DIAG) {
#pragma unroll
            for (int i = 0; i < 4; ++i) h[u][i] = fmaf(h[u][i], __builtin_amdgcn_exp2f(a[i] * d), dx * B[u][i]);
        } else {
            const float decay = __builtin_amdgcn_exp2f(a[0] * d);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[u][i] = fmaf(h[u][i], decay, dx * B[u][i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y = fmaf(h[u][i], C[u][i], y);
#pragma unroll
        for (int m = 1; m < LP; m *= 2) y += __shfl_xor(y, m);
        y = fmaf(D, x[u], y);
        if (p.z) y *= silu_fast(z[u]);
        if (have && b0 + u < (unsigned)p.rows) {
            const size_t b = b0 + u;
            *reinterpret_cast<v4 *>(p.h_out + (b * total + r) * N + 4 * sub) = h[u];
            if (sub == 0) store_io(p.y, b * p.y_stride + r, y, IO);
        }
    }
}

template <int IO, int N, bool DIAG>
int launch(const TokenParams &p, hipStream_t stream)
{
    constexpr unsigned ROWS = 1024 / N;
    const unsigned gx = ((unsigned)p.H * p.P + ROWS - 1) / ROWS;
    if (p.rows >= 65535 * 4) return (int)hipErrorInvalidValue;                             // refused by the host's checks
    if (p.rows >= 8) hipLaunchKernelGGL((selective_step_kernel<IO, N, DIAG, 4>), dim3(gx, (p.rows + 3) / 4), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((selective_step_kernel<IO, N, DIAG, 1>), dim3(gx, p.rows), dim3(256), 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, bool DIAG>
int launch_n(const TokenParams &p, hipStream_t stream)
{
    switch (p.N) {
        case 16: return launch<IO, 16, DIAG>(p, stream);
        case 32: return launch<IO, 32, DIAG>(p, stream);
        case 64: return launch<IO, 64, DIAG>(p, stream);
    }
    if constexpr (!DIAG) {
        if (p.N == 128) return launch<IO, 128, false>(p, stream);
        if (p.N == 256) return launch<IO, 256, false>(p, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_selective_step(const TokenParams &p, hipStream_t stream)
{
    if (p.io == SSMV_BF16) return p.diag ? launch_n<SSMV_BF16, true>(p, stream) : launch_n<SSMV_BF16, false>(p, stream);
    return p.diag ? launch_n<SSMV_F32, true>(p, stream) : launch_n<SSMV_F32, false>(p, stream);
}

}  // namespace ssmv
