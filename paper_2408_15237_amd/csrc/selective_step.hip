// One token of every row through the recurrence, from state to state.
#include "decode_internal.h"

namespace ssmv {
namespace {

typedef float v4 __attribute__((ext_vector_type(4)));

// four adjacent values of a row of B or C
template <int IO>
struct Four {
    uint32_t w[IO == SSMV_BF16 ? 2 : 4];
    __device__ __forceinline__ void load(const void *base, size_t idx)
    {
        __builtin_memcpy(w, static_cast<const char *>(base) + idx * (IO == SSMV_BF16 ? 2 : 4), sizeof(w));
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (IO == SSMV_BF16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};

template <int CTRL>
__device__ __forceinline__ float quad(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
// the value that lane i of a quad holds
__device__ __forceinline__ float quad_get(float v, int i) { return i == 0 ? quad<0x00>(v) : i == 1 ? quad<0x55>(v) : i == 2 ? quad<0xAA>(v) : quad<0xFF>(v); }

// N/4 lanes share a state row, 16 bytes each, so that a wave's accesses are contiguous; they are bound by memory, 8 bytes a state
// value.  States are loaded through the caches (several rows may continue from one) and stored past them (their next use is a token
// later, behind all other layers): 256 rows x 5120 x 16, new states in every call, 25.0 us; loads past the caches too 32.9, stores
// through them too 34.9, loads past and stores through them 32.1.  A workgroup takes 1024/N state rows (channels) of U rows of the batch, which share A and D.  With U = 4 lane u of every
// quad fetches and prepares the token of row u, hands it round the quad, and finishes that row's output.
template <int IO, int N, bool DIAG, int U>
__global__ __launch_bounds__(256) void selective_step_kernel(const TokenParams p)
{
    constexpr int LP = N / 4, ROWS = 256 / LP;
    const unsigned sub = threadIdx.x % LP, mine = U == 4 ? sub & 3u : 0u;
    const unsigned r_raw = blockIdx.x * ROWS + threadIdx.x / LP, total = (unsigned)p.H * p.P;
    const bool have = r_raw < total;
    const unsigned r = have ? r_raw : total - 1;             // lanes past the end read the last row again and store nothing
    const unsigned hd = DIAG ? r : r / (unsigned)p.P;
    const unsigned grp = DIAG ? 0 : hd / (unsigned)(p.H / p.G);
    const unsigned b0 = blockIdx.y * U, last = (unsigned)p.rows - 1;

    // everything is requested ahead of the first use of any of it
    v4 h[U];
    Four<IO> B[U], C[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned b = min(b0 + u, last);
        const int src = p.src_row ? p.src_row[b] : (int)b;
        h[u] = v4{0.f, 0.f, 0.f, 0.f};
        if (p.h_in && (unsigned)src < (unsigned)p.rows_in)
            h[u] = *(reinterpret_cast<const v4 *>(p.h_in + ((size_t)src * total + r) * N + 4 * sub));
    }
    const size_t bm = min(b0 + mine, last);
    const float x = load_io(p.x, bm * p.x_stride + r, IO);
    float dt = load_io(p.dt, bm * p.dt_stride + hd, IO);
    const float z = p.z ? load_io(p.z, bm * p.z_stride + r, IO) : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned b = min(b0 + u, last);
        B[u].load(p.Bm, b * p.b_stride + (size_t)grp * N + 4 * sub);
        C[u].load(p.Cm, b * p.c_stride + (size_t)grp * N + 4 * sub);
    }
    v4 a = DIAG ? *reinterpret_cast<const v4 *>(p.A + (size_t)r * N + 4 * sub) : v4{p.A[hd], 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < (DIAG ? 4 : 1); ++i) a[i] = decay_rate(a[i]);
    const float D = p.D[hd], bias = p.dt_bias ? p.dt_bias[hd] : 0.f;
    if (p.softplus) dt = softplus_exact(dt + bias);
    const float dx = dt * x, e = DIAG ? 0.f : __builtin_amdgcn_exp2f(a[0] * dt);
    float out = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float d = U == 4 ? quad_get(dt, u) : dt, dxu = U == 4 ? quad_get(dx, u) : dx, decay = U == 4 ? quad_get(e, u) : e;
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[u][i] = fmaf(h[u][i], DIAG ? __builtin_amdgcn_exp2f(a[i] * d) : decay, dxu * B[u].get(i));
            y = fmaf(h[u][i], C[u].get(i), y);
        }
        y += quad<0xB1>(y);
        y += quad<0x4E>(y);
#pragma unroll
        for (int m = 4; m < LP; m *= 2) y += __shfl_xor(y, m);
        out = U == 1 || mine == (unsigned)u ? y : out;
        if (have && b0 + u <= last)
            __builtin_nontemporal_store(h[u], reinterpret_cast<v4 *>(p.h_out + ((size_t)(b0 + u) * total + r) * N + 4 * sub));
    }
    out = fmaf(D, x, out);
    if (p.z) out *= silu_fast(z);
    if (have && sub < (unsigned)U && b0 + sub <= last) store_io(p.y, (size_t)(b0 + sub) * p.y_stride + r, out, IO);
}

template <int IO, int N, bool DIAG>
int launch(const TokenParams &p, hipStream_t stream)
{
    constexpr unsigned ROWS = 1024 / N;
    const unsigned gx = ((unsigned)p.H * p.P + ROWS - 1) / ROWS;
    // four rows to a workgroup where that leaves four workgroups for every compute unit
    if ((size_t)gx * p.rows >= 4096) hipLaunchKernelGGL((selective_step_kernel<IO, N, DIAG, 4>), dim3(gx, (p.rows + 3) / 4), dim3(256), 0, stream, p);
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
